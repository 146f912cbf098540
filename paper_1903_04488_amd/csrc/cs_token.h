// What the entry points of token log probabilities and their kernels (one translation unit a type of logits) share.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "cs_rows.h"
#include "csketch.h"

namespace cs {

constexpr int kMaxTop = CS_TOKEN_MAX_TOP;
constexpr int kMaxParts = 64;                // workgroups that share a row

// A row's (or part's) sums relative to its largest value m: S = sum 2^((x - m) k), U = sum 2^((x - m) k) (x - m) k.
struct Sums {
    float m, S, U;
};

// Where a part of a row leaves what it found: parts x top keys (0: none), then parts x 3 sums
struct Parts {
    uint64_t* key;
    Sums* sums;
};
struct TokenOut {
    float *logp, *entropy, *lse;
    int64_t* top_idx;
    float* top_logp;
};

constexpr int64_t kTokenMaxVocab = static_cast<int64_t>(1) << 30;
constexpr int64_t kTokenMaxRows = (static_cast<int64_t>(1) << 24) - 1;   // (a launch has fewer than 2^32 threads)

inline bool token_ok(int64_t rows, int64_t vocab, int64_t stride, int32_t fmt, float scale) {
    return rows_ok(rows, vocab, stride, fmt) && vocab <= kTokenMaxVocab && rows <= kTokenMaxRows && scale > 0.f && scale < INFINITY;
}
inline int32_t packs_of(int64_t vocab, int32_t fmt) {
    const int64_t p = 16 / fmt_bytes(fmt);
    return static_cast<int32_t>((vocab + p - 1) / p);
}
// Workgroups of 256 threads take a row each where there are enough rows; few rows have workgroups of 1024 (us, 1000 x 60000 bf16
// 26 / 30 with 256; 1500 x 60000 36 / 35), and long ones of them are shared by several (1 x 130000 bf16 in 3 parts 10; a part
// of less than 32768 values cost more for the join than it saved when rows were not held yet: 1 x 32768 f32 with alternatives 41 in 8
// parts, which is 10 in one held row now; smaller parts of held rows have not been measured).
inline bool few_rows(int64_t rows) { return rows < 1024; }
inline int parts_of(int64_t rows, int64_t vocab) {
    if (!few_rows(rows)) return 1;
    int64_t parts = 512 / (rows ? rows : 1);
    if (parts > vocab / 32768) parts = vocab / 32768;
    if (parts > kMaxParts) parts = kMaxParts;
    return static_cast<int>(parts < 1 ? 1 : parts);
}
inline size_t token_bytes(int64_t rows, int64_t vocab, int top) {
    const int64_t parts = parts_of(rows, vocab);
    if (parts == 1) return 0;
    return static_cast<size_t>(rows * parts) * (sizeof(Sums) + static_cast<size_t>(top) * 8);
}
inline Parts parts_in(void* ws, int64_t rows, int parts, int top) {
    Parts p;
    p.key = static_cast<uint64_t*>(ws);
    p.sums = reinterpret_cast<Sums*>(p.key + rows * parts * top);
    return p;
}

struct TokenArgs {
    const void* logits;
    int64_t rows, vocab, stride;
    int32_t fmt;
    float scale;
    const int64_t* target;
    TokenOut out;
    int top;
    void* ws;
    const float *lse, *entropy, *g_logp, *g_entropy;
    void* dlogits;
    int64_t d_stride;
    hipStream_t stream;
};

enum TokenCall { kTokenForward, kTokenGrad, kTokenLoss };
int token_f32(TokenCall call, const TokenArgs& a);
int token_bf16(TokenCall call, const TokenArgs& a);
int token_f16(TokenCall call, const TokenArgs& a);

}  // namespace cs

// Log probabilities of given tokens under rows of logits, with the entropy and the largest alternatives of every row,
// and the gradient of log probability and entropy.  With z = scale x:
//     lse = ln sum exp z,  logp = z_t - lse,  H = lse - sum p z,  p = exp(z - lse)
//     dx_v = scale (g ([v = t] - p_v) - h p_v (ln p_v + H))
// One pass over a row keeps a running reference B, s = sum 2^d and u = sum 2^d d with d = x k - B, k = scale log2(e): one
// fused multiply-add, one exponential and two accumulations a value, all in binary32.  B is a binary32 number that is at
// least k times the largest value so far (up to rounding), so d is exact up to one rounding of its own size however
// large the logits are.
#include <hip/hip_runtime.h>
#include <float.h>
#include <stdint.h>

#include "cs_rows.h"
#include "csketch.h"

namespace cs {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxTop = CS_TOKEN_MAX_TOP;
constexpr int kList = 1024;                  // candidates for the alternatives of a part
constexpr int kMaxParts = 64;                // workgroups that share a row
constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.69314718055994531f;
constexpr float kFar = -200.f;               // 2^kFar is 0 beside any sum

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// A row's (or part's) sums relative to its largest value m: S = sum 2^((x - m) k), U = sum 2^((x - m) k) (x - m) k.
struct Sums {
    float m, S, U;
};

// candidates before others: larger values first, among equal ones the lower index; a NaN counts as -inf
__device__ __forceinline__ float ranked(float v) { return v == v ? v : -INFINITY; }

struct TokenShared {
    float f[3][16];
    float value[kThreads];
    int32_t pack[kThreads];
    int32_t chosen[kMaxTop];
    float list_value[kList];
    int64_t list_at[kList];
    int32_t n;
    float best_value[16];
    int64_t best_at[16];
};

__device__ __forceinline__ float block_max(float v, float (&buf)[16]) {
    v = wave_max(v);
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
    __syncthreads();
    v = buf[0];
#pragma unroll
    for (int w = 1; w < kThreads / 64; ++w) v = fmaxf(v, buf[w]);
    return v;
}
// (buffers of its own: no barrier before)
__device__ __forceinline__ void block_add2(float& a, float& b, float (&ba)[16], float (&bb)[16]) {
    a = wave_sum(a);
    b = wave_sum(b);
    if ((threadIdx.x & 63) == 0) {
        ba[threadIdx.x >> 6] = a;
        bb[threadIdx.x >> 6] = b;
    }
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) {
        a += ba[w];
        b += bb[w];
    }
}

// What a thread has seen of its part of a row: packs first, first + kThreads, ...
template <typename T, bool TOP>
struct Scan {
    static constexpr int P = kPack<T>;
    float B = -FLT_MAX, s = 0.f, u = 0.f, most = -INFINITY, best = -INFINITY;
    int32_t best_pack = INT32_MAX;

    __device__ __forceinline__ void meet(const float (&v)[P], float k, int32_t pack) {
        float top = fmaxf(v[0], v[1]);
#pragma unroll
        for (int e = 2; e < P; e += 2) top = fmaxf(fmaxf(v[e], v[e + 1]), top);
        if (TOP) {
            // (the first pack counts also where it holds nothing above -inf)
            if (top > best || best_pack == INT32_MAX) {
                best = ranked(top);
                best_pack = pack;
            }
        } else {
            most = fmaxf(most, top);
        }
        const float b = top * k;
        if (b > B) {
            const float f = exp2_of(B - b);
            u = f * fmaf(s, fmaxf(B - b, kFar), u);
            s *= f;
            B = b;
        }
#pragma unroll
        for (int e = 0; e < P; ++e) {
            const float d = fmaf(v[e], k, -B), x = exp2_of(d);
            s += x;
            u = fmaf(x, fmaxf(d, kFar), u);
        }
    }
    __device__ __forceinline__ float largest() const { return TOP ? best : most; }
};

// the last pack of a row, where the row ends inside it
template <typename T>
__device__ __forceinline__ void load_tail(const T* row, int64_t at, int64_t vocab, float (&v)[kPack<T>]) {
#pragma unroll
    for (int e = 0; e < kPack<T>; ++e) v[e] = at + e < vocab ? static_cast<float>(row[at + e]) : -INFINITY;
}

// Packs [first, last) of a row (`last` may be one that the row ends in).
template <typename T, bool TOP>
__device__ __forceinline__ Sums scan_part(const T* row, int64_t vocab, int32_t first, int32_t last, float k, TokenShared& sh,
                                          Scan<T, TOP>& scan) {
    constexpr int P = kPack<T>;
    const int32_t whole = static_cast<int32_t>(vocab / P);         // packs before one that the row ends in
    const int32_t stop = last < whole ? last : whole;
    for (int32_t q = first + static_cast<int32_t>(threadIdx.x); q < stop; q += kThreads) {
        float v[P];
        load_pack<T, P>(row + static_cast<int64_t>(q) * P, v);
        scan.meet(v, k, q);
    }
    if (last > whole && first <= whole && (whole - first) % kThreads == static_cast<int32_t>(threadIdx.x)) {
        float v[P];
        load_tail(row, static_cast<int64_t>(whole) * P, vocab, v);
        scan.meet(v, k, whole);
    }
    Sums r;
    r.m = block_max(scan.largest(), sh.f[0]);
    const float B = block_max(scan.B, sh.f[1]);
    __syncthreads();
    const float f = exp2_of(scan.B - B);
    float s = scan.s * f, u = f * fmaf(scan.s, fmaxf(scan.B - B, kFar), scan.u);
    block_add2(s, u, sh.f[0], sh.f[2]);
    // from B to the largest value itself
    const float off = fmaf(r.m, k, -B), g = exp2_of(-off);
    r.S = s * g;
    r.U = g * fmaf(-off, s, u);
    // Where the reference leaves binary32 (values beyond 2e38: masks of the type's lowest value in a row that has nothing
    // else) and where the row holds a NaN or +inf, once more with differences of the values themselves.  (The largest
    // value adds 1 to S.)
    if (!(r.S >= 0.5f && r.S < INFINITY) && r.m > -INFINITY) {
        __syncthreads();
        s = u = 0.f;
        const int64_t end = static_cast<int64_t>(last) * P < vocab ? static_cast<int64_t>(last) * P : vocab;
        for (int64_t i = static_cast<int64_t>(first) * P + threadIdx.x; i < end; i += kThreads) {
            const float d = (static_cast<float>(row[i]) - r.m) * k, x = exp2_of(d);
            s += x;
            u = fmaf(x, fmaxf(d, kFar), u);
        }
        block_add2(s, u, sh.f[0], sh.f[2]);
        r.S = s;
        r.U = u;
    } else if (r.m == -INFINITY && !(s == s)) {      // NaN and -inf alone
        r.S = r.U = s;
    } else if (r.m == -INFINITY) {
        r.S = r.U = 0.f;
    }
    return r;
}

// The `top` largest of packs [first, last) of a row, in order, by `emit(rank, value, index)`.  Of the threads' largest values
// the top-th in order (equal ones: lower pack first) is a bound that `top` values reach, so the largest are
// among those of the `top` threads before it that reach it too: usually hardly more than `top` values, which are
// then ranked by counting.
template <typename T, typename Emit>
__device__ __forceinline__ void largest_of_part(const T* row, int64_t vocab, int32_t first, int32_t last, int top,
                                                const Scan<T, true>& scan, TokenShared& sh, Emit emit) {
    constexpr int P = kPack<T>;
    const int tid = threadIdx.x;
    sh.value[tid] = scan.best;
    sh.pack[tid] = scan.best_pack;
    if (tid == 0) sh.n = 0;
    __syncthreads();
    int rank = 0;
    for (int j = 0; j < kThreads; ++j) {
        const float v = sh.value[j];
        const int32_t q = sh.pack[j];
        // (threads without a pack have none to lose: by their number)
        rank += v > scan.best || (v == scan.best && (q < scan.best_pack || (q == scan.best_pack && j < tid)));
    }
    if (rank < top) sh.chosen[rank] = tid;
    __syncthreads();
    const float bound = sh.value[sh.chosen[top - 1]];
    const int32_t bound_pack = sh.pack[sh.chosen[top - 1]];
    const int32_t each = (last - first + kThreads - 1) / kThreads;         // packs of a thread
    // (pack q of candidate number w, and whether it exists)
    auto pack_of = [&](int32_t w) { return first + sh.chosen[w / each] + (w % each) * kThreads; };
    for (int32_t w = tid; w < top * each; w += kThreads) {
        const int32_t q = pack_of(w);
        if (q >= last) continue;
        const int64_t at = static_cast<int64_t>(q) * P;
        float v[P];
        if (at + P <= vocab) load_pack<T, P>(row + at, v);
        else load_tail(row, at, vocab, v);
#pragma unroll
        for (int e = 0; e < P; ++e) {
            const float x = ranked(v[e]);
            if (at + e < vocab && (x > bound || (x == bound && q <= bound_pack))) {
                const int32_t slot = atomicAdd(&sh.n, 1);
                if (slot < kList) {
                    sh.list_value[slot] = x;
                    sh.list_at[slot] = at + e;
                }
            }
        }
    }
    __syncthreads();
    const int32_t n = sh.n;
    if (n <= kList) {
        for (int32_t i = tid; i < n; i += kThreads) {
            const float x = sh.list_value[i];
            const int64_t at = sh.list_at[i];
            int32_t before = 0;
            for (int32_t j = 0; j < n; ++j) {
                const float v = sh.list_value[j];
                before += v > x || (v == x && sh.list_at[j] < at);
            }
            if (before < top) emit(before, x, at);
        }
        for (int32_t i = n + tid; i < top; i += kThreads) emit(i, -INFINITY, static_cast<int64_t>(-1));
        return;
    }
    // More than the list holds (long runs of equal values): one after the other, each the first behind the one before.
    float prev = INFINITY;
    int64_t prev_at = -1;
    for (int r = 0; r < top; ++r) {
        float best = -INFINITY;
        int64_t best_at = INT64_MAX;
        for (int32_t w = tid; w < top * each; w += kThreads) {
            const int32_t q = pack_of(w);
            if (q >= last) continue;
            const int64_t at = static_cast<int64_t>(q) * P;
            for (int e = 0; e < P && at + e < vocab; ++e) {
                const float x = ranked(static_cast<float>(row[at + e]));
                if ((x < prev || (x == prev && at + e > prev_at)) && (x > best || (x == best && at + e < best_at))) {
                    best = x;
                    best_at = at + e;
                }
            }
        }
#pragma unroll
        for (int d = 32; d; d >>= 1) {
            const float v = __shfl_xor(best, d);
            const int64_t a = __shfl_xor(best_at, d);
            if (v > best || (v == best && a < best_at)) {
                best = v;
                best_at = a;
            }
        }
        __syncthreads();
        if ((tid & 63) == 0) {
            sh.best_value[tid >> 6] = best;
            sh.best_at[tid >> 6] = best_at;
        }
        __syncthreads();
        for (int w = 0; w < kThreads / 64; ++w)
            if (sh.best_value[w] > best || (sh.best_value[w] == best && sh.best_at[w] < best_at)) {
                best = sh.best_value[w];
                best_at = sh.best_at[w];
            }
        prev = best;
        prev_at = best_at;
        if (tid == 0) emit(r, best, best_at);
    }
}

// Where a part of a row leaves what it found: parts x 3 sums, then parts x top values, then as many indices (-1: none)
struct Parts {
    Sums* sums;
    float* value;
    int64_t* at;
};
struct TokenOut {
    float *logp, *entropy, *lse;
    int64_t* top_idx;
    float* top_logp;
};

// log probability of value x in a row with sums r; `log_sum` = ln S
__device__ __forceinline__ float logp_of(float x, const Sums& r, float log_sum, float scale) {
    // (x = m = -inf: a row with nothing in it gives nothing any probability)
    return r.m == -INFINITY && r.S == r.S ? -INFINITY : fmaf(x - r.m, scale, -log_sum);
}

template <typename T>
__device__ __forceinline__ void row_results(const T* logits, int64_t vocab, int64_t row, const int64_t* target, float scale,
                                            const Sums& r, float log_sum, const TokenOut& out) {
    const bool empty = r.m == -INFINITY && r.S == r.S;
    if (out.lse) out.lse[row] = empty ? -INFINITY : fmaf(r.m, scale, log_sum);
    if (out.entropy) out.entropy[row] = empty ? 0.f : log_sum - kLn2 * (r.U / r.S);
    if (out.logp) {
        const int64_t t = target[row];
        const bool counts = t >= 0 && t < vocab;
        out.logp[row] = counts ? logp_of(static_cast<float>(logits[t]), r, log_sum, scale) : 0.f;
    }
}

template <typename T, bool TOP>
__global__ void __launch_bounds__(kThreads)
k_token(const T* logits, int64_t vocab, int64_t stride, float scale, const int64_t* target, TokenOut out, int top, int parts,
        int32_t packs, Parts ws) {
    __shared__ TokenShared sh;
    const int64_t row = blockIdx.x / static_cast<unsigned>(parts);
    const int part = blockIdx.x % static_cast<unsigned>(parts);
    const T* x = logits + row * stride;
    const int32_t each = (packs + parts - 1) / parts;
    const int32_t first = min(part * each, packs), last = min(first + each, packs);
    const float k = scale * kLog2e;
    Scan<T, TOP> scan;
    const Sums r = scan_part<T, TOP>(x, vocab, first, last, k, sh, scan);
    const float log_sum = logf(r.S);
    const int64_t at = row * parts + part;
    if (threadIdx.x == 0) {
        if (parts > 1) ws.sums[at] = r;
        else row_results(x, vocab, row, target, scale, r, log_sum, out);
    }
    if constexpr (TOP) {
        largest_of_part<T>(x, vocab, first, last, top, scan, sh, [&](int rank, float v, int64_t i) {
            if (parts > 1) {
                ws.value[at * top + rank] = v;
                ws.at[at * top + rank] = i;
            } else {
                out.top_idx[row * top + rank] = i;
                out.top_logp[row * top + rank] = logp_of(v, r, log_sum, scale);
            }
        });
    }
}

// a row's parts joined
template <typename T, bool TOP>
__global__ void __launch_bounds__(kThreads)
k_token_join(const T* logits, int64_t vocab, int64_t stride, float scale, const int64_t* target, TokenOut out, int top,
             int parts, Parts ws) {
    __shared__ float value[kMaxParts * kMaxTop];
    __shared__ int64_t index[kMaxParts * kMaxTop];
    __shared__ int32_t n;
    const int64_t row = blockIdx.x;
    const float k = scale * kLog2e;
    const int lane = threadIdx.x & 63;
    // every wavefront joins the sums for itself: a part a lane
    Sums p = {-INFINITY, 0.f, 0.f};
    if (lane < parts) p = ws.sums[row * parts + lane];
    Sums r;
    r.m = wave_max(p.m);
    const float d = p.m == r.m ? 0.f : (p.m - r.m) * k, f = exp2_of(d);
    r.S = wave_sum(p.S * f);
    r.U = wave_sum(f * fmaf(p.S, fmaxf(d, kFar), p.U));
    const float log_sum = logf(r.S);
    if (threadIdx.x == 0) row_results(logits + row * stride, vocab, row, target, scale, r, log_sum, out);
    if (TOP) {
        if (threadIdx.x == 0) n = 0;
        // `top` values reach the last one of any part's list
        float bound = -INFINITY;
        if (lane < parts) bound = ws.value[(row * parts + lane) * top + top - 1];
        bound = wave_max(bound);
        __syncthreads();
        for (int i = threadIdx.x; i < parts * top; i += kThreads) {
            const float v = ws.value[row * parts * top + i];
            const int64_t at = ws.at[row * parts * top + i];
            if (at >= 0 && v >= bound) {
                const int32_t slot = atomicAdd(&n, 1);
                value[slot] = v;
                index[slot] = at;
            }
        }
        __syncthreads();
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const float v = value[i];
            const int64_t at = index[i];
            int before = 0;
            for (int j = 0; j < n; ++j) before += value[j] > v || (value[j] == v && index[j] < at);
            if (before < top) {
                out.top_idx[row * top + before] = at;
                out.top_logp[row * top + before] = logp_of(v, r, log_sum, scale);
            }
        }
    }
}

// Gradient of a value: constants of its row.  ln p = x scale - lse.
struct RowGrad {
    float scale, lse, H, g, h;       // g = 0 where the row has no target
    int64_t target;
    bool empty;
    __device__ __forceinline__ RowGrad(int64_t row, int64_t vocab, float scale_, const int64_t* target_, float lse_, float H_,
                                       const float* g_logp, const float* g_entropy)
        : scale(scale_), lse(lse_), H(H_), g(0.f), h(g_entropy ? g_entropy[row] : 0.f), target(target_ ? target_[row] : -1),
          empty(lse_ == -INFINITY) {
        if (target < 0 || target >= vocab) target = -1;
        else if (g_logp) g = g_logp[row];
    }
    __device__ __forceinline__ float of(float x, bool is_target) const {
        const float l = fmaf(x, scale, -lse), p = exp2_of(l * kLog2e);
        // p (ln p + H) of a value with no probability is 0
        float d = -p * fmaf(h, fmaxf(l, kFar) + H, g);
        if (is_target) d += g;
        return empty ? 0.f : d * scale;
    }
};

template <bool PAST, typename T>
__device__ __forceinline__ void grad_packs(const T* x, T* dx, int64_t vocab, int64_t first, int64_t last, const RowGrad& row) {
    constexpr int P = kPack<T>;
    for (int64_t q = first + threadIdx.x; q < last; q += kThreads) {
        const int64_t at = q * P;
        float v[P];
        if (at + P <= vocab) {
            load_pack<T, P>(x + at, v);
#pragma unroll
            for (int e = 0; e < P; ++e) v[e] = row.of(v[e], at + e == row.target);
            store_pack<PAST>(dx + at, v);
        } else {
            for (int64_t i = at; i < vocab; ++i) dx[i] = static_cast<T>(row.of(static_cast<float>(x[i]), i == row.target));
        }
    }
}

template <typename T, bool PAST>
__global__ void __launch_bounds__(kThreads)
k_token_grad(const T* logits, int64_t vocab, int64_t stride, float scale, const int64_t* target, const float* lse,
             const float* entropy, const float* g_logp, const float* g_entropy, T* dlogits, int64_t d_stride, int pieces,
             int64_t packs) {
    const int64_t row = blockIdx.x / static_cast<unsigned>(pieces);
    const int64_t each = (packs + pieces - 1) / pieces, first = each * (blockIdx.x % static_cast<unsigned>(pieces));
    const RowGrad r(row, vocab, scale, target, lse[row], entropy ? entropy[row] : 0.f, g_logp, g_entropy);
    grad_packs<PAST>(logits + row * stride, dlogits + row * d_stride, vocab, first, min(first + each, packs), r);
}

// forward and gradient of a row in one workgroup: the row's second read comes from the caches
template <typename T, bool PAST>
__global__ void __launch_bounds__(kThreads)
k_token_loss(const T* logits, int64_t vocab, int64_t stride, float scale, const int64_t* target, TokenOut out,
             const float* g_logp, const float* g_entropy, T* dlogits, int64_t d_stride, int32_t packs) {
    __shared__ TokenShared sh;
    const int64_t row = blockIdx.x;
    const T* x = logits + row * stride;
    Scan<T, false> scan;
    const Sums r = scan_part<T, false>(x, vocab, 0, packs, scale * kLog2e, sh, scan);
    const float log_sum = logf(r.S);
    const bool empty = r.m == -INFINITY && r.S == r.S;
    if (threadIdx.x == 0) row_results(x, vocab, row, target, scale, r, log_sum, out);
    __syncthreads();                                  // (dlogits may be the logits, whose target has been read)
    const RowGrad g(row, vocab, scale, target, empty ? -INFINITY : fmaf(r.m, scale, log_sum),
                    empty ? 0.f : log_sum - kLn2 * (r.U / r.S), g_logp, g_entropy);
    grad_packs<PAST>(x, dlogits + row * d_stride, vocab, 0, packs, g);
}

// ---------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------
constexpr int64_t kTokenMaxVocab = static_cast<int64_t>(1) << 30, kTokenMaxRows = static_cast<int64_t>(1) << 24;

bool token_ok(int64_t rows, int64_t vocab, int64_t stride, int32_t fmt, float scale) {
    return rows_ok(rows, vocab, stride, fmt) && vocab <= kTokenMaxVocab && rows <= kTokenMaxRows && scale > 0.f && scale < INFINITY;
}
int32_t packs_of(int64_t vocab, int32_t fmt) {
    const int64_t p = 16 / fmt_bytes(fmt);
    return static_cast<int32_t>((vocab + p - 1) / p);
}
// workgroups that share a row: so many that 512 are under way, none with less than 4096 values
int parts_of(int64_t rows, int64_t vocab) {
    int64_t parts = rows >= 512 ? 1 : 512 / (rows ? rows : 1);
    if (parts > vocab / 4096) parts = vocab / 4096;
    if (parts > kMaxParts) parts = kMaxParts;
    return static_cast<int>(parts < 1 ? 1 : parts);
}
size_t token_bytes(int64_t rows, int64_t vocab, int top) {
    const int64_t parts = parts_of(rows, vocab);
    if (parts == 1) return 0;
    return static_cast<size_t>(rows * parts) * (16 + static_cast<size_t>(top) * 12);
}
Parts parts_in(void* ws, int64_t rows, int parts, int top) {
    Parts p;
    p.at = static_cast<int64_t*>(ws);
    p.value = reinterpret_cast<float*>(p.at + rows * parts * top);
    p.sums = reinterpret_cast<Sums*>(p.value + rows * parts * top);
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

template <typename T, bool TOP>
int token_forward(const TokenArgs& a) {
    const int parts = parts_of(a.rows, a.vocab);
    const Parts ws = parts > 1 ? parts_in(a.ws, a.rows, parts, a.top) : Parts{};
    const T* x = static_cast<const T*>(a.logits);
    k_token<T, TOP><<<static_cast<unsigned>(a.rows * parts), kThreads, 0, a.stream>>>(
        x, a.vocab, a.stride, a.scale, a.target, a.out, a.top, parts, packs_of(a.vocab, a.fmt), ws);
    if (int rc = launched()) return rc;
    if (parts == 1) return CS_OK;
    k_token_join<T, TOP><<<static_cast<unsigned>(a.rows), kThreads, 0, a.stream>>>(x, a.vocab, a.stride, a.scale, a.target,
                                                                                  a.out, a.top, parts, ws);
    return launched();
}
template <typename T>
int token_grad(const TokenArgs& a) {
    const int64_t packs = packs_of(a.vocab, a.fmt);
    const int64_t most = ((static_cast<int64_t>(1) << 31) - 1) / a.rows;
    int64_t pieces = (packs + 4 * kThreads - 1) / (4 * kThreads);
    if (pieces > most) pieces = most;
    const auto kernel = past_caches(a.rows * a.vocab * sizeof(T)) ? k_token_grad<T, true> : k_token_grad<T, false>;
    kernel<<<static_cast<unsigned>(a.rows * pieces), kThreads, 0, a.stream>>>(
        static_cast<const T*>(a.logits), a.vocab, a.stride, a.scale, a.target, a.lse, a.entropy, a.g_logp, a.g_entropy,
        static_cast<T*>(a.dlogits), a.d_stride, static_cast<int>(pieces), packs);
    return launched();
}
template <typename T>
int token_loss(TokenArgs a) {
    if (parts_of(a.rows, a.vocab) > 1) {              // few rows
        if (int rc = token_forward<T, false>(a)) return rc;
        a.lse = a.out.lse, a.entropy = a.out.entropy;
        return token_grad<T>(a);
    }
    const auto kernel = past_caches(a.rows * a.vocab * sizeof(T)) ? k_token_loss<T, true> : k_token_loss<T, false>;
    kernel<<<static_cast<unsigned>(a.rows), kThreads, 0, a.stream>>>(
        static_cast<const T*>(a.logits), a.vocab, a.stride, a.scale, a.target, a.out, a.g_logp, a.g_entropy,
        static_cast<T*>(a.dlogits), a.d_stride, packs_of(a.vocab, a.fmt));
    return launched();
}

#define CS_BY_FMT(fmt, F, ...)                                        \
    ((fmt) == CS_FMT_F32    ? F<float __VA_OPT__(, ) __VA_ARGS__>(a)  \
     : (fmt) == CS_FMT_BF16 ? F<bf16 __VA_OPT__(, ) __VA_ARGS__>(a)   \
                            : F<f16 __VA_OPT__(, ) __VA_ARGS__>(a))

struct Span {
    const void* p;
    int64_t bytes;
};
// no two of the arrays that are written may meet, and none may meet one that is read
template <int NW, int NR>
bool spans_apart(const Span (&written)[NW], const Span (&read)[NR]) {
    for (int i = 0; i < NW; ++i) {
        for (int j = 0; j < i; ++j)
            if (spans_meet(written[i].p, written[i].bytes, written[j].p, written[j].bytes)) return false;
        for (int j = 0; j < NR; ++j)
            if (spans_meet(written[i].p, written[i].bytes, read[j].p, read[j].bytes)) return false;
    }
    return true;
}
int64_t row_span(int64_t rows, int64_t vocab, int64_t stride, int32_t fmt) {
    return rows > 0 ? ((rows - 1) * stride + vocab) * fmt_bytes(fmt) : 0;
}
// dlogits may be the logits themselves, value for value, and must not meet them otherwise
bool dlogits_ok(const TokenArgs& a) {
    if (!a.dlogits || !rows_ok(a.rows, a.vocab, a.d_stride, a.fmt)) return false;
    if (a.dlogits == a.logits && (a.d_stride == a.stride || a.rows == 1)) return true;
    const int64_t b = fmt_bytes(a.fmt);
    return !rows_meet(a.dlogits, a.d_stride * b, a.logits, a.stride * b, a.rows, a.vocab * b);
}

}  // namespace
}  // namespace cs

using namespace cs;

extern "C" int cs_token_workspace_bytes(int64_t rows, int64_t vocab, int32_t top, size_t* bytes) {
    if (rows < 0 || rows > kTokenMaxRows || vocab < 1 || vocab > kTokenMaxVocab || top < 0 || top > kMaxTop || top > vocab || !bytes)
        return CS_EINVAL;
    *bytes = token_bytes(rows, vocab, top);
    return CS_OK;
}

extern "C" int cs_token_logprobs(const void* logits, int64_t rows, int64_t vocab, int64_t stride, int32_t fmt, float scale,
                                 const int64_t* target, float* logp, float* entropy, float* lse, int32_t top,
                                 int64_t* top_idx, float* top_logp, void* workspace, size_t ws_bytes, void* stream) {
    if (!token_ok(rows, vocab, stride, fmt, scale) || top < 0 || top > kMaxTop || top > vocab) return CS_EINVAL;
    if ((logp && !target) || (top && (!top_idx || !top_logp))) return CS_EINVAL;
    if (rows == 0) return CS_OK;
    if (!logits) return CS_EINVAL;
    const size_t need = token_bytes(rows, vocab, top);
    if (ws_bytes < need) return CS_EWORKSPACE;
    if (need && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 7))) return CS_EINVAL;
    const Span written[] = {{logp, 4 * rows}, {entropy, 4 * rows}, {lse, 4 * rows}, {top ? top_idx : nullptr, 8 * rows * top},
                            {top ? top_logp : nullptr, 4 * rows * top}, {need ? workspace : nullptr, static_cast<int64_t>(need)}};
    const Span read[] = {{logits, row_span(rows, vocab, stride, fmt)}, {logp ? target : nullptr, 8 * rows}};
    if (!spans_apart(written, read)) return CS_EINVAL;
    TokenArgs a = {};
    a.logits = logits, a.rows = rows, a.vocab = vocab, a.stride = stride, a.fmt = fmt, a.scale = scale, a.target = target;
    a.out = TokenOut{logp, entropy, lse, top_idx, top_logp}, a.top = top, a.ws = workspace, a.stream = stream_of(stream);
    return top ? CS_BY_FMT(fmt, token_forward, true) : CS_BY_FMT(fmt, token_forward, false);
}

extern "C" int cs_token_logprobs_grad(const void* logits, int64_t rows, int64_t vocab, int64_t stride, int32_t fmt,
                                      float scale, const int64_t* target, const float* lse, const float* entropy,
                                      const float* g_logp, const float* g_entropy, void* dlogits, int64_t d_stride,
                                      void* stream) {
    if (!token_ok(rows, vocab, stride, fmt, scale) || (g_logp && !target) || (g_entropy && !entropy)) return CS_EINVAL;
    if (rows == 0) return CS_OK;
    TokenArgs a = {};
    a.logits = logits, a.rows = rows, a.vocab = vocab, a.stride = stride, a.fmt = fmt, a.scale = scale, a.target = target;
    a.lse = lse, a.entropy = g_entropy ? entropy : nullptr, a.g_logp = g_logp, a.g_entropy = g_entropy;
    a.dlogits = dlogits, a.d_stride = d_stride, a.stream = stream_of(stream);
    if (!logits || !lse || !dlogits_ok(a)) return CS_EINVAL;
    const Span written[] = {{dlogits, row_span(rows, vocab, d_stride, fmt)}};
    const Span read[] = {{target, 8 * rows}, {lse, 4 * rows}, {a.entropy, 4 * rows}, {g_logp, 4 * rows}, {g_entropy, 4 * rows}};
    if (!spans_apart(written, read)) return CS_EINVAL;
    return CS_BY_FMT(fmt, token_grad);
}

extern "C" int cs_token_loss(const void* logits, int64_t rows, int64_t vocab, int64_t stride, int32_t fmt, float scale,
                             const int64_t* target, const float* g_logp, const float* g_entropy, float* logp,
                             float* entropy, float* lse, void* dlogits, int64_t d_stride, void* workspace, size_t ws_bytes,
                             void* stream) {
    if (!token_ok(rows, vocab, stride, fmt, scale)) return CS_EINVAL;
    if (rows == 0) return CS_OK;
    if (!logits || !target || !g_logp || !logp || !entropy || !lse) return CS_EINVAL;
    const size_t need = token_bytes(rows, vocab, 0);
    if (ws_bytes < need) return CS_EWORKSPACE;
    if (need && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 7))) return CS_EINVAL;
    TokenArgs a = {};
    a.logits = logits, a.rows = rows, a.vocab = vocab, a.stride = stride, a.fmt = fmt, a.scale = scale, a.target = target;
    a.out = TokenOut{logp, entropy, lse, nullptr, nullptr}, a.ws = workspace, a.g_logp = g_logp, a.g_entropy = g_entropy;
    a.dlogits = dlogits, a.d_stride = d_stride, a.stream = stream_of(stream);
    if (!dlogits_ok(a)) return CS_EINVAL;
    const Span written[] = {{logp, 4 * rows}, {entropy, 4 * rows}, {lse, 4 * rows}, {need ? workspace : nullptr, static_cast<int64_t>(need)}};
    const Span read[] = {{logits, row_span(rows, vocab, stride, fmt)}, {dlogits, row_span(rows, vocab, d_stride, fmt)},
                         {target, 8 * rows}, {g_logp, 4 * rows}, {g_entropy, 4 * rows}};
    const Span grad[] = {{dlogits, row_span(rows, vocab, d_stride, fmt)}};
    const Span rest[] = {{target, 8 * rows}, {g_logp, 4 * rows}, {g_entropy, 4 * rows}};
    if (!spans_apart(written, read) || !spans_apart(grad, rest)) return CS_EINVAL;
    return CS_BY_FMT(fmt, token_loss);
}

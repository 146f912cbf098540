// Matrices orthogonalised by Newton-Schulz products, and the optimizer step that does this with their momentum.
//     m = mu m + s g,  u = s g + mu m (nesterov) or m,  X = u / (|u|_F + eps)
//     steps times:  A = X X^T,  B = b A + c A A,  X = a X + B X          (on the shorter side: of a tall matrix with u^T)
//     p = p (1 - lr wd) - lr scale X
// Every step maps the singular values s to a s + b s^3 + c s^5 and leaves the singular vectors.
//
// Numbers.  The products take binary16 (11 bits) into binary32 sums, which is the matrix units' full rate; what goes past the
// products is kept longer, because the polynomial's slope raises relative errors near 1 and singular values a hundred times smaller
// than the largest are raised from step to step: X is held as the sum of two binary16 (22 bits), and A and B without
// their diagonals, which are binary32 and enter by
//     (A A)_ij = (A0 A0)_ij + (d_i + d_j) A0_ij + [i = j] d_i^2,   (B X)_ij = (B0 X)_ij + e_i X_ij.
// Of 512 x 512 to 1024 x 1024 with a flat, a stepped and a 1/k spectrum the result is 2.4e-4 to 8e-4 off (all of it in 11 bits: 1e-3 to
// 4e-3; in bfloat16: 1e-2 to 3e-2): less than half a step of bfloat16.  terms = 2 splits A0, B0 and X in all products (hi hi + hi lo +
// lo hi) and is as exact as products in binary32.  Everything is stored 2^10 times: entries of X, A and B are below 64.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "cs_rows.h"
#include "csketch.h"

namespace cs {
namespace {

constexpr int kThreads = 256;
constexpr int kEdge = 64;                    // of the pieces in which u is read, and what all sizes are rounded up to
constexpr int kDepth = 64;                   // values of K that are in LDS at a time
constexpr float kUp = 1024.f, kDown = 1.f / 1024.f;

typedef _Float16 Half8 __attribute__((ext_vector_type(8)));
typedef float Float4 __attribute__((ext_vector_type(4)));

// One matrix.  n x m: the shorter side first; np, mp: rounded up to whole tiles.
struct Matrix {
    void* p;
    const void* g;
    float* moment;
    int64_t p_stride, g_stride;
    int64_t at;                              // of its part of the workspace, bytes
    int32_t rows, cols, np, mp;
    int32_t first_piece, first_half, first_full, pieces;
};
struct Place {
    int32_t matrix, local;
};
constexpr int kBatch = 40;
struct Batch {
    Matrix t[kBatch];
};
static_assert(sizeof(Batch) < 3800, "kernel arguments are limited to 4 KB");

// A list in device memory: Matrix[count], then the places of all pieces, of the tiles of all lower halves of A, and of all tiles of X.
struct List {
    const Matrix* matrices;
    const Place *pieces, *halves, *fulls;
};

// A matrix's part of the workspace: X, X^T twice (read and written in turns), A0, B0, each as its upper and its lower 11 bits, and the
// diagonals of A and B.  With one term the lower bits of X alone are kept.
template <int TERMS>
struct Work {
    _Float16* base;
    int64_t nm, nn;
    int32_t np;
    __device__ __forceinline__ Work(char* ws, const Matrix& t)
        : base(reinterpret_cast<_Float16*>(ws + t.at)), nm(static_cast<int64_t>(t.np) * t.mp), nn(static_cast<int64_t>(t.np) * t.np), np(t.np) {}
    __device__ __forceinline__ _Float16* x(int low) const { return base + low * nm; }
    __device__ __forceinline__ _Float16* xt(int turn, int low) const { return base + (2 + turn * TERMS + low) * nm; }
    __device__ __forceinline__ _Float16* a(int low) const { return base + (2 + 2 * TERMS) * nm + low * nn; }
    __device__ __forceinline__ _Float16* b(int low) const { return base + (2 + 2 * TERMS) * nm + (TERMS + low) * nn; }
    __device__ __forceinline__ float* da() const { return reinterpret_cast<float*>(base + (2 + 2 * TERMS) * nm + 2 * TERMS * nn); }
    __device__ __forceinline__ float* db() const { return da() + np; }
};
int64_t work_bytes(int64_t np, int64_t mp, int terms) {
    return 2 * ((2 + 2 * terms) * np * mp + 2 * terms * np * np) + 2 * 4 * np;
}

__global__ void __launch_bounds__(64) k_list_matrices(Batch b, Matrix* out, int count) {
    if (static_cast<int>(threadIdx.x) < count) out[threadIdx.x] = b.t[threadIdx.x];
}
// every place's matrix: the last that begins at or before it
__global__ void __launch_bounds__(kThreads) k_list_places(const Matrix* matrices, int count, int which, Place* out, int64_t places) {
    const int64_t c = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    if (c >= places) return;
    const auto first = [&](int i) {
        const Matrix& t = matrices[i];
        return which == 0 ? t.first_piece : which == 1 ? t.first_half : t.first_full;
    };
    int lo = 0, hi = count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (first(mid) <= c) lo = mid;
        else hi = mid - 1;
    }
    out[c] = Place{lo, static_cast<int32_t>(c - first(lo))};
}

template <typename T>
__device__ __forceinline__ float value_at(const void* p, int64_t at) { return static_cast<float>(static_cast<const T*>(p)[at]); }
__device__ __forceinline__ float read(const void* p, int fmt, int64_t at) {
    return fmt == CS_FMT_F32 ? value_at<float>(p, at) : fmt == CS_FMT_BF16 ? value_at<bf16>(p, at) : value_at<f16>(p, at);
}
__device__ __forceinline__ void write(void* p, int fmt, int64_t at, float v) {
    if (fmt == CS_FMT_F32) static_cast<float*>(p)[at] = v;
    else if (fmt == CS_FMT_BF16) static_cast<bf16*>(p)[at] = static_cast<bf16>(v);
    else static_cast<f16*>(p)[at] = static_cast<f16>(v);
}
__device__ __forceinline__ bool skipped(const float* grad_scale) { return grad_scale && !(fabsf(*grad_scale) < INFINITY); }

struct Moment {
    float mu;
    int nesterov;
    const float* grad_scale;
};
// u at an element, with the moment as it is now
__device__ __forceinline__ float direction(const Matrix& t, int g_fmt, const Moment& k, float s, int64_t row, int64_t col) {
    if (!t.moment) return read(t.g, g_fmt, row * t.g_stride + col);
    const float m = t.moment[row * t.cols + col];
    return k.nesterov ? fmaf(k.mu, m, s * read(t.g, g_fmt, row * t.g_stride + col)) : m;
}
// rows and columns [row, row + 64), [col, col + 64) of the matrix as it is given
struct Piece {
    int32_t row, col;
    __device__ Piece(const Matrix& t, int32_t local) {
        const int32_t across = (t.rows <= t.cols ? t.mp : t.np) / kEdge;
        row = local / across * kEdge;
        col = local % across * kEdge;
    }
};

// The moment, and a piece's sum of squares of u (binary64, a fixed order).
__global__ void __launch_bounds__(kThreads) k_muon_moment(List list, int g_fmt, Moment k, double* squares) {
    __shared__ double sums[kThreads / 64];
    const Place at = list.pieces[blockIdx.x];
    const Matrix t = list.matrices[at.matrix];
    const Piece piece(t, at.local);
    const bool skip = skipped(k.grad_scale);
    const float s = k.grad_scale ? *k.grad_scale : 1.f;
    double sum = 0.;
    for (int i = threadIdx.x; i < kEdge * kEdge; i += kThreads) {
        const int64_t row = piece.row + i / kEdge, col = piece.col + i % kEdge;
        if (row < t.rows && col < t.cols && !skip) {
            if (t.moment) {
                float& m = t.moment[row * t.cols + col];
                m = fmaf(k.mu, m, s * read(t.g, g_fmt, row * t.g_stride + col));
            }
            const double u = direction(t, g_fmt, k, s, row, col);
            sum += u * u;
        }
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) squares[blockIdx.x] = sums[0] + sums[1] + sums[2] + sums[3];
}

// A matrix's 1 / (|u| + eps)
__global__ void __launch_bounds__(kThreads) k_muon_norm(List list, double eps, const double* squares, double* inverse) {
    __shared__ double sums[kThreads / 64];
    const Matrix& t = list.matrices[blockIdx.x];
    double sum = 0.;
    for (int i = threadIdx.x; i < t.pieces; i += kThreads) sum += squares[t.first_piece + i];
#pragma unroll
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63) == 0) sums[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        sum = sums[0] + sums[1] + sums[2] + sums[3];
        inverse[blockIdx.x] = sum == 0. ? 0. : 1. / (sqrt(sum) + eps);
    }
}

__device__ __forceinline__ void split(float v, _Float16& hi, _Float16& lo) {
    hi = static_cast<_Float16>(v);
    lo = static_cast<_Float16>(v - static_cast<float>(hi));
}

// X and X^T from u, zero behind the last row and column
template <int TERMS>
__global__ void __launch_bounds__(kThreads) k_muon_begin(List list, int g_fmt, Moment k, const double* inverse, char* ws) {
    __shared__ float tile[kEdge][kEdge + 1];
    const Place at = list.pieces[blockIdx.x];
    const Matrix t = list.matrices[at.matrix];
    const Piece piece(t, at.local);
    const Work<TERMS> w(ws, t);
    const float s = k.grad_scale ? *k.grad_scale : 1.f;
    const double one = inverse[at.matrix] * static_cast<double>(kUp);
    for (int i = threadIdx.x; i < kEdge * kEdge; i += kThreads) {
        const int64_t row = piece.row + i / kEdge, col = piece.col + i % kEdge;
        tile[i / kEdge][i % kEdge] =
            row < t.rows && col < t.cols ? static_cast<float>(direction(t, g_fmt, k, s, row, col) * one) : 0.f;
    }
    __syncthreads();
    const bool tall = t.rows > t.cols;
    // as it is given: X of a wide matrix, X^T of a tall one; and the other way round
    const int64_t across = tall ? t.np : t.mp, down = tall ? t.mp : t.np;
    const auto as_is = [&](int low) { return tall ? w.xt(0, low) : w.x(low); };
    const auto turned = [&](int low) { return tall ? w.x(low) : w.xt(0, low); };
    for (int i = threadIdx.x; i < kEdge * kEdge / 8; i += kThreads) {
        const int r = i / 8, c = i % 8 * 8;
        Half8 hi, lo;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            _Float16 h, l;
            split(tile[r][c + e], h, l);
            hi[e] = h, lo[e] = l;
        }
        int64_t to = (piece.row + r) * across + piece.col + c;
        *reinterpret_cast<Half8*>(as_is(0) + to) = hi;
        if (TERMS == 2 || !tall) *reinterpret_cast<Half8*>(as_is(1) + to) = lo;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            _Float16 h, l;
            split(tile[c + e][r], h, l);
            hi[e] = h, lo[e] = l;
        }
        to = (piece.col + r) * down + piece.row + c;
        *reinterpret_cast<Half8*>(turned(0) + to) = hi;
        if (TERMS == 2 || tall) *reinterpret_cast<Half8*>(turned(1) + to) = lo;
    }
}

enum { kGram, kSquare, kApply, kFinish };    // A = X X^T; B = b A + c A A; X = a X + B X; the same, into the parameters

struct Product {
    float a, b, c;
    int turn;                                // which of the two X^T is read
    // kFinish
    int p_fmt, optimizer, scale_rule;
    float decay, lr, lr_decay;
    const double* lr_now;
    const float* grad_scale;
};

typedef __attribute__((address_space(3))) void* LdsPointer;
typedef const __attribute__((address_space(1))) void* GlobalPointer;

// T rows of kDepth values, `stride` apart, into LDS: a row's eight packs of 16 bytes lie in the order pack ^ (row / 2 % 8), so that 16
// lanes that read the same pack of 16 rows meet all banks once.
template <int T>
__device__ __forceinline__ void stage(const _Float16* from, int64_t stride, _Float16* lds) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
    for (int q = 0; q < T / 32; ++q) {
        const int first = (q * 4 + wave) * 8, row = first + (lane >> 3), pack = (lane & 7) ^ (row >> 1 & 7);
        __builtin_amdgcn_global_load_lds(reinterpret_cast<GlobalPointer>(reinterpret_cast<uintptr_t>(from + row * stride + pack * 8)),
                                         (LdsPointer)(lds + first * kDepth), 16, 0, 0);
    }
}

// C = L R^T of rows of K values, T x T a workgroup of four wavefronts.
template <int T, int TERMS, int MODE>
__global__ void __launch_bounds__(kThreads, 2) k_muon_product(List list, Product k, char* ws) {
    constexpr int F = T / 32, LINE = T + 4;  // blocks of 16 a wavefront and side
    constexpr int kStage = 2 * T * kDepth;   // halves of a turn
    constexpr int kBytes = 2 * kStage * 2 > T * LINE * 4 ? 2 * kStage * 2 : T * LINE * 4;
    __shared__ __align__(16) char memory[kBytes];
    _Float16* const lds = reinterpret_cast<_Float16*>(memory);
    const Place at = (MODE == kGram || MODE == kSquare ? list.halves : list.fulls)[blockIdx.x];
    const Matrix t = list.matrices[at.matrix];
    const Work<TERMS> w(ws, t);
    int32_t ti, tj;
    if (MODE == kGram || MODE == kSquare) {          // tiles of the lower half, row by row
        ti = static_cast<int32_t>((sqrtf(8.f * at.local + 1.f) - 1.f) * 0.5f);
        while (ti * (ti + 1) / 2 > at.local) --ti;
        while ((ti + 1) * (ti + 2) / 2 <= at.local) ++ti;
        tj = at.local - ti * (ti + 1) / 2;
    } else {
        ti = at.local / (t.mp / T);
        tj = at.local % (t.mp / T);
    }
    const int32_t depth = MODE == kGram ? t.mp : t.np;
    const int64_t stride = depth;
    const auto left = [&](int low) { return MODE == kGram ? w.x(low) : MODE == kSquare ? w.a(low) : w.b(low); };
    const auto right = [&](int low) { return MODE == kGram ? w.x(low) : MODE == kSquare ? w.a(low) : w.xt(k.turn, low); };
    const int64_t l_at = static_cast<int64_t>(ti) * T * stride, r_at = static_cast<int64_t>(tj) * T * stride;
    const int32_t per = depth / kDepth, all = per * (TERMS == 2 ? 3 : 1);
    // terms = 2: hi hi, then hi lo, then lo hi
    const auto load = [&](int32_t i) {
        const int32_t part = TERMS == 2 ? i / per : 0, q = TERMS == 2 ? i % per : i;
        _Float16* to = lds + (i & 1) * kStage;
        stage<T>(left(part == 2) + l_at + q * kDepth, stride, to);
        stage<T>(right(part == 1) + r_at + q * kDepth, stride, to + T * kDepth);
    };
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wi = wave >> 1, wj = wave & 1;
    Float4 acc[F][F] = {};
    load(0);
    for (int32_t i = 0; i < all; ++i) {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (i + 1 < all) load(i + 1);
        const _Float16* const l = lds + (i & 1) * kStage + (wi * (T / 2) + (lane & 15)) * kDepth;
        const _Float16* const r = lds + (i & 1) * kStage + T * kDepth + (wj * (T / 2) + (lane & 15)) * kDepth;
#pragma unroll
        for (int q = 0; q < kDepth / 32; ++q) {
            const int pack = (((lane >> 4) + 4 * q) ^ ((lane & 15) >> 1)) * 8;
            Half8 lv[F], rv[F];
#pragma unroll
            for (int f = 0; f < F; ++f) lv[f] = *reinterpret_cast<const Half8*>(l + f * 16 * kDepth + pack);
#pragma unroll
            for (int f = 0; f < F; ++f) rv[f] = *reinterpret_cast<const Half8*>(r + f * 16 * kDepth + pack);
#pragma unroll
            for (int fi = 0; fi < F; ++fi)
#pragma unroll
                for (int fj = 0; fj < F; ++fj) acc[fi][fj] = __builtin_amdgcn_mfma_f32_16x16x32_f16(lv[fi], rv[fj], acc[fi][fj], 0, 0, 0);
        }
    }
    // through LDS, so that memory is met in rows of the output and in rows of its transpose
    __syncthreads();
    float* const tile = reinterpret_cast<float*>(memory);
#pragma unroll
    for (int fi = 0; fi < F; ++fi)
#pragma unroll
        for (int fj = 0; fj < F; ++fj)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                tile[(wi * (T / 2) + fi * 16 + (lane >> 4) * 4 + e) * LINE + wj * (T / 2) + fj * 16 + (lane & 15)] =
                    acc[fi][fj][e] * (kDown * kDown);
    __syncthreads();
    float lr = 0.f, keep = 0.f;
    if (MODE == kFinish) {
        if (skipped(k.grad_scale)) return;
        lr = k.lr, keep = k.decay;
        if (k.lr_now) {
            lr = static_cast<float>(*k.lr_now);
            keep = static_cast<float>(1. - *k.lr_now * k.lr_decay);
        }
        const float ratio = static_cast<float>(t.rows) / static_cast<float>(t.cols);
        lr *= k.scale_rule == CS_MUON_SCALE_SHAPE ? sqrtf(fmaxf(1.f, ratio))
              : k.scale_rule == CS_MUON_SCALE_RMS ? 0.2f * sqrtf(static_cast<float>(max(t.rows, t.cols))) : 1.f;
    }
    const bool tall = t.rows > t.cols;
    const auto finish = [&](int64_t row, int64_t col, float x) {
        if (row >= t.rows || col >= t.cols) return;
        const int64_t to = row * t.p_stride + col;
        write(t.p, k.p_fmt, to, k.optimizer ? fmaf(read(t.p, k.p_fmt, to), keep, -lr * x) : x);
    };
    const int64_t wide = MODE == kGram || MODE == kSquare ? t.np : t.mp;         // of an output row
    for (int i = threadIdx.x; i < T * T / 8; i += kThreads) {
        const int r = i / (T / 8), c = i % (T / 8) * 8, row = ti * T + r, col = tj * T + c;
        const int64_t to = row * wide + col;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = tile[r * LINE + c + e];
        if (MODE == kGram) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (row == col + e) {
                    w.da()[row] = v[e];
                    v[e] = 0.f;
                }
        } else {
            // the elements of A0 or X that go past the product
            const Half8 hi = *reinterpret_cast<const Half8*>((MODE == kSquare ? w.a(0) : w.x(0)) + to);
            Half8 lo = {};
            if (TERMS == 2 || MODE != kSquare) lo = *reinterpret_cast<const Half8*>((MODE == kSquare ? w.a(1) : w.x(1)) + to);
            const float d = MODE == kSquare ? w.da()[row] : k.a + w.db()[row];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = (static_cast<float>(hi[e]) + static_cast<float>(lo[e])) * kDown;
                if (MODE == kSquare) {
                    if (row == col + e) {
                        w.db()[row] = fmaf(k.b, d, k.c * fmaf(d, d, v[e]));
                        v[e] = 0.f;
                    } else {
                        v[e] = fmaf(k.b, x, k.c * fmaf(d + w.da()[col + e], x, v[e]));
                    }
                } else {
                    v[e] = fmaf(d, x, v[e]);
                }
            }
        }
        if (MODE == kFinish) {
            if (!tall)
#pragma unroll
                for (int e = 0; e < 8; ++e) finish(row, col + e, v[e]);
        } else {
            Half8 hi, lo;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                _Float16 h, l;
                split(v[e] * kUp, h, l);
                hi[e] = h, lo[e] = l;
            }
            const auto out = [&](int low) { return MODE == kGram ? w.a(low) : MODE == kSquare ? w.b(low) : w.x(low); };
            *reinterpret_cast<Half8*>(out(0) + to) = hi;
            if (TERMS == 2 || MODE == kApply) *reinterpret_cast<Half8*>(out(1) + to) = lo;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) tile[r * LINE + c + e] = v[e];
    }
    // the transpose: of A and B the tile on the other side, of X the one that the next product reads
    if (((MODE == kGram || MODE == kSquare) && ti == tj) || (MODE == kFinish && !tall)) return;
    __syncthreads();
    const int64_t high = t.np;
    for (int i = threadIdx.x; i < T * T / 8; i += kThreads) {
        const int r = i / (T / 8), c = i % (T / 8) * 8;
        const int64_t row = tj * T + r, col = ti * T + c;
        Half8 hi, lo;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float v = tile[(c + e) * LINE + r];
            if (MODE == kFinish) {
                finish(row, col + e, v);
            } else {
                _Float16 h, l;
                split(v * kUp, h, l);
                hi[e] = h, lo[e] = l;
            }
        }
        if (MODE == kFinish) continue;
        const auto out = [&](int low) { return MODE == kGram ? w.a(low) : MODE == kSquare ? w.b(low) : w.xt(1 - k.turn, low); };
        *reinterpret_cast<Half8*>(out(0) + row * high + col) = hi;
        if (TERMS == 2) *reinterpret_cast<Half8*>(out(1) + row * high + col) = lo;
    }
}

// ---------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------
constexpr int64_t kMaxSide = 1 << 20, kMaxShort = 1 << 15, kMaxMatrices = 1 << 20, kMaxPlaces = static_cast<int64_t>(1) << 24;

struct Plan {
    int64_t matrices, pieces, halves, fulls, work;   // work: bytes of all matrices
    int tile;
};
int64_t up_to(int64_t n, int64_t unit) { return (n + unit - 1) / unit * unit; }

bool stack_ok(const cs_matrix& s) {
    return s.count >= 0 && s.count <= kMaxMatrices && s.rows >= 0 && s.cols >= 0 && s.rows <= kMaxSide && s.cols <= kMaxSide &&
           (s.rows < s.cols ? s.rows : s.cols) <= kMaxShort;
}
// count of matrices that are there, and sizes; `each` is told of every stack
template <typename F>
bool plan_with(const cs_matrix* stacks, int32_t n, int terms, int tile, Plan& plan, F each) {
    plan = Plan{0, 0, 0, 0, 0, tile};
    for (int32_t i = 0; i < n; ++i) {
        const cs_matrix& s = stacks[i];
        if (!stack_ok(s)) return false;
        if (s.count == 0 || s.rows == 0 || s.cols == 0) continue;
        const int64_t np = up_to(s.rows < s.cols ? s.rows : s.cols, tile), mp = up_to(s.rows < s.cols ? s.cols : s.rows, tile);
        const int64_t down = np / tile, pieces = (np / kEdge) * (mp / kEdge), halves = down * (down + 1) / 2, fulls = down * (mp / tile);
        each(s, np, mp, plan, pieces, halves, fulls);
        plan.matrices += s.count;
        plan.pieces += s.count * pieces;
        plan.halves += s.count * halves;
        plan.fulls += s.count * fulls;
        plan.work += s.count * work_bytes(np, mp, terms);
        if (plan.matrices > kMaxMatrices || plan.pieces >= kMaxPlaces) return false;
    }
    return true;
}
bool plan_of(const cs_matrix* stacks, int32_t n, int terms, Plan& plan) {
    const auto none = [](const cs_matrix&, int64_t, int64_t, const Plan&, int64_t, int64_t, int64_t) {};
    if (!plan_with(stacks, n, terms, 128, plan, none)) return false;
    if (plan.halves >= 256) return true;
    return plan_with(stacks, n, terms, 64, plan, none);
}
size_t list_bytes(const Plan& p) {
    return static_cast<size_t>(p.matrices) * sizeof(Matrix) + static_cast<size_t>(p.pieces + p.halves + p.fulls) * sizeof(Place);
}
size_t workspace_bytes(const cs_matrix_list* l) {
    return static_cast<size_t>(l->work) + static_cast<size_t>(l->pieces + l->matrices) * sizeof(double);
}
List list_of(const cs_matrix_list* l) {
    const Matrix* t = static_cast<const Matrix*>(l->memory);
    const Place* at = reinterpret_cast<const Place*>(t + l->matrices);
    return List{t, at, at + l->pieces, at + l->pieces + l->halves};
}
bool list_ok(const cs_matrix_list* l) {
    return l && l->matrices >= 0 && l->pieces >= 0 && l->halves >= 0 && l->fulls >= 0 && l->work >= 0 && (l->tile == 64 || l->tile == 128) &&
           (l->terms == 1 || l->terms == 2) && fmt_ok(l->p_fmt) && fmt_ok(l->g_fmt) && (l->matrices == 0 || l->memory);
}

// The steps keep singular values of at most 1 below 2, and B within binary16.
bool steps_ok(const cs_muon* h) {
    if (h->steps < 1 || h->steps > CS_MUON_MAX_STEPS) return false;
    double most = 1.;
    for (int i = 0; i < h->steps; ++i) {
        const double a = h->coefs[i][0], b = h->coefs[i][1], c = h->coefs[i][2], q = most * most;
        if (!(fabs(a) <= 60. && fabs(b) * q + fabs(c) * q * q <= 60.)) return false;
        const auto f = [&](double s) { return fabs(s * (a + s * s * (b + s * s * c))); };
        double next = f(most);
        // where a + 3 b s^2 + 5 c s^4 is 0
        const double root = 9. * b * b - 20. * a * c;
        const double at[3] = {c != 0. && root >= 0. ? (-3. * b + sqrt(root)) / (10. * c) : -1.,
                              c != 0. && root >= 0. ? (-3. * b - sqrt(root)) / (10. * c) : -1., c == 0. && b != 0. ? -a / (3. * b) : -1.};
        for (const double s : at)
            if (s > 0. && s < q) next = fmax(next, f(sqrt(s)));
        if (!(next <= 2.)) return false;
        most = next;
    }
    return true;
}
bool hyper_ok(const cs_muon* h) {
    const auto fine = [](double x) { return x >= 0. && x < INFINITY; };
    return h && fine(h->lr) && h->momentum >= 0. && h->momentum < 1. && fine(h->weight_decay) && fine(h->eps) && h->scale >= 0 &&
           h->scale <= CS_MUON_SCALE_ONE && steps_ok(h);
}

template <int T, int TERMS>
int run_as(const cs_muon* h, const cs_matrix_list* l, bool optimizer, const double* lr, const float* grad_scale, char* ws, hipStream_t s) {
    const List at = list_of(l);
    double* const squares = reinterpret_cast<double*>(ws + l->work);
    double* const inverse = squares + l->pieces;
    const Moment moment = {static_cast<float>(h->momentum), optimizer ? h->nesterov : 0, grad_scale};
    const unsigned pieces = static_cast<unsigned>(l->pieces), halves = static_cast<unsigned>(l->halves), fulls = static_cast<unsigned>(l->fulls);
    k_muon_moment<<<pieces, kThreads, 0, s>>>(at, l->g_fmt, moment, squares);
    k_muon_norm<<<static_cast<unsigned>(l->matrices), kThreads, 0, s>>>(at, h->eps, squares, inverse);
    k_muon_begin<TERMS><<<pieces, kThreads, 0, s>>>(at, l->g_fmt, moment, inverse, ws);
    if (int rc = launched()) return rc;
    for (int i = 0; i < h->steps; ++i) {
        Product k = {};
        k.a = static_cast<float>(h->coefs[i][0]), k.b = static_cast<float>(h->coefs[i][1]), k.c = static_cast<float>(h->coefs[i][2]);
        k.turn = i & 1;
        k_muon_product<T, TERMS, kGram><<<halves, kThreads, 0, s>>>(at, k, ws);
        k_muon_product<T, TERMS, kSquare><<<halves, kThreads, 0, s>>>(at, k, ws);
        if (i + 1 < h->steps) {
            k_muon_product<T, TERMS, kApply><<<fulls, kThreads, 0, s>>>(at, k, ws);
        } else {
            k.p_fmt = l->p_fmt, k.optimizer = optimizer, k.scale_rule = h->scale;
            k.lr = static_cast<float>(h->lr), k.decay = static_cast<float>(1. - h->lr * h->weight_decay);
            k.lr_decay = static_cast<float>(h->weight_decay);
            k.lr_now = lr, k.grad_scale = grad_scale;
            k_muon_product<T, TERMS, kFinish><<<fulls, kThreads, 0, s>>>(at, k, ws);
        }
        if (int rc = launched()) return rc;
    }
    return CS_OK;
}
int run(const cs_muon* h, const cs_matrix_list* l, bool optimizer, const double* lr, const float* grad_scale, void* workspace, size_t ws_bytes,
        void* stream) {
    if (!hyper_ok(h) || !list_ok(l) || (l->matrices && l->moments != (optimizer ? 1 : 0))) return CS_EINVAL;
    if (l->matrices == 0) return CS_OK;
    const size_t need = workspace_bytes(l);
    if (ws_bytes < need) return CS_EWORKSPACE;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15)) return CS_EINVAL;
    const Span written[] = {{workspace, static_cast<int64_t>(need)}};
    const Span read[] = {{l->memory, static_cast<int64_t>(list_bytes(Plan{l->matrices, l->pieces, l->halves, l->fulls, 0, 0}))}, {lr, 8},
                         {grad_scale, 4}};
    if (!spans_apart(written, read)) return CS_EINVAL;
    char* const ws = static_cast<char*>(workspace);
    const hipStream_t s = stream_of(stream);
    if (l->tile == 128) return l->terms == 1 ? run_as<128, 1>(h, l, optimizer, lr, grad_scale, ws, s) : run_as<128, 2>(h, l, optimizer, lr, grad_scale, ws, s);
    return l->terms == 1 ? run_as<64, 1>(h, l, optimizer, lr, grad_scale, ws, s) : run_as<64, 2>(h, l, optimizer, lr, grad_scale, ws, s);
}

}  // namespace
}  // namespace cs

using namespace cs;

extern "C" int cs_matrix_list_bytes(const cs_matrix* stacks, int32_t count, int32_t terms, size_t* bytes) {
    Plan plan;
    if (count < 0 || (count && !stacks) || !bytes || (terms != 1 && terms != 2) || !plan_of(stacks, count, terms, plan)) return CS_EINVAL;
    *bytes = list_bytes(plan);
    return CS_OK;
}

extern "C" int cs_matrix_list_build(const cs_matrix* stacks, int32_t count, int32_t p_fmt, int32_t g_fmt, int32_t terms, void* memory,
                                    size_t bytes, cs_matrix_list* list, void* stream) {
    Plan plan;
    if (count < 0 || (count && !stacks) || !list || !fmt_ok(p_fmt) || !fmt_ok(g_fmt) || (terms != 1 && terms != 2) ||
        !plan_of(stacks, count, terms, plan))
        return CS_EINVAL;
    const size_t need = list_bytes(plan);
    if (bytes < need) return CS_EWORKSPACE;
    if (need && (!memory || (reinterpret_cast<uintptr_t>(memory) & 7))) return CS_EINVAL;
    const int64_t pb = fmt_bytes(p_fmt), gb = fmt_bytes(g_fmt);
    int moments = -1;
    for (int32_t i = 0; i < count; ++i) {
        const cs_matrix& s = stacks[i];
        if (s.count == 0 || s.rows == 0 || s.cols == 0) continue;
        const uintptr_t p = reinterpret_cast<uintptr_t>(s.p), g = reinterpret_cast<uintptr_t>(s.g), m = reinterpret_cast<uintptr_t>(s.m);
        if (!p || !g || p % pb || g % gb || m % 4 || (moments >= 0 && moments != (m != 0))) return CS_EINVAL;
        moments = m != 0;
        constexpr int64_t kFar = static_cast<int64_t>(1) << 38;
        if (s.p_stride < s.cols || s.g_stride < s.cols || s.p_stride > kFar / s.rows || s.g_stride > kFar / s.rows) return CS_EINVAL;
        const int64_t p_one = (s.rows - 1) * s.p_stride + s.cols, g_one = (s.rows - 1) * s.g_stride + s.cols;
        if (s.count > 1 && (s.p_step < p_one || s.g_step < g_one || s.p_step > kFar || s.g_step > kFar)) return CS_EINVAL;
        const int64_t p_bytes = ((s.count - 1) * s.p_step + p_one) * pb, g_bytes = ((s.count - 1) * s.g_step + g_one) * gb;
        const int64_t m_bytes = s.count * s.rows * s.cols * 4;
        // (without moments the result may take the place of what is read, value for value)
        const bool same = !m && p == g && p_fmt == g_fmt && s.p_stride == s.g_stride && (s.count == 1 || s.p_step == s.g_step);
        if ((!same && spans_meet(s.p, p_bytes, s.g, g_bytes)) || spans_meet(s.m, m_bytes, s.p, p_bytes) || spans_meet(s.m, m_bytes, s.g, g_bytes))
            return CS_EINVAL;
    }
    *list = cs_matrix_list{memory, plan.matrices, plan.pieces, plan.halves, plan.fulls, plan.work, p_fmt, g_fmt, terms, plan.tile, moments == 1};
    if (plan.matrices == 0) return CS_OK;
    Matrix* const matrices = static_cast<Matrix*>(memory);
    const hipStream_t st = stream_of(stream);
    Batch b = {};
    int filled = 0, rc = CS_OK;
    int64_t done = 0;
    const auto flush = [&] {
        if (!filled || rc) return;
        k_list_matrices<<<1, 64, 0, st>>>(b, matrices + done, filled);
        rc = launched();
        done += filled;
        filled = 0;
    };
    Plan again;
    plan_with(stacks, count, terms, plan.tile, again, [&](const cs_matrix& s, int64_t np, int64_t mp, const Plan& at, int64_t pieces, int64_t halves, int64_t fulls) {
        for (int64_t k = 0; k < s.count; ++k) {
            Matrix& t = b.t[filled];
            t.p = static_cast<char*>(s.p) + k * s.p_step * pb;
            t.g = static_cast<const char*>(s.g) + k * s.g_step * gb;
            t.moment = s.m ? s.m + k * s.rows * s.cols : nullptr;
            t.p_stride = s.p_stride, t.g_stride = s.g_stride;
            t.at = at.work + k * work_bytes(np, mp, terms);
            t.rows = static_cast<int32_t>(s.rows), t.cols = static_cast<int32_t>(s.cols);
            t.np = static_cast<int32_t>(np), t.mp = static_cast<int32_t>(mp);
            t.first_piece = static_cast<int32_t>(at.pieces + k * pieces), t.pieces = static_cast<int32_t>(pieces);
            t.first_half = static_cast<int32_t>(at.halves + k * halves), t.first_full = static_cast<int32_t>(at.fulls + k * fulls);
            if (++filled == kBatch) flush();
        }
    });
    flush();
    if (rc) return rc;
    Place* at = reinterpret_cast<Place*>(matrices + plan.matrices);
    const int64_t places[3] = {plan.pieces, plan.halves, plan.fulls};
    for (int which = 0; which < 3; ++which) {
        k_list_places<<<static_cast<unsigned>((places[which] + kThreads - 1) / kThreads), kThreads, 0, st>>>(
            matrices, static_cast<int>(plan.matrices), which, at, places[which]);
        if (int e = launched()) return e;
        at += places[which];
    }
    return CS_OK;
}

extern "C" int cs_muon_workspace_bytes(const cs_matrix_list* list, size_t* bytes) {
    if (!list_ok(list) || !bytes) return CS_EINVAL;
    *bytes = list->matrices ? workspace_bytes(list) : 0;
    return CS_OK;
}

extern "C" int cs_muon_step(const cs_muon* h, const cs_matrix_list* list, const double* lr_or_null, const float* grad_scale_or_null,
                            void* workspace, size_t ws_bytes, void* stream) {
    return run(h, list, true, lr_or_null, grad_scale_or_null, workspace, ws_bytes, stream);
}

extern "C" int cs_orthogonalize(const cs_muon* h, const cs_matrix_list* list, void* workspace, size_t ws_bytes, void* stream) {
    return run(h, list, false, nullptr, nullptr, workspace, ws_bytes, stream);
}

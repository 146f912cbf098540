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
constexpr int kDepth = 64;                   // values of a row in LDS, 128 bytes
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

// The tile of a workgroup: WI x WJ wavefronts, each with FI x FJ blocks of 16 x 16; `stages` parts of K are in LDS or on their way there.
template <int WI_, int WJ_, int FI_, int FJ_, int STAGES_>
struct Shape {
    static constexpr int WI = WI_, WJ = WJ_, FI = FI_, FJ = FJ_, STAGES = STAGES_;
    static constexpr int WAVES = WI * WJ, THREADS = WAVES * 64, TI = WI * FI * 16, TJ = WJ * FJ * 16;
    // Blocks that belong together: a lane has GI neighbouring rows of 4 GJ neighbouring columns of the output, so that both it and its
    // transpose are written in whole pieces of memory straight from the registers.
    static constexpr int GI = FI < 4 ? FI : 4, GJ = FJ < 4 ? FJ : 4;
    static constexpr int LOADS = (TI + TJ) / 8 / WAVES;                  // of 1 KB, a wavefront and stage
    static_assert(TI % (8 * WAVES) == 0 && TJ % (8 * WAVES) == 0, "whole loads");
};
// The row of the left tile that is place `at` of LDS: lane l of block f (of a group of GI) has row GI l + f.
template <typename S>
__device__ __forceinline__ int left_row(int at) {
    const int group = at / (16 * S::GI), in = at % (16 * S::GI);
    return group * 16 * S::GI + in % 16 * S::GI + in / 16;
}
// The right one: a lane of the result has rows 4 q .. 4 q + 3 of every block, which are columns 4 GJ q + 4 f + (0 .. 3) of a group.
template <typename S>
__device__ __forceinline__ int right_row(int at) {
    const int group = at / (16 * S::GJ), in = at % (16 * S::GJ), m = in % 16;
    return group * 16 * S::GJ + m / 4 * 4 * S::GJ + in / 16 * 4 + m % 4;
}

// Rows of 128 bytes into LDS, 64 values of K (one term) or 32 values of both terms.  A row's eight packs of 16 bytes lie in the order pack ^ (place /
// 2 % 8): 16 lanes that read the same pack of 16 rows meet all banks once.
template <typename S, int TERMS, bool LEFT>
__device__ __forceinline__ void stage(const _Float16* high, const _Float16* low, int64_t stride, _Float16* lds) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
    for (int q = 0; q < (LEFT ? S::TI : S::TJ) / (8 * S::WAVES); ++q) {
        const int first = (q * S::WAVES + wave) * 8, at = first + (lane >> 3), row = LEFT ? left_row<S>(at) : right_row<S>(at);
        const int pack = (lane & 7) ^ (at >> 1 & 7);
        const _Float16* from = (TERMS == 2 ? (pack < 4 ? high : low) + pack % 4 * 8 : high + pack * 8) + row * stride;
        __builtin_amdgcn_global_load_lds(reinterpret_cast<GlobalPointer>(reinterpret_cast<uintptr_t>(from)),
                                         (LdsPointer)(lds + first * kDepth), 16, 0, 0);
    }
}
// All but `left` of this wavefront's loads have arrived and its reads of LDS are done; then so are all wavefronts'.
template <int LEFT>
__device__ __forceinline__ void arrived() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory"); }

template <int N>
__device__ __forceinline__ void load_halves(const _Float16* p, Half8 (&v)[N]) {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = *reinterpret_cast<const Half8*>(p + 8 * e);
}
template <int N>
__device__ __forceinline__ void store_halves(_Float16* high, _Float16* low, const float (&v)[N]) {
    typedef _Float16 Halves __attribute__((ext_vector_type(N < 8 ? N : 8)));
#pragma unroll
    for (int e = 0; e < N; e += 8) {
        Halves hi, lo;
#pragma unroll
        for (int k = 0; k < (N < 8 ? N : 8); ++k) {
            _Float16 h, l;
            split(v[e + k] * kUp, h, l);
            hi[k] = h, lo[k] = l;
        }
        *reinterpret_cast<Halves*>(high + e) = hi;
        if (low) *reinterpret_cast<Halves*>(low + e) = lo;
    }
}

// N neighbouring parameters from column `col` of a row on: p = keep p - lr x (keep 0: x itself)
struct Update {
    float lr, keep;
    bool optimizer;
};
template <typename T, int N>
__device__ __forceinline__ void update_as(const Matrix& t, const Update& u, int64_t row, int64_t col, const float (&x)[N]) {
    if (row >= t.rows || col >= t.cols) return;
    T* const p = static_cast<T*>(t.p) + row * t.p_stride + col;
    if (col + N <= t.cols) {
        constexpr int P = N < kPack<T> ? N : kPack<T>;
#pragma unroll
        for (int e = 0; e < N; e += P) {
            float v[P];
            if (u.optimizer) load_pack<T, P>(p + e, v);
#pragma unroll
            for (int k = 0; k < P; ++k) v[k] = u.optimizer ? fmaf(v[k], u.keep, -u.lr * x[e + k]) : x[e + k];
            store_pack<false>(p + e, v);
        }
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (col + e < t.cols) p[e] = static_cast<T>(u.optimizer ? fmaf(static_cast<float>(p[e]), u.keep, -u.lr * x[e]) : x[e]);
    }
}
template <int N>
__device__ __forceinline__ void update(const Matrix& t, int p_fmt, const Update& u, int64_t row, int64_t col, const float (&x)[N]) {
    if (p_fmt == CS_FMT_F32) update_as<float>(t, u, row, col, x);
    else if (p_fmt == CS_FMT_BF16) update_as<bf16>(t, u, row, col, x);
    else update_as<f16>(t, u, row, col, x);
}

// Workgroups of a launch go round the 8 dies: each die gets neighbouring places, whose tiles read the same rows.
__device__ __forceinline__ int place_of_block() {
    const int per = gridDim.x / 8, more = gridDim.x % 8, die = blockIdx.x % 8, at = blockIdx.x / 8;
    return die * per + min(die, more) + at;
}
// Tiles in bands of 8 rows, column by column of a band; of a lower half those on and below the diagonal.
__device__ __forceinline__ void tile_of(int32_t local, int32_t down, int32_t across, int32_t& ti, int32_t& tj) {
    const int32_t band = local / (8 * across), in = local - band * 8 * across, high = min(8, down - 8 * band);
    ti = 8 * band + in % high;
    tj = in / high;
}
__device__ __forceinline__ void half_tile_of(int32_t local, int32_t down, int32_t& ti, int32_t& tj) {
    int32_t band = static_cast<int32_t>((sqrtf(8.f * local + 1.f) - 1.f) * 0.0625f);
    while (4 * band * (8 * band + 1) > local) --band;
    while (4 * (band + 1) * (8 * band + 9) <= local) ++band;
    int32_t in = local - 4 * band * (8 * band + 1);
    const int32_t high = min(8, down - 8 * band);
    if (in < 8 * band * high) {
        ti = 8 * band + in % high;
        tj = in / high;
        return;
    }
    in -= 8 * band * high;
    ti = 0;
    while (in > ti) in -= ++ti;
    ti += 8 * band;
    tj = 8 * band + in;
}

// C = L R^T of rows of K values, a tile a workgroup.
template <typename S, int TERMS, int MODE>
__global__ void __launch_bounds__(S::THREADS, 2) k_muon_product(List list, Product k, char* ws) {
    constexpr bool HALF = MODE == kGram || MODE == kSquare;
    constexpr int N = 4 * S::GJ, PART = (S::TI + S::TJ) * kDepth, ROWS = S::FI, GROUPS = S::FJ / S::GJ;
    constexpr int STEP = kDepth / TERMS;     // values of K a stage
    __shared__ __align__(1024) _Float16 lds[S::STAGES * PART];
    const Place at = (HALF ? list.halves : list.fulls)[place_of_block()];
    const Matrix t = list.matrices[at.matrix];
    const Work<TERMS> w(ws, t);
    int32_t ti, tj;
    if (HALF) half_tile_of(at.local, t.np / S::TI, ti, tj);
    else tile_of(at.local, t.np / S::TI, t.mp / S::TJ, ti, tj);
    const int32_t depth = MODE == kGram ? t.mp : t.np, all = depth / STEP;
    const int64_t stride = depth;
    const auto left = [&](int low) { return (MODE == kGram ? w.x(low) : MODE == kSquare ? w.a(low) : w.b(low)) + ti * S::TI * stride; };
    const auto right = [&](int low) { return (MODE == kGram ? w.x(low) : MODE == kSquare ? w.a(low) : w.xt(k.turn, low)) + tj * S::TJ * stride; };
    const _Float16* const l_at[2] = {left(0), left(TERMS - 1)};
    const _Float16* const r_at[2] = {right(0), right(TERMS - 1)};
    const auto load = [&](int32_t i, int turn) {
        _Float16* const to = lds + turn * PART;
        stage<S, TERMS, true>(l_at[0] + i * STEP, l_at[1] + i * STEP, stride, to);
        stage<S, TERMS, false>(r_at[0] + i * STEP, r_at[1] + i * STEP, stride, to + S::TI * kDepth);
    };
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wi = wave / S::WJ, wj = wave % S::WJ;
    Float4 acc[S::FI][S::FJ] = {};
    const auto multiply = [&](int turn) {
        const _Float16* const l = lds + turn * PART + (wi * S::FI * 16 + (lane & 15)) * kDepth;
        const _Float16* const r = lds + turn * PART + (S::TI + wj * S::FJ * 16 + (lane & 15)) * kDepth;
        Half8 lv[TERMS][S::FI], rv[TERMS][S::FJ];
        const auto read = [&](int q, Half8(&lq)[S::FI], Half8(&rq)[S::FJ]) {
            const int pack = (((lane >> 4) + 4 * q) ^ ((lane & 15) >> 1)) * 8;
#pragma unroll
            for (int f = 0; f < S::FI; ++f) lq[f] = *reinterpret_cast<const Half8*>(l + f * 16 * kDepth + pack);
#pragma unroll
            for (int f = 0; f < S::FJ; ++f) rq[f] = *reinterpret_cast<const Half8*>(r + f * 16 * kDepth + pack);
        };
        const auto add = [&](const Half8(&lq)[S::FI], const Half8(&rq)[S::FJ]) {
#pragma unroll
            for (int fi = 0; fi < S::FI; ++fi)
#pragma unroll
                for (int fj = 0; fj < S::FJ; ++fj) acc[fi][fj] = __builtin_amdgcn_mfma_f32_16x16x32_f16(rq[fj], lq[fi], acc[fi][fj], 0, 0, 0);
        };
        if constexpr (TERMS == 2) {
            read(0, lv[0], rv[0]);
            read(1, lv[1], rv[1]);
            add(lv[0], rv[0]);
            add(lv[0], rv[1]);
            add(lv[1], rv[0]);
        } else {
            read(0, lv[0], rv[0]);
            add(lv[0], rv[0]);
            read(1, lv[0], rv[0]);
            add(lv[0], rv[0]);
        }
    };
    int turn = 0, next = S::STAGES - 1;
#pragma unroll
    for (int i = 0; i < S::STAGES - 1; ++i)
        if (i < all) load(i, i);
    for (int32_t i = 0; i + 1 < all; ++i) {
        if (i + S::STAGES - 1 <= all) arrived<(S::STAGES - 2) * S::LOADS>();
        else arrived<0>();
        if (i + S::STAGES - 1 < all) load(i + S::STAGES - 1, next);
        next = next + 1 == S::STAGES ? 0 : next + 1;
        multiply(turn);
        turn = turn + 1 == S::STAGES ? 0 : turn + 1;
    }
    arrived<0>();
    // What the last part of the output needs of A0 or X is on its way while the last products are taken.
    const int32_t row0 = ti * S::TI + wi * S::FI * 16 + (lane & 15) * S::GI, col0 = tj * S::TJ + wj * S::FJ * 16 + (lane >> 4) * N;
    const int64_t wide = HALF ? t.np : t.mp;             // of an output row
    const auto row_of = [&](int fi) { return row0 + fi / S::GI * 16 * S::GI + fi % S::GI; };
    constexpr bool READS = MODE != kGram, LOW = READS && (TERMS == 2 || !HALF);
    Half8 hi[READS ? ROWS : 1][GROUPS][N / 8 ? N / 8 : 1], lo[LOW ? ROWS : 1][GROUPS][N / 8 ? N / 8 : 1];
    if constexpr (READS) {
#pragma unroll
        for (int fi = 0; fi < ROWS; ++fi)
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                const int64_t from = row_of(fi) * wide + col0 + g * 4 * N;
                load_halves((HALF ? w.a(0) : w.x(0)) + from, hi[fi][g]);
                if constexpr (LOW) load_halves((HALF ? w.a(1) : w.x(1)) + from, lo[fi][g]);
            }
    }
    multiply(turn);

    Update u = {k.lr, k.decay, k.optimizer != 0};
    if constexpr (MODE == kFinish) {
        if (skipped(k.grad_scale)) return;
        if (k.lr_now) {
            u.lr = static_cast<float>(*k.lr_now);
            u.keep = static_cast<float>(1. - *k.lr_now * k.lr_decay);
        }
        const float ratio = static_cast<float>(t.rows) / static_cast<float>(t.cols);
        u.lr *= k.scale_rule == CS_MUON_SCALE_SHAPE ? sqrtf(fmaxf(1.f, ratio))
                : k.scale_rule == CS_MUON_SCALE_RMS ? 0.2f * sqrtf(static_cast<float>(max(t.rows, t.cols))) : 1.f;
    }
    const bool tall = t.rows > t.cols;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        const int32_t col = col0 + g * 4 * N;
        float dj[N];
        if constexpr (MODE == kSquare) {
#pragma unroll
            for (int e = 0; e < N; e += 4) {
                const Float4 d = *reinterpret_cast<const Float4*>(w.da() + col + e);
#pragma unroll
                for (int x = 0; x < 4; ++x) dj[e + x] = d[x];
            }
        }
#pragma unroll
        for (int gi = 0; gi < S::FI; gi += S::GI) {
            float out[S::GI][N];
#pragma unroll
            for (int f = 0; f < S::GI; ++f) {
                const int fi = gi + f;
                const int32_t row = row_of(fi);
                const float d = MODE == kSquare ? w.da()[row] : MODE == kGram ? 0.f : k.a + w.db()[row];
                float diagonal = 0.f;
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const float c = acc[fi][g * S::GJ + e / 4][e % 4] * (kDown * kDown);
                    float x = 0.f;
                    if constexpr (READS) {
                        x = static_cast<float>(hi[fi][g][e / 8][e % 8]);
                        if constexpr (LOW) x += static_cast<float>(lo[fi][g][e / 8][e % 8]);
                        x *= kDown;
                    }
                    out[f][e] = MODE == kGram ? c : MODE == kSquare ? fmaf(k.b, x, k.c * fmaf(d + dj[e], x, c)) : fmaf(d, x, c);
                    if (HALF && row == col + e) {
                        diagonal = MODE == kGram ? c : fmaf(k.b, d, k.c * fmaf(d, d, c));
                        out[f][e] = 0.f;
                    }
                }
                if (HALF && row >= col && row < col + N) (MODE == kGram ? w.da() : w.db())[row] = diagonal;
                if constexpr (MODE == kFinish) {
                    if (!tall) update(t, k.p_fmt, u, row, col, out[f]);
                } else {
                    const int64_t to = row * wide + col;
                    const auto place = [&](int low) { return (MODE == kGram ? w.a(low) : MODE == kSquare ? w.b(low) : w.x(low)) + to; };
                    store_halves(place(0), TERMS == 2 || MODE == kApply ? place(1) : nullptr, out[f]);
                }
            }
            // the transpose: of A and B the tile on the other side, of X the one that the next product reads
            if (HALF ? ti == tj : MODE == kFinish && !tall) continue;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                float turned[S::GI];
#pragma unroll
                for (int f = 0; f < S::GI; ++f) turned[f] = out[f][e];
                if constexpr (MODE == kFinish) {
                    update(t, k.p_fmt, u, col + e, row_of(gi), turned);
                } else {
                    const int64_t to = static_cast<int64_t>(col + e) * t.np + row_of(gi);
                    const auto place = [&](int low) { return (MODE == kGram ? w.a(low) : MODE == kSquare ? w.b(low) : w.xt(1 - k.turn, low)) + to; };
                    store_halves(place(0), TERMS == 2 ? place(1) : nullptr, turned);
                }
            }
        }
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

using Large = Shape<2, 2, 4, 4, 2>;
using Small = Shape<2, 2, 2, 2, 4>;

template <typename S, int TERMS>
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
        k_muon_product<S, TERMS, kGram><<<halves, S::THREADS, 0, s>>>(at, k, ws);
        k_muon_product<S, TERMS, kSquare><<<halves, S::THREADS, 0, s>>>(at, k, ws);
        if (i + 1 < h->steps) {
            k_muon_product<S, TERMS, kApply><<<fulls, S::THREADS, 0, s>>>(at, k, ws);
        } else {
            k.p_fmt = l->p_fmt, k.optimizer = optimizer, k.scale_rule = h->scale;
            k.lr = static_cast<float>(h->lr), k.decay = static_cast<float>(1. - h->lr * h->weight_decay);
            k.lr_decay = static_cast<float>(h->weight_decay);
            k.lr_now = lr, k.grad_scale = grad_scale;
            k_muon_product<S, TERMS, kFinish><<<fulls, S::THREADS, 0, s>>>(at, k, ws);
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
    if (l->tile == 128) return l->terms == 1 ? run_as<Large, 1>(h, l, optimizer, lr, grad_scale, ws, s) : run_as<Large, 2>(h, l, optimizer, lr, grad_scale, ws, s);
    return l->terms == 1 ? run_as<Small, 1>(h, l, optimizer, lr, grad_scale, ws, s) : run_as<Small, 2>(h, l, optimizer, lr, grad_scale, ws, s);
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

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
// 4e-3; in bfloat16: 1e-2 to 3e-2): less than half a step of bfloat16 (3.9e-3; its rounding is 1.7e-3 in the mean square).  Of rank one it is
// 1.7e-3, with a quarter of the directions a hundred times the rest or more 2.5e-3, the most that was found.  terms = 2 splits A0, B0 and X in
// all products (hi hi + hi lo + lo hi) and is as exact as products in binary32 (64 x 4097 9e-7, these 1.4e-6; 512 x 512 3.3e-6, 2.4e-6 to 5e-6).
// Everything is stored 2^10 times: entries of X, A and B are below 64.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "cs_rows.h"
#include "csketch.h"

namespace cs {
namespace {

constexpr int kThreads = 256;
constexpr int kEdge = 64;                    // of the pieces in which u is read, and what all sizes are rounded up to
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
    int32_t first_piece, first_half, first_full, pieces;      // (of a thin one first_piece is its first slab)
};
struct Place {
    int32_t matrix, local;
};
// A tile of an output, with all that its workgroup has to know before its first load
struct Tile {
    int64_t at;
    int32_t np, mp, ti, tj, matrix, unused;
};
constexpr int kBatch = 40;
struct Batch {
    Matrix t[kBatch];
};
static_assert(sizeof(Batch) < 3800, "kernel arguments are limited to 4 KB");

// A list in device memory: Matrix[count], then the tiles of lower halves of A (whole ones, then quarters of those that are left), all tiles of
// X, and the places of all pieces and slabs.
struct List {
    const Matrix* matrices;
    const Tile *halves, *fulls;
    const Place *pieces, *slabs;
};

// A matrix's part of the workspace: X twice (read and written in turns), A0, B0, and the diagonals of A and B.  Values are two halves, the upper and the
// lower 11 bits.  Where the products take both (two terms) they lie in one array, 32 upper ones and then the 32 lower ones of the same columns;
// otherwise the lower ones of X have one array of their own and there are no others.
template <int TERMS>
struct Work {
    _Float16* base;
    int64_t nm, nn;
    int32_t np;
    __device__ __forceinline__ Work(char* ws, int64_t at, int32_t n, int32_t m)
        : base(reinterpret_cast<_Float16*>(ws + at)), nm(static_cast<int64_t>(n) * m), nn(static_cast<int64_t>(n) * n), np(n) {}
    __device__ __forceinline__ _Float16* x(int turn) const { return base + turn * TERMS * nm; }
    __device__ __forceinline__ _Float16* x_low(int turn) const { return TERMS == 1 ? base + 2 * nm : x(turn) + 32; }
    __device__ __forceinline__ _Float16* a() const { return base + (2 + TERMS) * nm; }
    __device__ __forceinline__ _Float16* b() const { return a() + TERMS * nn; }
    __device__ __forceinline__ float* da() const { return reinterpret_cast<float*>(b() + TERMS * nn); }
    __device__ __forceinline__ float* db() const { return da() + np; }
    // of an array's value
    static __device__ __forceinline__ int64_t place(int64_t row, int32_t col, int32_t width) {
        return TERMS == 1 ? row * width + col : row * 2 * width + col / 32 * 64 + col % 32;
    }
};
int64_t work_bytes(int64_t np, int64_t mp, int terms) { return 2 * ((2 + terms) * np * mp + 2 * terms * np * np) + 2 * 4 * np; }

__global__ void __launch_bounds__(64) k_list_matrices(Batch b, Matrix* out, int count) {
    if (static_cast<int>(threadIdx.x) < count) out[threadIdx.x] = b.t[threadIdx.x];
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

enum { kPieces, kHalves, kTails, kFulls };
// The matrix of every place (the last that begins at or before it), and what there is to know of it; high, wide: of a tile.
// kTails: quarters of tiles, from tile number `from` on.
template <int WHICH, typename Out>
__global__ void __launch_bounds__(kThreads)
k_list_places(const Matrix* matrices, int begin, int end, int high, int wide, Out* out, int64_t places, int64_t from) {
    const int64_t place = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    if (place >= places) return;
    const int64_t c = from + (WHICH == kTails ? place / 4 : place);
    const auto first = [&](int i) {
        const Matrix& t = matrices[i];
        return WHICH == kPieces ? t.first_piece : WHICH == kFulls ? t.first_full : t.first_half;
    };
    int lo = begin, hi = end - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (first(mid) <= c) lo = mid;
        else hi = mid - 1;
    }
    const int32_t local = static_cast<int32_t>(c - first(lo));
    if constexpr (WHICH == kPieces) {
        out[place] = Place{lo, local};
    } else {
        const Matrix& t = matrices[lo];
        Tile tile = {t.at, t.np, t.mp, 0, 0, lo, 0};
        if (WHICH == kFulls) tile_of(local, t.np / high, t.mp / wide, tile.ti, tile.tj);
        else half_tile_of(local, t.np / high, tile.ti, tile.tj);
        if (WHICH == kTails) {
            tile.ti = 2 * tile.ti + static_cast<int32_t>(place >> 1 & 1);
            tile.tj = 2 * tile.tj + static_cast<int32_t>(place & 1);
        }
        out[place] = tile;
    }
}

__device__ __forceinline__ bool skipped(const float* grad_scale) { return grad_scale && !(fabsf(*grad_scale) < INFINITY); }

// N neighbouring values of a row from column `col` on, 0 from column `cols` on
template <typename T, int N>
__device__ __forceinline__ void read_as(const T* row, int32_t col, int32_t cols, float (&v)[N]) {
    if (N > 1 && col + N <= cols) {
        constexpr int P = N < 2 ? 2 : N < kPack<T> ? N : kPack<T>;
#pragma unroll
        for (int e = 0; e < N; e += P) {
            float part[P];
            load_pack<T, P>(row + col + e, part);
#pragma unroll
            for (int k = 0; k < P; ++k)
                if (e + k < N) v[e + k] = part[k];
        }
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = col + e < cols ? static_cast<float>(row[col + e]) : 0.f;
    }
}
template <int N>
__device__ __forceinline__ void read_row(const void* p, int fmt, int64_t row_at, int32_t col, int32_t cols, float (&v)[N]) {
    if (fmt == CS_FMT_F32) read_as<float, N>(static_cast<const float*>(p) + row_at, col, cols, v);
    else if (fmt == CS_FMT_BF16) read_as<bf16, N>(static_cast<const bf16*>(p) + row_at, col, cols, v);
    else read_as<f16, N>(static_cast<const f16*>(p) + row_at, col, cols, v);
}

struct Moment {
    float mu;
    int nesterov, g_fmt;
    const float* grad_scale;
};
// u of N neighbouring elements, 0 outside the matrix.  STEP: the moment takes the gradient first, and is written.
template <bool STEP, int N>
__device__ __forceinline__ void direction(const Matrix& t, const Moment& k, float s, int32_t row, int32_t col, float (&u)[N]) {
    if (row >= t.rows || col >= t.cols) {
#pragma unroll
        for (int e = 0; e < N; ++e) u[e] = 0.f;
        return;
    }
    float m[N];
    if (!t.moment || STEP || k.nesterov) read_row<N>(t.g, k.g_fmt, row * t.g_stride, col, t.cols, u);
    if (!t.moment) return;
    float* const at = t.moment + static_cast<int64_t>(row) * t.cols;
    read_as<float, N>(at, col, t.cols, m);
#pragma unroll
    for (int e = 0; e < N; ++e) {
        if (STEP) m[e] = fmaf(k.mu, m[e], s * u[e]);
        u[e] = k.nesterov ? fmaf(k.mu, m[e], s * u[e]) : m[e];
    }
    if (!STEP) return;
    if (N > 1 && col + N <= t.cols) {
        store_pack<false>(at + col, m);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (col + e < t.cols) at[col + e] = m[e];
    }
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

// The sum over a workgroup of kThreads, in a fixed order, in every thread
__device__ __forceinline__ double workgroup_sum(double sum, double (&buf)[kThreads / 64]) {
#pragma unroll
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = sum;
    __syncthreads();
    sum = 0.;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) sum += buf[w];
    return sum;
}
// 1 / (|u| + eps) from the sum of squares, or 0 for a matrix of zeros
__device__ __forceinline__ double inverse_of(double sum, double eps) { return sum == 0. ? 0. : 1. / (sqrt(sum) + eps); }

constexpr int kFour = 4;                     // neighbouring elements a thread

// The moment, and a piece's sum of squares of u (binary64, a fixed order).
__global__ void __launch_bounds__(kThreads) k_muon_moment(List list, Moment k, double* squares) {
    __shared__ double buf[kThreads / 64];
    const Place at = list.pieces[blockIdx.x];
    const Matrix t = list.matrices[at.matrix];
    const Piece piece(t, at.local);
    double sum = 0.;
    if (!skipped(k.grad_scale)) {
        const float s = k.grad_scale ? *k.grad_scale : 1.f;
#pragma unroll
        for (int i = 0; i < kEdge * kEdge / kFour; i += kThreads) {
            const int q = i + threadIdx.x;
            float u[kFour];
            direction<true>(t, k, s, piece.row + q / (kEdge / kFour), piece.col + q % (kEdge / kFour) * kFour, u);
#pragma unroll
            for (int e = 0; e < kFour; ++e) sum = fma(static_cast<double>(u[e]), static_cast<double>(u[e]), sum);
        }
    }
    sum = workgroup_sum(sum, buf);
    if (threadIdx.x == 0) squares[blockIdx.x] = sum;
}

// A matrix's sum of squares, in place of its first piece's
__global__ void __launch_bounds__(kThreads) k_muon_norm(List list, double* squares) {
    __shared__ double buf[kThreads / 64];
    const Matrix& t = list.matrices[blockIdx.x];
    double sum = 0.;
    for (int i = threadIdx.x; i < t.pieces; i += kThreads) sum += squares[t.first_piece + i];
    sum = workgroup_sum(sum, buf);
    if (threadIdx.x == 0 && t.pieces) squares[t.first_piece] = sum;
}

// A binary32 number that the compiler has to have as such.  Without it a product and sum that is rounded to binary16 in two places may be rounded
// by way of binary32 in one and directly in the other: next to a tie the two are a step of binary16 apart, and what is left of one upper half
// was stored beside the other (one value in ten thousand, by 2^-11 of it: some matrices with two terms 14 times as far off as the others).
__device__ __forceinline__ float held(float v) {
    asm("" : "+v"(v));
    return v;
}
__device__ __forceinline__ void split(float v, _Float16& hi, _Float16& lo) {
    v = held(v);
    hi = static_cast<_Float16>(v);
    lo = static_cast<_Float16>(v - static_cast<float>(hi));
}

// X from u, zero behind the last row and column.  joined: a matrix's squares are summed already.
template <int TERMS>
__global__ void __launch_bounds__(kThreads) k_muon_begin(List list, Moment k, double eps, const double* squares, bool joined, char* ws) {
    __shared__ float tile[kEdge][kEdge + 1];
    __shared__ double buf[kThreads / 64];
    const Place at = list.pieces[blockIdx.x];
    const Matrix t = list.matrices[at.matrix];
    const Piece piece(t, at.local);
    const Work<TERMS> w(ws, t.at, t.np, t.mp);
    const float s = k.grad_scale ? *k.grad_scale : 1.f;
    float u[kEdge * kEdge / kFour / kThreads][kFour];
#pragma unroll
    for (int i = 0; i < kEdge * kEdge / kFour; i += kThreads) {
        const int q = i + threadIdx.x;
        direction<false>(t, k, s, piece.row + q / (kEdge / kFour), piece.col + q % (kEdge / kFour) * kFour, u[i / kThreads]);
    }
    double sum = 0.;
    if (joined) {
        sum = squares[t.first_piece];
    } else {
        for (int i = threadIdx.x; i < t.pieces; i += kThreads) sum += squares[t.first_piece + i];
        sum = workgroup_sum(sum, buf);
    }
    const double one = inverse_of(sum, eps) * static_cast<double>(kUp);
#pragma unroll
    for (int i = 0; i < kEdge * kEdge / kFour; i += kThreads) {
        const int q = i + threadIdx.x;
#pragma unroll
        for (int e = 0; e < kFour; ++e)
            tile[q / (kEdge / kFour)][q % (kEdge / kFour) * kFour + e] = static_cast<float>(u[i / kThreads][e] * one);
    }
    __syncthreads();
    // (of a tall matrix the transpose)
    const bool tall = t.rows > t.cols;
    for (int i = threadIdx.x; i < kEdge * kEdge / 8; i += kThreads) {
        const int r = i / 8, c = i % 8 * 8;
        Half8 hi, lo;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            _Float16 h, l;
            split(tall ? tile[c + e][r] : tile[r][c + e], h, l);
            hi[e] = h, lo[e] = l;
        }
        const int64_t to = Work<TERMS>::place((tall ? piece.col : piece.row) + r, (tall ? piece.row : piece.col) + c, t.mp);
        *reinterpret_cast<Half8*>(w.x(0) + to) = hi;
        *reinterpret_cast<Half8*>(w.x_low(0) + to) = lo;
    }
}

enum { kWhole, kPartial, kJoin };
enum { kGram, kSquare, kApply, kFinish };    // A = X X^T; B = b A + c A A; X = a X + B X; the same, into the parameters

// What is made of the last X: p = decay p - lr scale X, or X itself
struct Last {
    int p_fmt, optimizer, scale_rule;
    float decay, lr, lr_decay;
    const double* lr_now;
    const float* grad_scale;
};
struct Steps {
    int count;
    float coefs[CS_MUON_MAX_STEPS][3];
};
struct Product {
    float a, b, c;
    int turn;                                // which of the two X is read
    Last last;                               // kFinish
    int slices;                              // of K, and where their products are left
    Float4* partials;
};

typedef __attribute__((address_space(3))) void* LdsPointer;
typedef const __attribute__((address_space(1))) void* GlobalPointer;

// The tile of a workgroup: WI x WJ wavefronts, each with FI x FJ blocks of 16 x 16; STAGES parts of 64 values of K are in LDS or on their
// way there; AHEAD: operands are read from there a step ahead.  WAVES_PER_SIMD: as many as the registers are shared out for.
template <int WI_, int WJ_, int FI_, int FJ_, int STAGES_, int WAVES_PER_SIMD_, bool AHEAD_>
struct Shape {
    static constexpr int WI = WI_, WJ = WJ_, FI = FI_, FJ = FJ_, STAGES = STAGES_, DEPTH = 64, WAVES_PER_SIMD = WAVES_PER_SIMD_;
    static constexpr bool AHEAD = AHEAD_;
    static constexpr int WAVES = WI * WJ, THREADS = WAVES * 64, TI = WI * FI * 16, TJ = WJ * FJ * 16;
    // Blocks that belong together: a lane has GI neighbouring rows of 4 GJ neighbouring columns of the output, so that both it and its
    // transpose are written in whole pieces of memory straight from the registers.
    static constexpr int GI = FI < 4 ? FI : 4, GJ = FJ;
    static constexpr int PACKS = DEPTH / 8, ROWS = 64 / PACKS;           // of 16 bytes, a row; rows that a wavefront loads at once
    static constexpr int LOADS = (TI + TJ) / ROWS / WAVES;               // of 1 KB, a wavefront and stage
    static_assert(TI % (ROWS * WAVES) == 0 && TJ % (ROWS * WAVES) == 0 && FI % GI == 0 && FJ <= 4, "");
    // the order of a row's packs in LDS: 16 lanes that read the same pack of 16 rows meet all banks once
    static __device__ __forceinline__ int order(int place) { return place >> 1 & 7; }
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

// Rows of DEPTH halves into LDS, their packs of 16 bytes in the order pack ^ order(place).  The lane's offsets in memory are the same for all parts
// of K.
template <typename S, bool LEFT>
struct Stage {
    static constexpr int N = (LEFT ? S::TI : S::TJ) / (S::ROWS * S::WAVES);
    uint32_t offset[N];
    __device__ __forceinline__ explicit Stage(uint32_t row_bytes) {
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
        for (int q = 0; q < N; ++q) {
            const int at = (q * S::WAVES + wave) * S::ROWS + lane / S::PACKS, row = LEFT ? left_row<S>(at) : right_row<S>(at);
            offset[q] = row * row_bytes + ((lane % S::PACKS) ^ S::order(at)) * 16;
        }
    }
    __device__ __forceinline__ void load(const char* from, _Float16* lds) const {
        const int wave = threadIdx.x >> 6;
#pragma unroll
        for (int q = 0; q < N; ++q)
            __builtin_amdgcn_global_load_lds(reinterpret_cast<GlobalPointer>(reinterpret_cast<uintptr_t>(from + offset[q])),
                                             (LdsPointer)(lds + (q * S::WAVES + wave) * 512), 16, 0, 0);
    }
};
// The right operand of B X: columns of X, which lies in rows.  A part of K is 64 (of two terms 32) rows of the tile's columns; LDS gives them
// transposed (four lanes hold 16 columns of a row, and a lane gets a column of four rows).  A row's packs lie in the order pack ^ order(row): a
// quarter of a wavefront reads four rows, which meet different banks.
template <typename S, int TERMS>
struct Columns {
    static constexpr int N = S::TJ / (8 * S::WAVES), PACKS = S::TJ * TERMS / 8, WIDTH = PACKS * 8;
    static constexpr int ODD = TERMS == 2 ? (S::GJ == 4 ? 1 : 4) : S::GJ == 4 ? 1 : PACKS == 8 ? 0 : 4;
    static constexpr int HIGH = TERMS == 2 ? (S::GJ == 4 ? 4 : 8) : PACKS == 8 ? 4 : 8;
    static __device__ __forceinline__ int order(int row) { return (row & 1) * ODD ^ (row >> 1 & 1) * HIGH; }
    uint32_t offset[N];
    __device__ __forceinline__ explicit Columns(uint32_t row_bytes) {
        const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
#pragma unroll
        for (int q = 0; q < N; ++q) {
            const int at = (q * S::WAVES + wave) * 64 + lane, row = at / PACKS;
            offset[q] = row * row_bytes + (at % PACKS ^ order(row)) * 16;
        }
    }
    __device__ __forceinline__ void load(const char* from, _Float16* lds) const {
        const int wave = threadIdx.x >> 6;
#pragma unroll
        for (int q = 0; q < N; ++q)
            __builtin_amdgcn_global_load_lds(reinterpret_cast<GlobalPointer>(reinterpret_cast<uintptr_t>(from + offset[q])),
                                             (LdsPointer)(lds + (q * S::WAVES + wave) * 512), 16, 0, 0);
    }
    // 8 values of K of a column a lane: block f of wavefront wj; q: the second 32 rows, or the lower halves
    static __device__ __forceinline__ Half8 take(const _Float16* lds, int wj, int f, int q) {
        typedef short Short4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) Short4* Pointer;
        const int lane = threadIdx.x & 63, col = wj * S::FJ * 16 + (lane & 3) * 4 * S::GJ + f * 4;
        const int in = TERMS == 1 ? col : col / 32 * 64 + col % 32 + q * 32;
        union {
            Short4 part[2];
            Half8 all;
        } v;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int row = (TERMS == 1 ? q * 32 : 0) + (lane >> 4) * 8 + h * 4 + (lane >> 2 & 3);
            v.part[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Pointer)(lds + row * WIDTH + ((in / 8 ^ order(row)) * 8 + in % 8)));
        }
        return v.all;
    }
};
// All but `left` of this wavefront's loads have arrived and its reads of LDS are done; then so are all wavefronts'.
template <int LEFT>
__device__ __forceinline__ void arrived() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory"); }

// p = keep p - lr x, or x itself
struct Update {
    float lr, keep;
    bool optimizer;
};
__device__ __forceinline__ Update update_of(const Last& k, const Matrix& t) {
    Update u = {k.lr, k.decay, k.optimizer != 0};
    if (k.lr_now) {
        u.lr = static_cast<float>(*k.lr_now);
        u.keep = static_cast<float>(1. - *k.lr_now * k.lr_decay);
    }
    const float ratio = static_cast<float>(t.rows) / static_cast<float>(t.cols);
    u.lr *= k.scale_rule == CS_MUON_SCALE_SHAPE ? sqrtf(fmaxf(1.f, ratio))
            : k.scale_rule == CS_MUON_SCALE_RMS ? 0.2f * sqrtf(static_cast<float>(max(t.rows, t.cols))) : 1.f;
    return u;
}
// N neighbouring parameters from column `col` of a row on: as they are (or 0), and written
template <int N>
__device__ __forceinline__ void read_p(const Matrix& t, int p_fmt, int32_t row, int32_t col, float (&v)[N]) {
    if (row < t.rows && col < t.cols) {
        read_row<N>(t.p, p_fmt, row * t.p_stride, col, t.cols, v);
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = 0.f;
    }
}
template <typename T, int N>
__device__ __forceinline__ void write_as(const Matrix& t, int32_t row, int32_t col, const float (&v)[N]) {
    T* const p = static_cast<T*>(t.p) + row * t.p_stride + col;
    if (N > 1 && col + N <= t.cols) {
        constexpr int P = N < 2 ? 2 : N < kPack<T> ? N : kPack<T>;
#pragma unroll
        for (int e = 0; e < N; e += P) {
            float part[P];
#pragma unroll
            for (int k = 0; k < P; ++k) part[k] = v[e + k < N ? e + k : 0];
            store_pack<false>(p + e, part);
        }
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (col + e < t.cols) p[e] = static_cast<T>(v[e]);
    }
}
template <int N>
__device__ __forceinline__ void write_p(const Matrix& t, int p_fmt, int32_t row, int32_t col, const float (&v)[N]) {
    if (row >= t.rows || col >= t.cols) return;
    if (p_fmt == CS_FMT_F32) write_as<float>(t, row, col, v);
    else if (p_fmt == CS_FMT_BF16) write_as<bf16>(t, row, col, v);
    else write_as<f16>(t, row, col, v);
}
// A lane's H rows of W columns of X into the parameters (of a tall matrix into its transpose), which are all asked for first.
template <int H, int W>
__device__ __forceinline__ void finish(const Matrix& t, int p_fmt, const Update& u, int32_t row, int32_t col, const float (&x)[H][W]) {
    float old[H][W];
    if (t.rows > t.cols) {
        if (u.optimizer)
#pragma unroll
            for (int e = 0; e < W; ++e) {
                float v[H];
                read_p(t, p_fmt, col + e, row, v);
#pragma unroll
                for (int f = 0; f < H; ++f) old[f][e] = v[f];
            }
#pragma unroll
        for (int e = 0; e < W; ++e) {
            float v[H];
#pragma unroll
            for (int f = 0; f < H; ++f) v[f] = u.optimizer ? fmaf(old[f][e], u.keep, -u.lr * x[f][e]) : x[f][e];
            write_p(t, p_fmt, col + e, row, v);
        }
    } else {
        if (u.optimizer)
#pragma unroll
            for (int f = 0; f < H; ++f) read_p(t, p_fmt, row + f, col, old[f]);
#pragma unroll
        for (int f = 0; f < H; ++f) {
            float v[W];
#pragma unroll
            for (int e = 0; e < W; ++e) v[e] = u.optimizer ? fmaf(old[f][e], u.keep, -u.lr * x[f][e]) : x[f][e];
            write_p(t, p_fmt, row + f, col, v);
        }
    }
}

// Workgroups of a launch go round the 8 dies: each die gets neighbouring places, whose tiles read the same rows.
__device__ __forceinline__ int place_of_block() {
    const int per = gridDim.x / 8, more = gridDim.x % 8, die = blockIdx.x % 8, at = blockIdx.x / 8;
    return die * per + min(die, more) + at;
}
// C = L R^T of rows of K values, a tile a workgroup.  Few tiles with many values of K are taken in slices of K by workgroups of their own (kPartial),
// whose products a second launch adds up (kJoin).
template <typename S, int TERMS, int MODE, int PHASE>
__global__ void __launch_bounds__(S::THREADS, S::WAVES_PER_SIMD) k_muon_product(List list, Product k, char* ws) {
    constexpr bool HALF = MODE == kGram || MODE == kSquare;
    constexpr int N = 4 * S::GJ, PART = (S::TI + S::TJ) * S::DEPTH;
    __shared__ __align__(1024) _Float16 lds[PHASE == kJoin ? 8 : S::STAGES * PART];
    const int32_t place = PHASE == kPartial ? blockIdx.x / k.slices : PHASE == kJoin ? blockIdx.x : place_of_block();
    const Tile t = (HALF ? list.halves : list.fulls)[place];
    if (HALF && t.ti < t.tj) return;                         // (a quarter above the diagonal: the one below it is written twice)
    const Work<TERMS> w(ws, t.at, t.np, t.mp);
    const int32_t depth = (MODE == kGram ? t.mp : t.np) * TERMS, parts = depth / S::DEPTH;
    // (of a slice of K the parts from `from` on)
    const int32_t slice = PHASE == kPartial ? blockIdx.x % k.slices : 0;
    const int32_t from = PHASE == kPartial ? static_cast<int32_t>(static_cast<int64_t>(parts) * slice / k.slices) : 0;
    const int32_t all = (PHASE == kPartial ? static_cast<int32_t>(static_cast<int64_t>(parts) * (slice + 1) / k.slices) : parts) - from;
    const Stage<S, true> l_stage(depth * 2);
    const char* const left = reinterpret_cast<const char*>((MODE == kGram ? w.x(k.turn) : MODE == kSquare ? w.a() : w.b()) +
                                                           static_cast<int64_t>(t.ti) * S::TI * depth + from * S::DEPTH);
    using Right = typename std::conditional<HALF, Stage<S, false>, Columns<S, TERMS>>::type;
    const Right r_stage(HALF ? depth * 2 : t.mp * TERMS * 2);
    const char* const right = reinterpret_cast<const char*>(
        HALF ? (MODE == kGram ? w.x(k.turn) : w.a()) + static_cast<int64_t>(t.tj) * S::TJ * depth + from * S::DEPTH : w.x(k.turn) + t.tj * S::TJ * TERMS);
    const int64_t r_step = HALF ? S::DEPTH * 2 : static_cast<int64_t>(t.mp) * (S::DEPTH * 2);
    const auto load = [&](int32_t i, int turn) {
        l_stage.load(left + i * (S::DEPTH * 2), lds + turn * PART);
        r_stage.load(right + i * r_step, lds + turn * PART + S::TI * S::DEPTH);
    };
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, wi = wave / S::WJ, wj = wave % S::WJ;
    Float4 acc[S::FI][S::FJ] = {};
    // what 32 values of K take: of a part in LDS the first and the second 32 of one term, or both terms' 32
    struct Operands {
        Half8 l[S::FI], r[S::FJ];
    };
    const int l_from = (wi * S::FI * 16 + (lane & 15)) * S::DEPTH, r_from = (S::TI + wj * S::FJ * 16 + (lane & 15)) * S::DEPTH;
    const auto take = [&](Operands& v, int turn, int q) {
        const _Float16* const part = lds + turn * PART + ((((lane >> 4) + 4 * q) ^ S::order(lane & 15)) * 8);
#pragma unroll
        for (int f = 0; f < S::FI; ++f) v.l[f] = *reinterpret_cast<const Half8*>(part + l_from + f * 16 * S::DEPTH);
#pragma unroll
        for (int f = 0; f < S::FJ; ++f) {
            if constexpr (HALF) v.r[f] = *reinterpret_cast<const Half8*>(part + r_from + f * 16 * S::DEPTH);
            else v.r[f] = Right::take(lds + turn * PART + S::TI * S::DEPTH, wj, f, q);
        }
    };
    const auto add = [&](const Half8(&l)[S::FI], const Half8(&r)[S::FJ]) {
#pragma unroll
        for (int fi = 0; fi < S::FI; ++fi)
#pragma unroll
            for (int fj = 0; fj < S::FJ; ++fj) acc[fi][fj] = __builtin_amdgcn_mfma_f32_16x16x32_f16(r[fj], l[fi], acc[fi][fj], 0, 0, 0);
    };
    const auto add_second = [&](const Operands& first, const Operands& second) {
        if (TERMS == 2) {
            add(first.l, second.r);
            add(second.l, first.r);
        } else {
            add(second.l, second.r);
        }
    };
    // of a tile's slices, a lane's blocks each: the slices' products, which the join adds up in their order
    Float4* const sums = k.partials + (static_cast<int64_t>(place) * k.slices + slice) * (S::FI * S::FJ * S::THREADS) + threadIdx.x;
#pragma unroll
    for (int i = 0; i < S::STAGES - 1; ++i)
        if (PHASE != kJoin && i < all) load(i, i);
    Operands first, second;
    if constexpr (PHASE == kJoin) {
#pragma unroll 8
        for (int i = 0; i < k.slices; ++i)
#pragma unroll
            for (int fi = 0; fi < S::FI; ++fi)
#pragma unroll
                for (int fj = 0; fj < S::FJ; ++fj) acc[fi][fj] += sums[(i * S::FI * S::FJ + fi * S::FJ + fj) * S::THREADS];
    } else if constexpr (PHASE == kPartial) {
        int turn = 0, next = S::STAGES - 1;
        for (int32_t i = 0; i < all; ++i) {
            if (i + S::STAGES - 1 <= all) arrived<(S::STAGES - 2) * S::LOADS>();
            else arrived<0>();
            if (i + S::STAGES - 1 < all) load(i + S::STAGES - 1, next);
            next = next + 1 == S::STAGES ? 0 : next + 1;
            take(first, turn, 0);
            take(second, turn, 1);
            add(first.l, first.r);
            add_second(first, second);
            turn = turn + 1 == S::STAGES ? 0 : turn + 1;
        }
#pragma unroll
        for (int fi = 0; fi < S::FI; ++fi)
#pragma unroll
            for (int fj = 0; fj < S::FJ; ++fj) sums[(fi * S::FJ + fj) * S::THREADS] = acc[fi][fj];
        return;
    } else if constexpr (S::AHEAD) {
        // Operands are read from LDS while products are taken of those before: the second half of a part's with its first half's, and the next part's
        // first half, which has arrived by then, with the second half's.
        static_assert(!S::AHEAD || S::STAGES == 2, "a part has the step before to arrive in");
        if (all > 1) load(1, 1);
        if (all > 1) arrived<S::LOADS>();
        else arrived<0>();
        take(first, 0, 0);
        const auto step = [&](int32_t i, int turn, Operands& v, Operands& next) {
            take(second, turn, 1);
            add(v.l, v.r);
            arrived<0>();
            if (i + 2 < all) load(i + 2, turn);
            take(next, turn ^ 1, 0);
            add_second(v, second);
        };
        int32_t i = 0;
        if constexpr (TERMS == 2) {                      // (an even number of parts)
            Operands other;
            for (; i + 2 < all; i += 2) {
                step(i, 0, first, other);
                step(i + 1, 1, other, first);
            }
            step(i, 0, first, other);
            first = other;
            ++i;
        } else {
            for (; i + 1 < all; ++i) {
                Operands other;
                step(i, i & 1, first, other);
                first = other;
            }
        }
        take(second, i & 1, 1);
    } else {
        int turn = 0, next = S::STAGES - 1;
        for (int32_t i = 0; i + 1 < all; ++i) {
            if (i + S::STAGES - 1 <= all) arrived<(S::STAGES - 2) * S::LOADS>();
            else arrived<0>();
            if (i + S::STAGES - 1 < all) load(i + S::STAGES - 1, next);
            next = next + 1 == S::STAGES ? 0 : next + 1;
            take(first, turn, 0);
            take(second, turn, 1);
            add(first.l, first.r);
            add_second(first, second);
            turn = turn + 1 == S::STAGES ? 0 : turn + 1;
        }
        arrived<0>();
        take(first, turn, 0);
        take(second, turn, 1);
    }
    // What the last part of the output needs of A0 or X is on its way while the last products are taken (of a tile of 256 half of it, which
    // is what the registers have room for).
    constexpr bool READS = MODE != kGram, LOW = READS && (TERMS == 2 || !HALF);
    const int32_t row0 = t.ti * S::TI + wi * S::FI * 16 + (lane & 15) * S::GI, col = t.tj * S::TJ + wj * S::FJ * 16 + (lane >> 4) * N;
    const int32_t wide = HALF ? t.np : t.mp;             // of an output row
    const auto row_of = [&](int fi) { return row0 + fi / S::GI * 16 * S::GI + fi % S::GI; };
    Half8 hi[S::GI][N / 8], lo[S::GI][N / 8];
    const auto fetch = [&](int gi) {
        if constexpr (READS) {
#pragma unroll
            for (int f = 0; f < S::GI; ++f) {
                const int64_t from = Work<TERMS>::place(row_of(gi + f), col, wide);
#pragma unroll
                for (int e = 0; e < N / 8; ++e) {
                    hi[f][e] = *reinterpret_cast<const Half8*>((HALF ? w.a() : w.x(k.turn)) + from + 8 * e);
                    if constexpr (LOW) lo[f][e] = *reinterpret_cast<const Half8*>((HALF ? w.a() + 32 : w.x_low(k.turn)) + from + 8 * e);
                }
            }
        }
    };
    fetch(0);
    if (PHASE == kWhole) {
        add(first.l, first.r);
        add_second(first, second);
    }

    Update u = {};
    Matrix matrix;
    if constexpr (MODE == kFinish) {
        if (skipped(k.last.grad_scale)) return;
        matrix = list.matrices[t.matrix];
        u = update_of(k.last, matrix);
    }
    float dj[N];
    if constexpr (MODE == kSquare) {
#pragma unroll
        for (int e = 0; e < N; e += 4) {
            const Float4 d = *reinterpret_cast<const Float4*>(w.da() + col + e);
#pragma unroll
            for (int x = 0; x < 4; ++x) dj[e + x] = d[x];
        }
    }
    // (all in the unit of what is stored: 2^10 times; the products are 2^20 times)
#pragma unroll
    for (int gi = 0; gi < S::FI; gi += S::GI) {
        if (gi) fetch(gi);
        float out[MODE == kFinish ? S::GI : 1][N];
#pragma unroll
        for (int f = 0; f < S::GI; ++f) {
            const int fi = gi + f;
            const int32_t row = row_of(fi);
            const float d = MODE == kSquare ? fmaf(k.c, w.da()[row], k.b) : MODE == kGram ? 0.f : k.a + w.db()[row];
            float diagonal = 0.f;
            float(&v)[N] = out[MODE == kFinish ? f : 0];
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float c = acc[fi][e / 4][e % 4];
                float x = 0.f;
                if constexpr (READS) x = static_cast<float>(hi[f][e / 8][e % 8]);
                if constexpr (LOW) x += static_cast<float>(lo[f][e / 8][e % 8]);
                if (MODE == kGram) v[e] = c * kDown;
                else if (MODE == kSquare) v[e] = fmaf(fmaf(k.c, dj[e], d), x, c * (k.c * kDown));
                else v[e] = fmaf(d, x, c * kDown);
                if (HALF && row == col + e) {
                    diagonal = MODE == kGram ? c * (kDown * kDown) : fmaf(d, dj[e], c * (k.c * kDown * kDown));
                    v[e] = 0.f;
                }
            }
            if (HALF && row >= col && row < col + N) (MODE == kGram ? w.da() : w.db())[row] = diagonal;
            if constexpr (MODE == kFinish) {
#pragma unroll
                for (int e = 0; e < N; ++e) v[e] *= kDown;
            } else {
                const int64_t to = Work<TERMS>::place(row, col, wide);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    _Float16 h = static_cast<_Float16>(v[e]), l = h;
                    if (TERMS == 2 || MODE == kApply) split(v[e], h, l);
                    hi[f][e / 8][e % 8] = h, lo[f][e / 8][e % 8] = l;
                }
#pragma unroll
                for (int e = 0; e < N / 8; ++e) {
                    *reinterpret_cast<Half8*>((MODE == kGram ? w.a() : MODE == kSquare ? w.b() : w.x(1 - k.turn)) + to + 8 * e) = hi[f][e];
                    if (TERMS == 2 || MODE == kApply)
                        *reinterpret_cast<Half8*>((MODE == kGram ? w.a() + 32 : MODE == kSquare ? w.b() + 32 : w.x_low(1 - k.turn)) + to + 8 * e) = lo[f][e];
                }
            }
        }
        if constexpr (MODE == kFinish) finish(matrix, k.last.p_fmt, u, row_of(gi), col, out);
        // the tile on the other side of A and B
        if (!HALF || t.ti == t.tj) continue;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            typedef _Float16 Halves __attribute__((ext_vector_type(S::GI)));
            Halves h, l;
#pragma unroll
            for (int f = 0; f < S::GI; ++f) h[f] = hi[f][e / 8][e % 8], l[f] = lo[f][e / 8][e % 8];
            _Float16* const to = (MODE == kGram ? w.a() : w.b()) + Work<TERMS>::place(col + e, row_of(gi), t.np);
            *reinterpret_cast<Halves*>(to) = h;
            if (TERMS == 2) *reinterpret_cast<Halves*>(to + 32) = l;
        }
    }
}

// A small matrix (n <= 64, m <= M) a workgroup, in one launch: X in binary32 in registers, what the products read in LDS.  16 wavefronts, a block
// of 16 x 16 of A and M / 64 of X each: five steps are a chain of fifteen products and barriers (64 x 64, two terms: 2.3 us a step and
// 4 us besides, 15.9 in all, with four wavefronts of 2 x 2 blocks 17.2; one term 11.0; by tiles 70.  64 x 250, two terms: 31 and by tiles 66; 1000 of
// them 141 and 323).
constexpr int kLittleThreads = 1024;
typedef _Float16 Half4 __attribute__((ext_vector_type(4)));
template <int M, int TERMS>
struct Little {
    static constexpr int N = 64, F = M / 64, WIDE = M + 8, HIGH = N + 8;     // (rows 16 bytes further: 16 of them meet all banks)
    static constexpr int X = N * WIDE, A = N * HIGH;
    static constexpr int HALVES = TERMS * (X + 2 * A) + 2 * 2 * N;
    // A lane has a row of 4 F columns of X (4 each of F blocks) and 4 of A.
    _Float16 *const x_at, *const a_at, *const b_at;
    float *const da, *const db;
    const int lane, wi, wj, row, col, a_col;
    __device__ __forceinline__ explicit Little(_Float16* lds)
        : x_at(lds), a_at(x_at + TERMS * X), b_at(a_at + TERMS * A), da(reinterpret_cast<float*>(b_at + TERMS * A)), db(da + N),
          lane(threadIdx.x & 63), wi(threadIdx.x >> 8), wj(threadIdx.x >> 6 & 3), row(wi * 16 + (lane & 15)),
          col(wj * (M / 4) + (lane >> 4) * 4), a_col(wj * 16 + (lane >> 4) * 4) {}

    // four neighbouring values, and their lower halves
    static __device__ __forceinline__ void keep(const float (&v)[4], _Float16* at, int size) {
        Half4 h, l;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            _Float16 hi = static_cast<_Float16>(v[e]), lo = hi;
            if (TERMS == 2) split(v[e], hi, lo);
            h[e] = hi, l[e] = lo;
        }
        *reinterpret_cast<Half4*>(at) = h;
        if (TERMS == 2) *reinterpret_cast<Half4*>(at + size) = l;
    }
    __device__ __forceinline__ void keep_x(const float (&x)[F][4]) const {
#pragma unroll
        for (int f = 0; f < F; ++f) keep(x[f], x_at + row * WIDE + col + 16 * f, X);
    }
    // 8 values of K of a row a lane
    __device__ __forceinline__ void rows(Half8 (&v)[TERMS], const _Float16* at, int step, int size, int first, int q) const {
#pragma unroll
        for (int low = 0; low < TERMS; ++low)
            v[low] = *reinterpret_cast<const Half8*>(at + low * size + (first + (lane & 15)) * step + (lane >> 4) * 8 + q);
    }
    static __device__ __forceinline__ void add(Float4& acc, const Half8 (&l)[TERMS], const Half8 (&r)[TERMS]) {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(r[0], l[0], acc, 0, 0, 0);
        if (TERMS == 2) {
            acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(r[TERMS - 1], l[0], acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(r[0], l[TERMS - 1], acc, 0, 0, 0);
        }
    }
    // this wavefront's block of L L^T
    __device__ __forceinline__ Float4 square(const _Float16* at, int step, int size, int depth) const {
        Float4 acc = {};
#pragma unroll
        for (int q = 0; q < depth; q += 32) {
            Half8 l[TERMS], r[TERMS];
            rows(l, at, step, size, wi * 16, q);
            rows(r, at, step, size, wj * 16, q);
            add(acc, l, r);
        }
        return acc;
    }
    __device__ __forceinline__ Float4 gram() const { return square(x_at, WIDE, X, M); }
    // B from X X^T (`acc`; 2^20 times)
    __device__ __forceinline__ void polynomial(Float4 acc, float b, float c) const {
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = acc[e] * kDown;
            if (row == a_col + e) {
                da[row] = v[e] * kDown;
                v[e] = 0.f;
            }
        }
        keep(v, a_at + row * HIGH + a_col, A);
        __syncthreads();
        acc = square(a_at, HIGH, A, N);
        const float d = fmaf(c, da[row], b);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float dj = da[a_col + e];
            if (row == a_col + e) {
                db[row] = fmaf(d, dj, acc[e] * (c * kDown * kDown));
                v[e] = 0.f;
            } else {
                v[e] = fmaf(fmaf(c, dj, d), v[e], acc[e] * (c * kDown));
            }
        }
        keep(v, b_at + row * HIGH + a_col, A);
        __syncthreads();
    }
    // X = a X + B X
    __device__ __forceinline__ void apply(float a, float (&x)[F][4]) const {
        const float keeps = a + db[row];
#pragma unroll
        for (int f = 0; f < F; ++f) {
            Float4 acc = {};
#pragma unroll
            for (int q = 0; q < N; q += 32) {
                Half8 l[TERMS], r[TERMS];
                rows(l, b_at, HIGH, A, wi * 16, q);
                // columns of X, from its rows
#pragma unroll
                for (int low = 0; low < TERMS; ++low) {
                    typedef short Short4 __attribute__((ext_vector_type(4)));
                    typedef __attribute__((address_space(3))) Short4* Pointer;
                    union {
                        Short4 part[2];
                        Half8 all;
                    } of;
#pragma unroll
                    for (int h = 0; h < 2; ++h)
                        of.part[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                            (Pointer)(x_at + low * X + (q + (lane >> 4) * 8 + h * 4 + (lane >> 2 & 3)) * WIDE + wj * (M / 4) + 16 * f + (lane & 3) * 4));
                    r[low] = of.all;
                }
                add(acc, l, r);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) x[f][e] = fmaf(keeps, x[f][e], acc[e] * kDown);
        }
    }
    // A lane's elements of an array with the matrix's rows, of X's columns from `first` on (0 behind the end): all loads before the first conversion, as
    // what waits here is a workgroup alone (64 x 4096: the first launch 12.9 us with the loads one after the other).
    template <typename T>
    __device__ __forceinline__ void read(const Matrix& t, const T* p, int64_t stride, int32_t first, float (&v)[F][4]) const {
        T raw[F][4];
#pragma unroll
        for (int f = 0; f < F; ++f) {
            const int32_t at = first + col + 16 * f;
#pragma unroll
            for (int e = 0; e < 4; ++e) raw[f][e] = static_cast<T>(0.f);
            if (t.rows > t.cols) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (row < t.cols && at + e < t.rows) raw[f][e] = p[(at + e) * stride + row];
            } else if (row < t.rows && at + 4 <= t.cols) {
                __builtin_memcpy(raw[f], p + row * stride + at, sizeof(raw[f]));
            } else if (row < t.rows) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (at + e < t.cols) raw[f][e] = p[row * stride + at + e];
            }
        }
#pragma unroll
        for (int f = 0; f < F; ++f)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[f][e] = static_cast<float>(raw[f][e]);
    }
    __device__ __forceinline__ void read(const Matrix& t, const void* p, int fmt, int64_t stride, int32_t first, float (&v)[F][4]) const {
        if (fmt == CS_FMT_F32) read(t, static_cast<const float*>(p), stride, first, v);
        else if (fmt == CS_FMT_BF16) read(t, static_cast<const bf16*>(p), stride, first, v);
        else read(t, static_cast<const f16*>(p), stride, first, v);
    }
    // u of the columns from `first` on, the moment's step taken; returns the sum of its squares, in every lane
    __device__ __forceinline__ double begin(const Matrix& t, const Moment& k, int32_t first, float (&x)[F][4],
                                            double (&buf)[kLittleThreads / 64]) const {
        const float s = k.grad_scale ? *k.grad_scale : 1.f;
        float m[F][4];
        if (t.moment) read(t, t.moment, t.cols, first, m);
        read(t, t.g, k.g_fmt, t.g_stride, first, x);
        if (t.moment) {
#pragma unroll
            for (int f = 0; f < F; ++f) {
                const int32_t at = first + col + 16 * f;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    m[f][e] = fmaf(k.mu, m[f][e], s * x[f][e]);
                    x[f][e] = k.nesterov ? fmaf(k.mu, m[f][e], s * x[f][e]) : m[f][e];
                }
                if (t.rows > t.cols) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (row < t.cols && at + e < t.rows) t.moment[static_cast<int64_t>(at + e) * t.cols + row] = m[f][e];
                } else if (row < t.rows) {
                    float* const to = t.moment + static_cast<int64_t>(row) * t.cols + at;
                    if (at + 4 <= t.cols) {
                        __builtin_memcpy(to, m[f], sizeof(m[f]));
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (at + e < t.cols) to[e] = m[f][e];
                    }
                }
            }
        }
        double sum = 0.;
#pragma unroll
        for (int f = 0; f < F; ++f)
#pragma unroll
            for (int e = 0; e < 4; ++e) sum = fma(static_cast<double>(x[f][e]), static_cast<double>(x[f][e]), sum);
#pragma unroll
        for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
        if (lane == 0) buf[threadIdx.x >> 6] = sum;
        __syncthreads();
        sum = buf[lane & 15];
#pragma unroll
        for (int d = 8; d; d >>= 1) sum += __shfl_xor(sum, d);
        return sum;
    }
    __device__ __forceinline__ void end(const Matrix& t, const Last& last, int32_t first, float (&x)[F][4]) const {
        const Update u = update_of(last, t);
        float old[F][4];
        if (u.optimizer) read(t, t.p, last.p_fmt, t.p_stride, first, old);
#pragma unroll
        for (int f = 0; f < F; ++f) {
            const int32_t at = first + col + 16 * f;
#pragma unroll
            for (int e = 0; e < 4; ++e) x[f][e] = u.optimizer ? fmaf(old[f][e], u.keep, -u.lr * (x[f][e] * kDown)) : x[f][e] * kDown;
            if (t.rows > t.cols) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float one[1] = {x[f][e]};
                    write_p(t, last.p_fmt, at + e, row, one);
                }
            } else {
                write_p(t, last.p_fmt, row, at, x[f]);
            }
        }
    }
};
template <int M, int TERMS>
__global__ void __launch_bounds__(kLittleThreads) k_muon_little(List list, Moment moment, double eps, Steps steps, Last last) {
    using L = Little<M, TERMS>;
    __shared__ __align__(16) _Float16 lds[L::HALVES];
    __shared__ double buf[kLittleThreads / 64];
    if (skipped(last.grad_scale)) return;
    const Matrix t = list.matrices[blockIdx.x];
    const L w(lds);
    float x[L::F][4];
    const double one = inverse_of(w.begin(t, moment, 0, x, buf), eps) * static_cast<double>(kUp);
#pragma unroll
    for (int f = 0; f < L::F; ++f)
#pragma unroll
        for (int e = 0; e < 4; ++e) x[f][e] = static_cast<float>(x[f][e] * one);
    for (int i = 0; i < steps.count; ++i) {
        w.keep_x(x);
        __syncthreads();
        w.polynomial(w.gram(), steps.coefs[i][1], steps.coefs[i][2]);
        w.apply(steps.coefs[i][0], x);
        __syncthreads();
    }
    w.end(t, last, 0, x);
}

// A thin matrix (n <= 64, longer ones) in slabs of 256 columns, a workgroup each and a launch a step: it adds up the slabs' X X^T of the step before in
// their order, makes B of it (every workgroup the same), takes its slab to the next X and leaves that one's X X^T.  The first launch has no norm
// yet: it leaves u, and u u^T with u by the slab's own norm.
constexpr int kSlab = 256, kMaxSlabs = 32;
struct Slabs {
    Float4* x;                               // u or X, of a slab F x kLittleThreads
    Float4* all_sums;                        // X X^T, of a slab kLittleThreads, twice (read and written in turns)
    double* squares;                         // a slab each
    int32_t slabs;
    __device__ __forceinline__ Slabs(char* ws, const Matrix& t) {
        slabs = t.mp / kSlab;
        x = reinterpret_cast<Float4*>(ws + t.at);
        all_sums = x + slabs * (kSlab / 64 * kLittleThreads);
        squares = reinterpret_cast<double*>(all_sums + 2 * slabs * kLittleThreads);
    }
    __device__ __forceinline__ Float4* sums(int turn) const { return all_sums + turn * slabs * kLittleThreads + threadIdx.x; }
};
int64_t slab_bytes(int64_t slabs) { return slabs * ((kSlab / 64 + 2) * kLittleThreads * 16 + 16); }

template <int TERMS>
__global__ void __launch_bounds__(kLittleThreads) k_muon_slab_begin(List list, Moment moment, double eps, char* ws) {
    using L = Little<kSlab, TERMS>;
    __shared__ __align__(16) _Float16 lds[L::HALVES];
    __shared__ double buf[kLittleThreads / 64];
    if (skipped(moment.grad_scale)) return;
    const Place at = list.slabs[blockIdx.x];
    const Matrix t = list.matrices[at.matrix];
    const Slabs k(ws, t);
    const L w(lds);
    float x[L::F][4];
    const double sum = w.begin(t, moment, at.local * kSlab, x, buf);
    const double one = inverse_of(sum, eps) * static_cast<double>(kUp);
#pragma unroll
    for (int f = 0; f < L::F; ++f) {
        k.x[(at.local * L::F + f) * kLittleThreads + threadIdx.x] = Float4{x[f][0], x[f][1], x[f][2], x[f][3]};
#pragma unroll
        for (int e = 0; e < 4; ++e) x[f][e] = static_cast<float>(x[f][e] * one);
    }
    w.keep_x(x);
    __syncthreads();
    k.sums(0)[at.local * kLittleThreads] = w.gram();
    if (threadIdx.x == 0) k.squares[at.local] = sum;
}
template <int TERMS>
__global__ void __launch_bounds__(kLittleThreads) k_muon_slab(List list, Steps steps, int step, double eps, Last last, char* ws) {
    using L = Little<kSlab, TERMS>;
    __shared__ __align__(16) _Float16 lds[L::HALVES];
    if (skipped(last.grad_scale)) return;
    const Place at = list.slabs[blockIdx.x];
    const Matrix t = list.matrices[at.matrix];
    const Slabs k(ws, t);
    const L w(lds);
    float x[L::F][4];
#pragma unroll
    for (int f = 0; f < L::F; ++f) {
        const Float4 v = k.x[(at.local * L::F + f) * kLittleThreads + threadIdx.x];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[f][e] = v[e];
    }
    const Float4* const sums = k.sums(step & 1);
    Float4 acc = {};
    if (step == 0) {
        double sum = 0.;
        for (int i = 0; i < k.slabs; ++i) sum += k.squares[i];
        const double one = inverse_of(sum, eps);
        for (int i = 0; i < k.slabs; ++i) {
            const double own = k.squares[i], r = own == 0. ? 0. : one / inverse_of(own, eps);
            acc += sums[i * kLittleThreads] * static_cast<float>(r * r);
        }
#pragma unroll
        for (int f = 0; f < L::F; ++f)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[f][e] = static_cast<float>(x[f][e] * (one * static_cast<double>(kUp)));
    } else {
#pragma unroll 8
        for (int i = 0; i < k.slabs; ++i) acc += sums[i * kLittleThreads];
    }
    w.keep_x(x);
    w.polynomial(acc, steps.coefs[step][1], steps.coefs[step][2]);
    w.apply(steps.coefs[step][0], x);
    if (step + 1 == steps.count) {
        w.end(t, last, at.local * kSlab, x);
        return;
    }
    __syncthreads();
    w.keep_x(x);
#pragma unroll
    for (int f = 0; f < L::F; ++f)
        k.x[(at.local * L::F + f) * kLittleThreads + threadIdx.x] = Float4{x[f][0], x[f][1], x[f][2], x[f][3]};
    __syncthreads();
    k.sums(1 - (step & 1))[at.local * kLittleThreads] = w.gram();
}

// ---------------------------------------------------------------------------------------
constexpr int64_t kMaxSide = 1 << 20, kMaxShort = 1 << 15, kMaxMatrices = 1 << 20, kMaxPlaces = static_cast<int64_t>(1) << 24;

// Kinds of tiles: edges, how many are on the GPU at once, and how long they take (us) for a part of 64 values of K, with one, two or three on a CU, and
// besides.  Of 52 lists (one of 90 x 90, 200 of 100 x 100, 40 of 700 x 700, 36 of 512 x 2048, one of 4096 x 2048, ..; one and two terms) that were
// timed in all kinds of tiles, those that these numbers choose are 0.3 % slower than the best on average and 2.5 % at most; of 16 others 1 % and
// 5.6 %.
struct Kind {
    int high, wide, at_once;
    double step[3], besides;
};
constexpr Kind kHalfKinds[] = {{64, 64, 768, {0.28, 0.5, 0.5}, 3.}, {128, 128, 512, {0.45, 0.87}, 8.}};
constexpr Kind kFullKinds[] = {{64, 64, 768, {0.28, 0.5, 0.5}, 3.}, {64, 128, 768, {0.4, 0.6, 0.95}, 5.}, {128, 128, 512, {0.68, 1.05}, 6.}, {256, 256, 256, {1.65}, 14.}};
constexpr int kHalfKindsN = 2, kFullKindsN = 4;
constexpr int kMaxSlices = 32;
constexpr int64_t kPartialBytes = 64 * 64 * 4;       // of a tile's slice

struct Plan {
    int64_t matrices, littles, thins, slabs, pieces, halves, tails, fulls, work;     // tails: quarters of the last tiles; work: bytes of all matrices
    int64_t most_pieces;                                                 // of a matrix in tiles
    double gram_steps, square_steps, full_steps;                         // parts of 64 values of K (both halves of them), of all tiles together
    int half_kind, full_kind;
    int slices[2];                                                       // of K, of X X^T and of A A in tiles of 64
};
int64_t up_to(int64_t n, int64_t unit) { return (n + unit - 1) / unit * unit; }

bool stack_ok(const cs_matrix& s) {
    return s.count >= 0 && s.count <= kMaxMatrices && s.rows >= 0 && s.cols >= 0 && s.rows <= kMaxSide && s.cols <= kMaxSide &&
           (s.rows < s.cols ? s.rows : s.cols) <= kMaxShort;
}
bool there(const cs_matrix& s) { return s.count > 0 && s.rows > 0 && s.cols > 0; }
// Matrices that a workgroup takes from their moments to their parameters.
bool little(const cs_matrix& s) { return (s.rows <= 64 || s.cols <= 64) && s.rows <= 256 && s.cols <= 256; }
// Matrices that may be taken in slabs, and how many of each.  All of them are if that is no more than a workgroup on every CU (us, slabs / tiles, two
// terms: 1 of 64 x 4096 70 / 110, 16 of 64 x 4096 104 / 159, 64 of 64 x 1024 86 / 137; more than that read each other's sums too often: 400 of
// 64 x 500 260 / 236, 10 of 64 x 8192 194 / 173).
bool thin(const cs_matrix& s) {
    const int64_t n = s.rows < s.cols ? s.rows : s.cols, m = s.rows < s.cols ? s.cols : s.rows;
    return n <= 64 && !little(s) && m <= kMaxSlabs * kSlab;
}
int64_t slabs_of(const cs_matrix& s) { return ((s.rows < s.cols ? s.cols : s.rows) + kSlab - 1) / kSlab; }
bool in_slabs(const cs_matrix* stacks, int32_t n) {
    int64_t slabs = 0;
    for (int32_t i = 0; i < n; ++i) {
        if (!stack_ok(stacks[i])) return false;
        if (there(stacks[i]) && thin(stacks[i])) slabs += stacks[i].count * slabs_of(stacks[i]);
        if (slabs > 256) return false;
    }
    return true;
}

// Counts and sizes with these tiles; `each` is told of every stack that has tiles.
template <typename F>
bool plan_with(const cs_matrix* stacks, int32_t n, int terms, int half_kind, int full_kind, Plan& plan, F each) {
    plan = Plan{};
    plan.half_kind = half_kind, plan.full_kind = full_kind;
    const int64_t half_tile = kHalfKinds[half_kind].high, full_high = kFullKinds[full_kind].high, full_wide = kFullKinds[full_kind].wide;
    const int64_t tile = half_tile > full_high ? half_tile : full_high;
    const bool slabs_too = in_slabs(stacks, n);
    for (int32_t i = 0; i < n; ++i) {
        const cs_matrix& s = stacks[i];
        if (!stack_ok(s)) return false;
        if (!there(s)) continue;
        plan.matrices += s.count;
        if (plan.matrices > kMaxMatrices) return false;
        if (little(s)) {
            plan.littles += s.count;
            continue;
        }
        if (slabs_too && thin(s)) {
            const int64_t slabs = slabs_of(s);
            each(s, 64, slabs * kSlab, plan, slabs, 0, 0);
            plan.thins += s.count;
            plan.slabs += s.count * slabs;
            plan.work += s.count * slab_bytes(slabs);
            continue;
        }
        const int64_t np = up_to(s.rows < s.cols ? s.rows : s.cols, tile), mp = up_to(s.rows < s.cols ? s.cols : s.rows, full_wide);
        const int64_t down = np / half_tile, pieces = (np / kEdge) * (mp / kEdge), halves = down * (down + 1) / 2;
        const int64_t fulls = (np / full_high) * (mp / full_wide);
        each(s, np, mp, plan, pieces, halves, fulls);
        plan.pieces += s.count * pieces;
        if (pieces > plan.most_pieces) plan.most_pieces = pieces;
        plan.halves += s.count * halves;
        plan.fulls += s.count * fulls;
        plan.gram_steps += static_cast<double>(s.count * halves) * mp * terms / 64;
        plan.square_steps += static_cast<double>(s.count * halves) * np * terms / 64;
        plan.full_steps += static_cast<double>(s.count * fulls) * np * terms / 64;
        plan.work += s.count * work_bytes(np, mp, terms);
        if (plan.pieces >= kMaxPlaces) return false;
    }
    return true;
}
// How long so many tiles take with so many parts of K each, in rounds of what is on the GPU at once (a last round of few takes less).
double time_of(const Kind& kind, int64_t tiles, double steps) {
    const int64_t rounds = tiles / kind.at_once, left = tiles % kind.at_once;
    const auto round = [&](int64_t on_a_cu) { return kind.step[on_a_cu - 1] * steps + kind.besides; };
    return static_cast<double>(rounds) * round(kind.at_once / 256) + (left ? round((left + 255) / 256) : 0.);
}
// The same of tiles of 64, in as many slices of K as are best.  A launch to join n of them is 4.5 us and 0.15 a slice (256 x 4096: X X^T 18 us whole, in
// 32 slices 5.5 and 9.5).
double time_in_slices(int64_t tiles, double steps, int& slices) {
    double least = INFINITY;
    for (int n = 1; n <= kMaxSlices && (n == 1 || (tiles * n <= 768 && n * 2 <= steps)); n *= 2) {
        const double us = time_of(kHalfKinds[0], tiles * n, steps / n) + (n > 1 ? 4.5 + 0.15 * n : 0.);
        if (us < least) {
            least = us;
            slices = n;
        }
    }
    return least;
}
// A symmetric product.  Few tiles of 128 left by the last round would take nearly half as long as a whole one where K is long (528 tiles of 4096 x 4096:
// 70 us for 512 and 29 for the 16 that are left): they are taken as tiles of 64, four each, `tails` (12 us, in slices).
double half_time(int kind, int64_t tiles, double steps, int64_t tails, int& slices) {
    if (kind == 0) return time_in_slices(tiles, steps, slices);
    slices = 1;
    return time_of(kHalfKinds[1], tiles - tails / 4, steps) + (tails ? time_in_slices(tails, steps, slices) : 0.);
}
bool plan_of(const cs_matrix* stacks, int32_t n, int terms, Plan& plan) {
    const auto none = [](const cs_matrix&, int64_t, int64_t, const Plan&, int64_t, int64_t, int64_t) {};
    double least = INFINITY;
    bool ok = false;
    for (int half = 0; half < kHalfKindsN; ++half)
        for (int full = 0; full < kFullKindsN; ++full) {
            Plan whole;
            // (larger tiles fill up more: they may be too many where smaller ones are not)
            if (!plan_with(stacks, n, terms, half, full, whole, none)) continue;
            const int64_t halves = whole.halves, left = halves % kHalfKinds[half].at_once;
            for (const int64_t tails : {static_cast<int64_t>(0), half == 1 ? 4 * left : 0}) {
                Plan p = whole;
                p.halves -= tails / 4;
                p.tails = tails;
                const double us = halves ? half_time(half, halves, p.gram_steps / static_cast<double>(halves), tails, p.slices[0]) +
                                               half_time(half, halves, p.square_steps / static_cast<double>(halves), tails, p.slices[1]) +
                                               time_of(kFullKinds[full], p.fulls, p.full_steps / static_cast<double>(p.fulls)) : 0.;
                if (us < least) {
                    least = us;
                    plan = p;
                    ok = true;
                }
            }
        }
    return ok;
}
// tiles of 64 that may be in slices, and what their products need of the workspace
int64_t sliced_tiles(int half_kind, int64_t halves, int64_t tails) { return half_kind == 0 ? halves : tails; }
int64_t partial_bytes(const cs_matrix_list* l) {
    const int most = l->gram_slices > l->square_slices ? l->gram_slices : l->square_slices;
    return most > 1 ? sliced_tiles(l->half_kind, l->halves, l->tails) * most * kPartialBytes : 0;
}
size_t list_bytes(const Plan& p) {
    return static_cast<size_t>(p.matrices) * sizeof(Matrix) + static_cast<size_t>(p.halves + p.tails + p.fulls) * sizeof(Tile) +
           static_cast<size_t>(p.pieces + p.slabs) * sizeof(Place);
}
size_t workspace_bytes(const cs_matrix_list* l) {
    return static_cast<size_t>(l->work + partial_bytes(l)) + static_cast<size_t>(l->pieces) * sizeof(double);
}
List list_of(const cs_matrix_list* l) {
    const Matrix* t = static_cast<const Matrix*>(l->memory);
    const Tile* at = reinterpret_cast<const Tile*>(t + l->matrices);
    const Place* const pieces = reinterpret_cast<const Place*>(at + l->halves + l->tails + l->fulls);
    return List{t, at, at + l->halves + l->tails, pieces, pieces + l->pieces};
}
bool list_ok(const cs_matrix_list* l) {
    return l && l->most_pieces >= 0 && l->littles >= 0 && l->thins >= 0 && l->matrices >= l->littles + l->thins && l->slabs >= 0 && l->pieces >= 0 && l->halves >= 0 && l->tails >= 0 && l->fulls >= 0 &&
           l->work >= 0 && l->half_kind >= 0 && l->half_kind < kHalfKindsN && l->full_kind >= 0 && l->full_kind < kFullKindsN &&
           l->gram_slices >= 0 && l->gram_slices <= kMaxSlices && l->square_slices >= 0 && l->square_slices <= kMaxSlices &&
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

// A tile's wavefronts, for symmetric products (HALF) and for B X.  Few parts of K are over soon, and more wavefronts a SIMD hide what each
// waits for; large tiles have registers for two, and read LDS a step ahead instead.  us, symmetric products / B X:
//   48 of 512 x 512       128 x 128 as 4 x 2 wavefronts 14.5 + 16.0 / 34.7, as 2 x 2 ahead 16.2 + 18.0 / 33.5; 64 x 128 as 2 x 2 / 31.2, as 2 x 4 / 29.6
//   4096 x 4096           128 x 128 as 4 x 2 wavefronts 100 + 102 / 153, as 2 x 2 ahead 96.6 + 100.4 / 144; 256 x 256 / 144, ahead / 122
//   12 of 2048 x 512, two terms   128 x 128 as 2 x 4 wavefronts 43.9 + 17.8 / 49.1, ahead 46.6 + 18.4 / 47.2; 64 x 64 31.3 + 12.4 / 60
template <int HIGH, int WIDE, int TERMS, bool HALF>
struct ShapeOf;
template <int TERMS, bool HALF>
struct ShapeOf<64, 64, TERMS, HALF> : Shape<2, 2, 2, 2, 3, 3, false> {};
template <int TERMS>
struct ShapeOf<64, 128, TERMS, false> : Shape<2, 4, 2, 2, 2, 6, false> {};
template <>
struct ShapeOf<128, 128, 1, true> : Shape<4, 2, 2, 4, 2, 4, false> {};
template <>
struct ShapeOf<128, 128, 1, false> : Shape<2, 2, 4, 4, 2, 2, true> {};
template <>
struct ShapeOf<128, 128, 2, true> : Shape<2, 4, 4, 2, 2, 4, false> {};
template <>
struct ShapeOf<128, 128, 2, false> : Shape<2, 4, 4, 2, 2, 4, true> {};
template <int TERMS>
struct ShapeOf<256, 256, TERMS, false> : Shape<2, 4, 8, 4, 2, 2, TERMS == 1> {};

template <int TERMS, int MODE, int HIGH, int WIDE, int PHASE = kWhole>
int product_as(const List& list, int64_t places, const Product& k, char* ws, hipStream_t s) {
    using S = ShapeOf<HIGH, WIDE, TERMS, MODE == kGram || MODE == kSquare>;
    static_assert(S::TI == HIGH && S::TJ == WIDE, "");
    k_muon_product<S, TERMS, MODE, PHASE><<<static_cast<unsigned>(places), S::THREADS, 0, s>>>(list, k, ws);
    return launched();
}
template <int TERMS, int MODE>
int product(const cs_matrix_list* l, Product k, char* ws, hipStream_t s) {
    List list = list_of(l);
    if constexpr (MODE == kGram || MODE == kSquare) {
        int64_t tiles = l->halves;
        if (l->half_kind == 1) {
            if (l->halves)
                if (int rc = product_as<TERMS, MODE, 128, 128>(list, l->halves, k, ws, s)) return rc;
            list.halves += l->halves;
            tiles = l->tails;
        }
        if (tiles == 0) return CS_OK;
        k.slices = MODE == kGram ? l->gram_slices : l->square_slices;
        if (k.slices <= 1) return product_as<TERMS, MODE, 64, 64>(list, tiles, k, ws, s);       // (partial_bytes() has room for slices only)
        k.partials = reinterpret_cast<Float4*>(ws + l->work);
        if (int rc = product_as<TERMS, MODE, 64, 64, kPartial>(list, tiles * k.slices, k, ws, s)) return rc;
        return product_as<TERMS, MODE, 64, 64, kJoin>(list, tiles, k, ws, s);
    } else {
        switch (l->full_kind) {
            case 0: return product_as<TERMS, MODE, 64, 64>(list, l->fulls, k, ws, s);
            case 1: return product_as<TERMS, MODE, 64, 128>(list, l->fulls, k, ws, s);
            case 2: return product_as<TERMS, MODE, 128, 128>(list, l->fulls, k, ws, s);
            default: return product_as<TERMS, MODE, 256, 256>(list, l->fulls, k, ws, s);
        }
    }
}

// Pieces of a list's largest matrix up to which every workgroup that begins X sums their squares by itself, in place of a launch that does
// (4096 x 4096, 4096 pieces: that launch is 6 us).  Workgroups by themselves read the square of a matrix's pieces: 8192 x 8192 beside 100 of
// 128 x 128 216 us, with the launch 85 and 18.
constexpr int64_t kSquaresEach = 1024;

template <int TERMS>
int run_as(const cs_muon* h, const cs_matrix_list* l, bool optimizer, const double* lr, const float* grad_scale, char* ws, hipStream_t s) {
    const List at = list_of(l);
    const Moment moment = {static_cast<float>(h->momentum), optimizer ? h->nesterov : 0, l->g_fmt, grad_scale};
    Last last = {l->p_fmt, optimizer, h->scale, static_cast<float>(1. - h->lr * h->weight_decay), static_cast<float>(h->lr),
                 static_cast<float>(h->weight_decay), lr, grad_scale};
    Steps steps = {h->steps, {}};
    for (int i = 0; i < h->steps; ++i)
        for (int e = 0; e < 3; ++e) steps.coefs[i][e] = static_cast<float>(h->coefs[i][e]);
    if (l->littles) {
        const auto kernel = l->little_cols <= 64 ? k_muon_little<64, TERMS> : l->little_cols <= 128 ? k_muon_little<128, TERMS> : k_muon_little<256, TERMS>;
        kernel<<<static_cast<unsigned>(l->littles), kLittleThreads, 0, s>>>(at, moment, h->eps, steps, last);
        if (int rc = launched()) return rc;
    }
    if (l->thins) {
        const unsigned slabs = static_cast<unsigned>(l->slabs);
        k_muon_slab_begin<TERMS><<<slabs, kLittleThreads, 0, s>>>(at, moment, h->eps, ws);
        for (int i = 0; i < h->steps; ++i) k_muon_slab<TERMS><<<slabs, kLittleThreads, 0, s>>>(at, steps, i, h->eps, last, ws);
        if (int rc = launched()) return rc;
    }
    const int64_t before = l->littles + l->thins;
    if (l->matrices == before) return CS_OK;
    double* const squares = reinterpret_cast<double*>(ws + l->work + partial_bytes(l));
    const unsigned pieces = static_cast<unsigned>(l->pieces);
    k_muon_moment<<<pieces, kThreads, 0, s>>>(at, moment, squares);
    const bool joined = l->most_pieces > kSquaresEach;
    if (joined) {
        List others = at;
        others.matrices += before;
        k_muon_norm<<<static_cast<unsigned>(l->matrices - before), kThreads, 0, s>>>(others, squares);
    }
    k_muon_begin<TERMS><<<pieces, kThreads, 0, s>>>(at, moment, h->eps, squares, joined, ws);
    if (int rc = launched()) return rc;
    for (int i = 0; i < h->steps; ++i) {
        const Product k = {steps.coefs[i][0], steps.coefs[i][1], steps.coefs[i][2], i & 1, last, 1, nullptr};
        if (int rc = product<TERMS, kGram>(l, k, ws, s)) return rc;
        if (int rc = product<TERMS, kSquare>(l, k, ws, s)) return rc;
        if (int rc = i + 1 < h->steps ? product<TERMS, kApply>(l, k, ws, s) : product<TERMS, kFinish>(l, k, ws, s)) return rc;
    }
    return CS_OK;
}
int run(const cs_muon* h, const cs_matrix_list* l, bool optimizer, const double* lr, const float* grad_scale, void* workspace, size_t ws_bytes,
        void* stream) {
    if (!hyper_ok(h) || !list_ok(l) || (l->matrices && l->moments != (optimizer ? 1 : 0))) return CS_EINVAL;
    if (l->matrices == 0) return CS_OK;
    const size_t need = workspace_bytes(l);
    if (ws_bytes < need) return CS_EWORKSPACE;
    if (need && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 15))) return CS_EINVAL;
    Plan plan = {};
    plan.matrices = l->matrices, plan.slabs = l->slabs, plan.pieces = l->pieces, plan.halves = l->halves, plan.tails = l->tails, plan.fulls = l->fulls;
    const Span written[] = {{need ? workspace : nullptr, static_cast<int64_t>(need)}};
    const Span read[] = {{l->memory, static_cast<int64_t>(list_bytes(plan))}, {lr, 8}, {grad_scale, 4}};
    if (!spans_apart(written, read)) return CS_EINVAL;
    char* const ws = static_cast<char*>(workspace);
    const hipStream_t s = stream_of(stream);
    return l->terms == 1 ? run_as<1>(h, l, optimizer, lr, grad_scale, ws, s) : run_as<2>(h, l, optimizer, lr, grad_scale, ws, s);
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
    int64_t little_cols = 0;                 // the longest side of the small ones
    for (int32_t i = 0; i < count; ++i)
        if (there(stacks[i]) && little(stacks[i])) {
            const int64_t side = stacks[i].rows > stacks[i].cols ? stacks[i].rows : stacks[i].cols;
            if (side > little_cols) little_cols = side;
        }
    *list = cs_matrix_list{memory, plan.matrices, plan.littles, plan.thins, plan.slabs, plan.pieces, plan.halves, plan.tails, plan.fulls, plan.work, p_fmt, g_fmt, terms,
                           moments == 1, plan.half_kind, plan.full_kind, plan.slices[0], plan.slices[1], static_cast<int32_t>(little_cols),
                           static_cast<int32_t>(plan.most_pieces)};
    if (plan.matrices == 0) return CS_OK;
    Matrix* const matrices = static_cast<Matrix*>(memory);
    const hipStream_t st = stream_of(stream);
    Batch b = {};
    int filled = 0, rc = CS_OK;
    int64_t done = 0;
    const auto flush = [&] {
        if (!filled) return;
        if (!rc) {
            k_list_matrices<<<1, 64, 0, st>>>(b, matrices + done, filled);
            rc = launched();
        }
        done += filled;
        filled = 0;                          // (after a launch that failed too: the next matrices need the room)
    };
    const auto take = [&](const cs_matrix& s, int64_t k, Matrix more) {
        Matrix& t = b.t[filled];
        t = more;
        t.p = static_cast<char*>(s.p) + k * s.p_step * pb;
        t.g = static_cast<const char*>(s.g) + k * s.g_step * gb;
        t.moment = s.m ? s.m + k * s.rows * s.cols : nullptr;
        t.p_stride = s.p_stride, t.g_stride = s.g_stride;
        t.rows = static_cast<int32_t>(s.rows), t.cols = static_cast<int32_t>(s.cols);
        if (++filled == kBatch) flush();
    };
    // the small ones first, then the thin ones
    for (int32_t i = 0; i < count; ++i)
        if (there(stacks[i]) && little(stacks[i]))
            for (int64_t k = 0; k < stacks[i].count; ++k) take(stacks[i], k, Matrix{});
    const bool slabs_too = in_slabs(stacks, count);
    for (const bool thins : {true, false}) {
        Plan again;
        plan_with(stacks, count, terms, plan.half_kind, plan.full_kind, again,
                  [&](const cs_matrix& s, int64_t np, int64_t mp, const Plan& at, int64_t pieces, int64_t halves, int64_t fulls) {
            if ((slabs_too && thin(s)) != thins) return;
            for (int64_t k = 0; k < s.count; ++k) {
                Matrix t = {};
                t.at = at.work + k * (thins ? slab_bytes(pieces) : work_bytes(np, mp, terms));
                t.np = static_cast<int32_t>(np), t.mp = static_cast<int32_t>(mp);
                t.first_piece = static_cast<int32_t>((thins ? at.slabs : at.pieces) + k * pieces), t.pieces = static_cast<int32_t>(pieces);
                t.first_half = static_cast<int32_t>(at.halves + k * halves), t.first_full = static_cast<int32_t>(at.fulls + k * fulls);
                take(s, k, t);
            }
        });
    }
    flush();
    if (rc) return rc;
    Tile* const halves = reinterpret_cast<Tile*>(matrices + plan.matrices);
    Tile *const tails = halves + plan.halves, *const fulls = tails + plan.tails;
    const auto grid = [](int64_t n) { return static_cast<unsigned>((n + kThreads - 1) / kThreads); };
    const int thins = static_cast<int>(plan.littles), first = static_cast<int>(plan.littles + plan.thins), n = static_cast<int>(plan.matrices);
    Place *const pieces = reinterpret_cast<Place*>(fulls + plan.fulls), *const slabs = pieces + plan.pieces;
    if (plan.slabs) k_list_places<kPieces><<<grid(plan.slabs), kThreads, 0, st>>>(matrices, thins, first, kEdge, kEdge, slabs, plan.slabs, 0);
    if (first == n) return launched();
    const Kind &half = kHalfKinds[plan.half_kind], &full = kFullKinds[plan.full_kind];
    if (plan.halves) k_list_places<kHalves><<<grid(plan.halves), kThreads, 0, st>>>(matrices, first, n, half.high, half.wide, halves, plan.halves, 0);
    if (plan.tails) k_list_places<kTails><<<grid(plan.tails), kThreads, 0, st>>>(matrices, first, n, half.high, half.wide, tails, plan.tails, plan.halves);
    k_list_places<kFulls><<<grid(plan.fulls), kThreads, 0, st>>>(matrices, first, n, full.high, full.wide, fulls, plan.fulls, 0);
    k_list_places<kPieces><<<grid(plan.pieces), kThreads, 0, st>>>(matrices, first, n, kEdge, kEdge, pieces, plan.pieces, 0);
    if (int e = launched()) return e;
    return CS_OK;
}

extern "C" int cs_muon_workspace_bytes(const cs_matrix_list* list, size_t* bytes) {
    if (!list_ok(list) || !bytes) return CS_EINVAL;
    *bytes = workspace_bytes(list);
    return CS_OK;
}

extern "C" int cs_muon_step(const cs_muon* h, const cs_matrix_list* list, const double* lr_or_null, const float* grad_scale_or_null,
                            void* workspace, size_t ws_bytes, void* stream) {
    return run(h, list, true, lr_or_null, grad_scale_or_null, workspace, ws_bytes, stream);
}

extern "C" int cs_orthogonalize(const cs_muon* h, const cs_matrix_list* list, void* workspace, size_t ws_bytes, void* stream) {
    return run(h, list, false, nullptr, nullptr, workspace, ws_bytes, stream);
}

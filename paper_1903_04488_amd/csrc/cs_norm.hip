// Layer norm of rows, forward and backward with the gradients of weight and bias.
//     mu = mean x, rstd = 1 / sqrt(mean (x - mu)^2 + eps), xh = (x - mu) rstd, y = xh w + b
//     a = w dy,  dx = rstd (a - mean a - xh mean(a xh)),  dw = sum_rows dy xh,  db = sum_rows dy
// All sums in binary32; each output is rounded to its type once.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "cs_rows.h"
#include "csketch.h"

namespace cs {
namespace {

constexpr int kNormBlock = 256;

// ---------------------------------------------------------------------------------------
// Rows of any length, a value at a time: the forms for what the packed kernels below do not take (rows shorter than a pack, and longer
// than what is held).  A row is read three times, from the caches after the first.  With these alone: 32768 x 4096 bf16 with
// gradients 968 us, 8192 x 512 f32 37.
// ---------------------------------------------------------------------------------------
template <typename T, typename W>
__global__ void __launch_bounds__(kNormBlock)
k_norm_any(const T* x, int64_t x_stride, int64_t rows, int64_t cols, const W* weight, const W* bias, float eps, T* y,
           int64_t y_stride, float* mean, float* rstd) {
    __shared__ float lds[2][1][16];
    int turn = 0;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const T* xr = x + row * x_stride;
        float s[1] = {0.f};
        for (int64_t c = threadIdx.x; c < cols; c += kNormBlock) s[0] += static_cast<float>(xr[c]);
        block_sums<kNormBlock>(s, lds, turn);
        const float mu = s[0] / static_cast<float>(cols);
        float q[1] = {0.f};
        for (int64_t c = threadIdx.x; c < cols; c += kNormBlock) {
            const float d = static_cast<float>(xr[c]) - mu;
            q[0] = fmaf(d, d, q[0]);
        }
        block_sums<kNormBlock>(q, lds, turn);
        const float rs = 1.0f / sqrtf(q[0] / static_cast<float>(cols) + eps);
        T* yr = y + row * y_stride;
        for (int64_t c = threadIdx.x; c < cols; c += kNormBlock) {
            float v = (static_cast<float>(xr[c]) - mu) * rs;
            v = fmaf(v, weight ? static_cast<float>(weight[c]) : 1.f, bias ? static_cast<float>(bias[c]) : 0.f);
            yr[c] = static_cast<T>(v);
        }
        if (mean && threadIdx.x == 0) {
            mean[row] = mu;
            rstd[row] = rs;
        }
    }
}

template <typename T, typename W>
__global__ void __launch_bounds__(kNormBlock)
k_norm_grad_any(const T* dy, int64_t dy_stride, const T* x, int64_t x_stride, int64_t rows, int64_t cols, const W* weight,
                const float* mean, const float* rstd, T* dx, int64_t dx_stride) {
    __shared__ float lds[2][2][16];
    int turn = 0;
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const T *xr = x + row * x_stride, *dr = dy + row * dy_stride;
        const float mu = mean[row], rs = rstd[row];
        float s[2] = {0.f, 0.f};
        for (int64_t c = threadIdx.x; c < cols; c += kNormBlock) {
            const float a = static_cast<float>(dr[c]) * (weight ? static_cast<float>(weight[c]) : 1.f);
            s[0] += a;
            s[1] = fmaf(a, (static_cast<float>(xr[c]) - mu) * rs, s[1]);
        }
        block_sums<kNormBlock>(s, lds, turn);
        const float m1 = s[0] / static_cast<float>(cols), m2 = s[1] / static_cast<float>(cols);
        T* out = dx + row * dx_stride;
        for (int64_t c = threadIdx.x; c < cols; c += kNormBlock) {
            const float a = static_cast<float>(dr[c]) * (weight ? static_cast<float>(weight[c]) : 1.f);
            const float xh = (static_cast<float>(xr[c]) - mu) * rs;
            out[c] = static_cast<T>(rs * (a - m1 - xh * m2));
        }
    }
}

// partials[g][0][c] = sum dy xh, partials[g][1][c] = sum dy over the rows of share g (blockIdx.y): 64 columns a
// workgroup, four rows at a time
template <typename T>
__global__ void __launch_bounds__(kNormBlock)
k_norm_columns_any(const T* dy, int64_t dy_stride, const T* x, int64_t x_stride, int64_t rows, int64_t cols,
                   const float* mean, const float* rstd, float* partials) {
    __shared__ float lds[2][4][64];
    const int lane = threadIdx.x & 63, part = threadIdx.x >> 6;
    for (int64_t begin = static_cast<int64_t>(blockIdx.x) * 64; begin < cols; begin += static_cast<int64_t>(gridDim.x) * 64) {
        const int64_t c = begin + lane;
        float dw = 0.f, db = 0.f;
        if (c < cols)
            for (int64_t row = static_cast<int64_t>(blockIdx.y) * 4 + part; row < rows; row += static_cast<int64_t>(gridDim.y) * 4) {
                const float d = static_cast<float>(dy[row * dy_stride + c]);
                dw = fmaf(d, (static_cast<float>(x[row * x_stride + c]) - mean[row]) * rstd[row], dw);
                db += d;
            }
        lds[0][part][lane] = dw;
        lds[1][part][lane] = db;
        __syncthreads();
        if (part < 2 && c < cols)
            partials[(static_cast<int64_t>(blockIdx.y) * 2 + part) * cols + c] =
                (lds[part][0][lane] + lds[part][1][lane]) + (lds[part][2][lane] + lds[part][3][lane]);
        __syncthreads();
    }
}

// dweight and dbias from the shares' partial sums, in a fixed order: 16 columns a workgroup (64 contiguous bytes of every share), 64
// shares at a time, four requests a thread under way.  512 shares: of 4096 columns 7.0 us (16.8 MB of sums, 32.8 as counted), of 512 3.2 (latency); with
// 16 shares at a time and one request 20.
constexpr int kWeightsBlock = 1024;
template <typename W>
__global__ void __launch_bounds__(kWeightsBlock)
k_norm_weights(const float* partials, int shares, int64_t cols, W* dweight, W* dbias) {
    __shared__ float lds[kWeightsBlock / 64][16];
    W* out = blockIdx.y ? dbias : dweight;
    if (!out) return;
    const int at = threadIdx.x & 15, part = threadIdx.x >> 4;
    for (int64_t begin = static_cast<int64_t>(blockIdx.x) * 16; begin < cols; begin += static_cast<int64_t>(gridDim.x) * 16) {
        const int64_t c = begin + at;
        float s = 0.f;
        if (c < cols) {
            const float* p = partials + static_cast<int64_t>(blockIdx.y) * cols + c;
            int g = part;
            for (; g + 3 * 64 < shares; g += 4 * 64) {
                float v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = p[static_cast<int64_t>(g + 64 * k) * 2 * cols];
                s += (v[0] + v[1]) + (v[2] + v[3]);
            }
            for (; g < shares; g += 64) s += p[static_cast<int64_t>(g) * 2 * cols];
        }
        // a wavefront's four parts, then the wavefronts'
        s += __shfl_xor(s, 16);
        s += __shfl_xor(s, 32);
        if ((threadIdx.x & 63) < 16) lds[threadIdx.x >> 6][at] = s;
        __syncthreads();
        if (part == 0 && c < cols) {
            s = 0.f;
#pragma unroll
            for (int k = 0; k < kWeightsBlock / 64; ++k) s += lds[k][at];
            out[c] = static_cast<W>(s);
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------------------
// Rows in registers, 16-byte packs: TPR threads hold a row, ITEMS packs each (thread t packs t, t + TPR, ...).
// ---------------------------------------------------------------------------------------
// A thread's columns.  A row that ends inside a pack has its last pack moved back to end with the row: the columns that it then
// shares with the pack before are masked in sums (first: values of the last pack before it are another thread's) and written
// twice with the same value.
template <typename T, int TPR, int ITEMS>
struct Slots {
    static constexpr int P = kPack<T>;
    int last, first;                     // column of the last pack; its values from `first` on are this thread's (P: none)
    int t;
    __device__ __forceinline__ Slots(int thread, int cols) : t(thread) {
        const int at = (thread + TPR * (ITEMS - 1)) * P;
        last = min(at, cols - P);
        first = at < cols ? at - last : P;
    }
    __device__ __forceinline__ bool has(int i) const { return i < ITEMS - 1 || first < P; }
    __device__ __forceinline__ int at(int i) const { return i < ITEMS - 1 ? (t + TPR * i) * P : last; }
    __device__ __forceinline__ bool own(int i, int e) const { return i < ITEMS - 1 || e >= first; }
};

template <int TPR>
constexpr int threads_of() { return TPR < kNormBlock ? kNormBlock : TPR; }

// Mean, then the squares around it, both from registers: one read and one write of a row, a row more on its way meanwhile (a second
// one changed nothing).  A quarter of a wavefront, a wavefront, or a workgroup a row, so that short rows need no barrier and no
// lane is idle.  Bound by memory: 32768 x 4096 bf16 in 116 us, 537 MB at 4.6 TB/s (a copy: 4.8), vector ALU 66 % busy (two reductions a
// row are a third of that); 8192 x 512 f32 8.0 us, 4.2 TB/s.
template <typename T, typename W, int TPR, int ITEMS, bool PAST>
__global__ void __launch_bounds__(threads_of<TPR>())
k_norm(const T* x, int64_t x_stride, int64_t rows, int cols, const W* weight, const W* bias, float eps, T* y,
       int64_t y_stride, float* mean, float* rstd) {
    constexpr int P = kPack<T>, ROWS = threads_of<TPR>() / TPR;
    __shared__ float lds[2][1][16];
    int turn = 0;
    const int t = threadIdx.x % TPR;
    const Slots<T, TPR, ITEMS> slot(t, cols);
    const float per = 1.0f / static_cast<float>(cols);
    const int64_t step = static_cast<int64_t>(gridDim.x) * ROWS;
    int64_t row = static_cast<int64_t>(blockIdx.x) * ROWS + threadIdx.x / TPR;
    Raw<T, P> next[ITEMS];
    const auto request = [&](int64_t r) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
            if (slot.has(i)) next[i].load(x + r * x_stride + slot.at(i));
    };
    if (row < rows) request(row);
    for (; row < rows; row += step) {
        float v[ITEMS][P];
        float s[1] = {0.f};
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
#pragma unroll
            for (int e = 0; e < P; ++e) {
                v[i][e] = next[i][e];
                s[0] += slot.own(i, e) ? v[i][e] : 0.f;
            }
        if (row + step < rows) request(row + step);          // under way while this row is worked on
        block_sums<TPR>(s, lds, turn);
        const float mu = s[0] * per;
        float q[1] = {0.f};
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
#pragma unroll
            for (int e = 0; e < P; ++e) {
                v[i][e] -= mu;
                const float d = slot.own(i, e) ? v[i][e] : 0.f;
                q[0] = fmaf(d, d, q[0]);
            }
        block_sums<TPR>(q, lds, turn);
        const float rs = 1.0f / sqrtf(fmaf(q[0], per, eps));
        T* yr = y + row * y_stride;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            if (!slot.has(i)) continue;
            float w[P], b[P];
            if (weight) load_pack<W, P>(weight + slot.at(i), w);
            if (bias) load_pack<W, P>(bias + slot.at(i), b);
#pragma unroll
            for (int e = 0; e < P; ++e) v[i][e] = fmaf(v[i][e] * rs, weight ? w[e] : 1.f, bias ? b[e] : 0.f);
            store_pack<PAST>(yr + slot.at(i), v[i]);
        }
        if (mean && t == 0) {
            mean[row] = mu;
            rstd[row] = rs;
        }
    }
}

// Each group of TPR threads of a workgroup takes rows of its own and keeps the sums of its columns' gradients in registers
// until its last row: x and dy are read once, and what the sums cost is 512 shares of two rows each.  One pack a thread where
// there are threads for it: two sums and two inputs a value are what fills the registers (bf16: 107 with one pack, 155 with two, with
// which 32768 x 4096 took 207 us in place of 193).  Workgroups of 512 threads, as several rows' sums are joined in LDS
// before they leave: half as many shares as with 256 (3001 x 1999 f16 20.6 / 14.0 us).
// Bound by memory: 32768 x 4096 bf16 in 173 us, 805 MB at 4.65 TB/s; 8192 x 512 f32 12 us, 50 MB.
constexpr int kGradBlock = 512;
template <int TPR>
constexpr int grad_threads() { return TPR < kGradBlock ? kGradBlock : TPR; }
// Gradients of weight and bias of 8 packs of columns, by a workgroup for itself: eight threads side by side in a row, the rows in
// turn, four under way.
template <typename T, typename W, int THREADS>
__device__ __forceinline__ void norm_columns(int part, const T* dy, int64_t dy_stride, const T* x, int64_t x_stride, int64_t rows, int cols,
                                             const float* mean, const float* rstd, W* dweight, W* dbias) {
    constexpr int P = kPack<T>, RT = THREADS / 8, N = 4;
    __shared__ float sums[THREADS / 64][8][2 * P];
    const int c = threadIdx.x & 7, first_row = threadIdx.x >> 3;
    const int begin = (part * 8 + c) * P, at = min(begin, cols - P);
    float dw[P] = {}, db[P] = {};
    if (begin < cols)
        for (int64_t row = first_row; row < rows; row += N * RT) {
            Raw<T, P> rx[N], rd[N];
            float mu[N], rs[N];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const int64_t r = min(row + j * RT, rows - 1);
                rx[j].load(x + r * x_stride + at);
                rd[j].load(dy + r * dy_stride + at);
                mu[j] = mean[r], rs[j] = rstd[r];
            }
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (row + j * RT < rows)
#pragma unroll
                    for (int e = 0; e < P; ++e) {
                        dw[e] = fmaf(rd[j][e], (rx[j][e] - mu[j]) * rs[j], dw[e]);
                        db[e] += rd[j][e];
                    }
        }
#pragma unroll
    for (int e = 0; e < P; ++e) {
#pragma unroll
        for (int d = 8; d < 64; d <<= 1) {
            dw[e] += __shfl_xor(dw[e], d);
            db[e] += __shfl_xor(db[e], d);
        }
        if ((threadIdx.x & 63) < 8) {
            sums[threadIdx.x >> 6][c][e] = dw[e];
            sums[threadIdx.x >> 6][c][P + e] = db[e];
        }
    }
    __syncthreads();
    if (threadIdx.x < 8 * 2 * P) {
        const int pack = threadIdx.x / (2 * P), e = threadIdx.x % (2 * P), from = (part * 8 + pack) * P, to = min(from, cols - P);
        W* out = e < P ? dweight : dbias;
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) s += sums[w][pack][e];
        if (out && from < cols && e % P >= from - to) out[to + e % P] = static_cast<W>(s);
    }
}

// How the weights' gradients are taken: not at all; as partial sums, added up by k_norm_weights; or, of few rows, by
// workgroups of the same launch behind the `row_blocks` that take rows.
enum { kNoSums, kPartialSums, kOwnSums };
template <typename T, typename W, int TPR, int ITEMS, int SUMS, bool PAST>
__global__ void __launch_bounds__(grad_threads<TPR>())
k_norm_grad(const T* dy, int64_t dy_stride, const T* x, int64_t x_stride, int64_t rows, int cols, const W* weight,
            const float* mean, const float* rstd, T* dx, int64_t dx_stride, float* partials, int row_blocks, W* dweight, W* dbias) {
    constexpr int P = kPack<T>, ROWS = grad_threads<TPR>() / TPR;
    if constexpr (SUMS == kOwnSums)
        if (static_cast<int>(blockIdx.x) >= row_blocks) {
            norm_columns<T, W, grad_threads<TPR>()>(blockIdx.x - row_blocks, dy, dy_stride, x, x_stride, rows, cols, mean, rstd, dweight,
                                                    dbias);
            return;
        }
    __shared__ float lds[2][2][16];
    int turn = 0;
    const int t = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const Slots<T, TPR, ITEMS> slot(t, cols);
    const float per = 1.0f / static_cast<float>(cols);
    float dw[ITEMS][P] = {}, db[ITEMS][P] = {};
    const int64_t step = static_cast<int64_t>(row_blocks) * ROWS;
    int64_t first = static_cast<int64_t>(blockIdx.x) * ROWS;         // of the workgroup's rows
    Raw<T, P> next_x[ITEMS], next_dy[ITEMS];
    if (ROWS > 1)
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) next_x[i] = next_dy[i] = Raw<T, P>{};
    float next_mu = 0.f, next_rs = 0.f;
    // (a group without a row left reads none: where dx is x or dy, another group may be writing it)
    const auto request = [&](int64_t r) {
        next_mu = mean[r], next_rs = rstd[r];
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
            if (slot.has(i)) {
                next_x[i].load(x + r * x_stride + slot.at(i));
                next_dy[i].load(dy + r * dy_stride + slot.at(i));
            }
    };
    if (first + group < rows) request(first + group);
    for (; first < rows; first += step) {
        const int64_t row = first + group;
        const bool has_row = ROWS == 1 || row < rows;
        float v[ITEMS][P], a[ITEMS][P];
        // (without a row: what x was before, or 0, times 0, and dy 0)
        const float mu = has_row ? next_mu : 0.f, rs = has_row ? next_rs : 0.f;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
#pragma unroll
            for (int e = 0; e < P; ++e) v[i][e] = next_x[i][e], a[i][e] = has_row ? next_dy[i][e] : 0.f;
        if (row + step < rows) request(row + step);              // under way while this row is worked on
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            float w[P];
            if (weight && slot.has(i)) load_pack<W, P>(weight + slot.at(i), w);
#pragma unroll
            for (int e = 0; e < P; ++e) {
                const float xh = slot.own(i, e) ? (v[i][e] - mu) * rs : 0.f, d = slot.own(i, e) ? a[i][e] : 0.f;
                if (SUMS == kPartialSums) {
                    dw[i][e] = fmaf(d, xh, dw[i][e]);
                    db[i][e] += d;
                }
                const float h = weight ? d * w[e] : d;
                s[0] += slot.own(i, e) ? h : 0.f;
                s[1] = fmaf(slot.own(i, e) ? h : 0.f, xh, s[1]);
            }
        }
        if (!dx) continue;
        block_sums<TPR>(s, lds, turn);
        const float m1 = s[0] * per, m2 = s[1] * per;
        if (!has_row) continue;
        T* out = dx + row * dx_stride;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
            if (!slot.has(i)) continue;
            float w[P];
            if (weight) load_pack<W, P>(weight + slot.at(i), w);
#pragma unroll
            for (int e = 0; e < P; ++e) {
                const float h = weight ? a[i][e] * w[e] : a[i][e], xh = (v[i][e] - mu) * rs;
                a[i][e] = rs * (h - m1 - xh * m2);
            }
            store_pack<PAST>(out + slot.at(i), a[i]);
        }
    }
    if (SUMS != kPartialSums) return;
    float* mine = partials + static_cast<int64_t>(blockIdx.x) * 2 * cols;
    if (ROWS == 1) {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
#pragma unroll
            for (int e = 0; e < P; ++e)
                if (slot.own(i, e)) {
                    mine[slot.at(i) + e] = dw[i][e];
                    mine[cols + slot.at(i) + e] = db[i][e];
                }
    } else {
        // the groups' sums, one after the other (those of a wavefront, if it has several, by exchanges before)
        constexpr int PER = TPR < 64 ? 64 : TPR;
        __shared__ float sums[ROWS == 1 ? 1 : 2][ROWS == 1 ? 1 : TPR * ITEMS * P];
        if (TPR < 64)
#pragma unroll
            for (int i = 0; i < ITEMS; ++i)
#pragma unroll
                for (int e = 0; e < P; ++e)
#pragma unroll
                    for (int d = TPR; d < 64; d <<= 1) {
                        dw[i][e] += __shfl_xor(dw[i][e], d);
                        db[i][e] += __shfl_xor(db[i][e], d);
                    }
        for (int w = 0; w < grad_threads<TPR>() / PER; ++w) {
            if (static_cast<int>(threadIdx.x) / PER == w && threadIdx.x % PER < TPR) {
#pragma unroll
                for (int i = 0; i < ITEMS; ++i)
#pragma unroll
                    for (int e = 0; e < P; ++e)
                        if (slot.own(i, e)) {
                            const int c = slot.at(i) + e;
                            sums[0][c] = w ? sums[0][c] + dw[i][e] : dw[i][e];
                            sums[1][c] = w ? sums[1][c] + db[i][e] : db[i][e];
                        }
            }
            __syncthreads();
        }
        for (int c = threadIdx.x; c < cols; c += grad_threads<TPR>()) {
            mine[c] = sums[0][c];
            mine[cols + c] = sums[1][c];
        }
    }
}

// ---------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------
struct NormArgs {
    const void *x, *dy, *weight, *bias;
    int64_t rows, cols, x_stride, dy_stride, out_stride;
    float eps;
    void* out;                       // y or dx
    float *mean, *rstd;
    void *dweight, *dbias;
    float* partials;
    hipStream_t stream;
};

// How rows of `cols` values are held: threads a row and packs a thread, or threads = 0 (a value at a time).
struct Held {
    int threads, items;
};
Held held(int64_t cols, int32_t fmt) {
    const int64_t p = 16 / fmt_bytes(fmt), packs = (cols + p - 1) / p;
    if (cols < p) return {0, 0};
    if (packs <= 16) return {16, 1};
    // (us, rows that 256 threads would hold with 2 to 4 packs each / 512 with half as many: 65536 x 1500 f32 160 / 148, 32768 x 4096
    // bf16 117 / 115; but rows of up to 4 packs by a wavefront, not by more threads: 20000 x 1500 bf16 28 / 31)
    for (const int threads : {64, 512, 1024}) {
        const int64_t items = (packs + threads - 1) / threads;
        if (items <= 4) return {threads, static_cast<int>(items)};
    }
    return {0, 0};
}
// The same for the backward pass, which keeps two sums a column besides: as few packs a thread as there are threads for.
Held held_grad(int64_t cols, int32_t fmt) {
    const int64_t p = 16 / fmt_bytes(fmt), packs = (cols + p - 1) / p;
    if (cols < p) return {0, 0};
    if (packs <= 16) return {16, 1};
    for (const int threads : {64, 128, 256, 512, 1024}) {
        const int64_t items = (packs + threads - 1) / threads;
        // (1024 threads have 128 registers each: enough for four packs of four values, not for two of eight)
        if (threads == 1024 && p > 4) break;
        if (items <= (threads >= 512 ? 4 : 1)) return {threads, static_cast<int>(items)};
    }
    return {0, 0};
}

// Workgroups of `threads` threads for columns, `each` at a time, which they take in turns: a launch has fewer than 2^32 threads in a
// dimension, and rows up to 2^30 columns.
unsigned column_grid(int64_t cols, int each, int threads) {
    const int64_t n = (cols + each - 1) / each, most = (static_cast<int64_t>(1) << 32) / threads - 1;
    return static_cast<unsigned>(n < most ? n : most);
}
unsigned norm_grid(int64_t rows) { return static_cast<unsigned>(rows < 4096 ? rows : 4096); }
// workgroups of the backward pass over rows that are held in registers; each leaves partial sums of the weights' gradients
int grad_grid(int64_t rows, const Held& h, int32_t fmt) {
    const int64_t groups = h.threads < kGradBlock ? kGradBlock / h.threads : 1, n = (rows + groups - 1) / groups, most = h.items * (16 / fmt_bytes(fmt)) <= 8 ? 512 : 256;
    return static_cast<int>(n < most ? n : most);
}
// shares of the rows whose partial sums of the weights' gradients are added up at the end
int norm_shares(int64_t rows, int64_t cols, int32_t fmt) {
    const Held h = held_grad(cols, fmt);
    if (h.threads) return grad_grid(rows, h, fmt);
    const int64_t blocks = (cols + 63) / 64;
    int64_t want = blocks >= 1024 ? 1 : (1024 + blocks - 1) / blocks;
    if (want > (rows + 15) / 16) want = (rows + 15) / 16;
    return static_cast<int>(want < 1 ? 1 : want);
}

template <typename T, typename W, int TPR, int ITEMS>
int norm_forward_held(const NormArgs& a) {
    const int64_t each = threads_of<TPR>() / TPR, groups = (a.rows + each - 1) / each;
    const unsigned grid = static_cast<unsigned>(groups < 4096 ? groups : 4096);
    const auto kernel = past_caches(a.rows * a.cols * sizeof(T)) ? k_norm<T, W, TPR, ITEMS, true> : k_norm<T, W, TPR, ITEMS, false>;
    kernel<<<grid, threads_of<TPR>(), 0, a.stream>>>(
        static_cast<const T*>(a.x), a.x_stride, a.rows, static_cast<int>(a.cols), static_cast<const W*>(a.weight),
        static_cast<const W*>(a.bias), a.eps, static_cast<T*>(a.out), a.out_stride, a.mean, a.rstd);
    return launched();
}
// Few rows, or up to 2048 wide ones: the weights' gradients by workgroups of their own (the rows are read twice, the second time
// from the caches), in the same launch where dx is not written over what they read.  Rows of more than 8192 values in 32 bits
// always: 1024 threads have no registers for sums beside them.  (us a pass, own workgroups / partial sums: 1000 x 1024 bf16
// 18 / 22, 1500 x 1024 bf16 26 / 21, 1500 x 4096 bf16 27 / 33, 3000 x 8192 f32 125 / 110, 6000 x 16000 f32 509 / 641.)
bool own_sums(const NormArgs& a, const Held& h) {
    return (a.dweight || a.dbias) && (h.threads == 1024 || a.rows <= (h.threads == 512 ? 2048 : 1024));
}
template <typename T, typename W, int TPR, int ITEMS>
int norm_grad_held(const NormArgs& a, const Held& h, int shares) {
    const bool past = past_caches(a.rows * a.cols * sizeof(T));
    const auto launch = [&](auto kernel, int row_blocks, int64_t more) {
        kernel<<<static_cast<unsigned>(row_blocks + more), grad_threads<TPR>(), 0, a.stream>>>(
            static_cast<const T*>(a.dy), a.dy_stride, static_cast<const T*>(a.x), a.x_stride, a.rows, static_cast<int>(a.cols),
            static_cast<const W*>(a.weight), a.mean, a.rstd, static_cast<T*>(a.out), a.out_stride, a.partials, row_blocks,
            static_cast<W*>(a.dweight), static_cast<W*>(a.dbias));
        return launched();
    };
    if (own_sums(a, h)) {
        const int64_t columns = (a.cols + 8 * kPack<T> - 1) / (8 * kPack<T>);
        const bool apart = a.out != a.dy && a.out != a.x;
        if (int rc = launch(past ? k_norm_grad<T, W, TPR, ITEMS, kOwnSums, TPR == 1024> : k_norm_grad<T, W, TPR, ITEMS, kOwnSums, false>,
                            a.out && apart ? shares : 0, columns))
            return rc;
        if (!a.out || apart) return CS_OK;
    } else if constexpr (TPR < 1024) {
        if (a.dweight || a.dbias)
            return launch(past ? k_norm_grad<T, W, TPR, ITEMS, kPartialSums, true> : k_norm_grad<T, W, TPR, ITEMS, kPartialSums, false>,
                          shares, 0);
    }
    return launch(past ? k_norm_grad<T, W, TPR, ITEMS, kNoSums, true> : k_norm_grad<T, W, TPR, ITEMS, kNoSums, false>, shares, 0);
}
#define CS_HELD(h, CALL)                                                                               \
    switch ((h).threads * 8 + (h).items) {                                                             \
        case 16 * 8 + 1: return CALL(16, 1);                                                           \
        case 64 * 8 + 1: return CALL(64, 1);                                                           \
        case 64 * 8 + 2: return CALL(64, 2);                                                           \
        case 64 * 8 + 3: return CALL(64, 3);                                                           \
        case 64 * 8 + 4: return CALL(64, 4);                                                           \
        case 512 * 8 + 1: return CALL(512, 1);                                                         \
        case 512 * 8 + 2: return CALL(512, 2);                                                         \
        case 512 * 8 + 3: return CALL(512, 3);                                                         \
        case 512 * 8 + 4: return CALL(512, 4);                                                         \
        case 1024 * 8 + 3: return CALL(1024, 3);                                                       \
        case 1024 * 8 + 4: return CALL(1024, 4);                                                       \
        default: return CS_EINVAL;                                                                     \
    }
#define CS_HELD_GRAD(h, CALL)                                                                          \
    switch ((h).threads * 8 + (h).items) {                                                             \
        case 16 * 8 + 1: return CALL(16, 1);                                                           \
        case 64 * 8 + 1: return CALL(64, 1);                                                           \
        case 128 * 8 + 1: return CALL(128, 1);                                                         \
        case 256 * 8 + 1: return CALL(256, 1);                                                         \
        case 512 * 8 + 1: return CALL(512, 1);                                                         \
        case 512 * 8 + 2: return CALL(512, 2);                                                         \
        case 512 * 8 + 3: return CALL(512, 3);                                                         \
        case 512 * 8 + 4: return CALL(512, 4);                                                         \
        default: return CS_EINVAL;                                                                     \
    }

template <typename T, typename W>
int norm_forward(const NormArgs& a) {
    const Held h = held(a.cols, std::is_same<T, float>::value ? CS_FMT_F32 : CS_FMT_BF16);
    if (h.threads) {
#define CS_CALL(TPR, ITEMS) (norm_forward_held<T, W, TPR, ITEMS>(a))
        CS_HELD(h, CS_CALL)
#undef CS_CALL
    }
    k_norm_any<T, W><<<norm_grid(a.rows), kNormBlock, 0, a.stream>>>(
        static_cast<const T*>(a.x), a.x_stride, a.rows, a.cols, static_cast<const W*>(a.weight),
        static_cast<const W*>(a.bias), a.eps, static_cast<T*>(a.out), a.out_stride, a.mean, a.rstd);
    return launched();
}

// dx and the shares' partial sums
template <typename T, typename W>
int norm_grad(const NormArgs& a, int shares) {
    const T *dy = static_cast<const T*>(a.dy), *x = static_cast<const T*>(a.x);
    const Held h = held_grad(a.cols, std::is_same<T, float>::value ? CS_FMT_F32 : CS_FMT_BF16);
    if (h.threads) {
#define CS_CALL(TPR, ITEMS) (norm_grad_held<T, W, TPR, ITEMS>(a, h, shares))
        if constexpr (sizeof(T) == 4)
            if (h.threads == 1024) return h.items == 3 ? CS_CALL(1024, 3) : CS_CALL(1024, 4);
        CS_HELD_GRAD(h, CS_CALL)
#undef CS_CALL
    }
    if (a.dweight || a.dbias) {
        const dim3 grid(column_grid(a.cols, 64, kNormBlock), shares);
        k_norm_columns_any<T><<<grid, kNormBlock, 0, a.stream>>>(dy, a.dy_stride, x, a.x_stride, a.rows, a.cols, a.mean,
                                                                 a.rstd, a.partials);
        if (int rc = launched()) return rc;
    }
    if (!a.out) return CS_OK;
    k_norm_grad_any<T, W><<<norm_grid(a.rows), kNormBlock, 0, a.stream>>>(
        dy, a.dy_stride, x, a.x_stride, a.rows, a.cols, static_cast<const W*>(a.weight), a.mean, a.rstd,
        static_cast<T*>(a.out), a.out_stride);
    return launched();
}

template <typename T, typename W>
int norm_backward(const NormArgs& a) {
    const int shares = a.rows ? norm_shares(a.rows, a.cols, std::is_same<T, float>::value ? CS_FMT_F32 : CS_FMT_BF16) : 0;
    if (a.rows)
        if (int rc = norm_grad<T, W>(a, shares)) return rc;
    if (!a.dweight && !a.dbias) return CS_OK;
    const Held h = held_grad(a.cols, std::is_same<T, float>::value ? CS_FMT_F32 : CS_FMT_BF16);
    if (a.rows && h.threads && own_sums(a, h)) return CS_OK;
    const dim3 grid(column_grid(a.cols, 16, kWeightsBlock), 2);
    k_norm_weights<W><<<grid, kWeightsBlock, 0, a.stream>>>(a.partials, shares, a.cols, static_cast<W*>(a.dweight),
                                                         static_cast<W*>(a.dbias));
    return launched();
}

// weights in 32 bits, or in the rows' type
template <template <typename, typename> class F>
int by_type(int32_t fmt, int32_t w_fmt, const NormArgs& a) {
    if (fmt == CS_FMT_F32) return F<float, float>::call(a);
    if (fmt == CS_FMT_BF16) return w_fmt == CS_FMT_F32 ? F<bf16, float>::call(a) : F<bf16, bf16>::call(a);
    return w_fmt == CS_FMT_F32 ? F<f16, float>::call(a) : F<f16, f16>::call(a);
}
template <typename T, typename W>
struct Forward {
    static int call(const NormArgs& a) { return norm_forward<T, W>(a); }
};
template <typename T, typename W>
struct Backward {
    static int call(const NormArgs& a) { return norm_backward<T, W>(a); }
};

constexpr int64_t kNormMaxCols = static_cast<int64_t>(1) << 30;

// out may be `in` itself, value for value, and must not meet it otherwise
bool apart_or_same(const void* out, int64_t out_stride, const void* in, int64_t in_stride, int64_t rows, int64_t cols, int32_t fmt) {
    if (out == in && (out_stride == in_stride || rows == 1)) return true;
    const int64_t b = fmt_bytes(fmt);
    return !rows_meet(out, out_stride * b, in, in_stride * b, rows, cols * b);
}
bool span_in_rows(const void* span, int64_t bytes, const void* rows_at, int64_t stride, int64_t rows, int64_t cols, int32_t fmt) {
    return rows > 0 && spans_meet(span, bytes, rows_at, ((rows - 1) * stride + cols) * fmt_bytes(fmt));
}

}  // namespace
}  // namespace cs

using namespace cs;

extern "C" int cs_layer_norm(const void* x, int64_t rows, int64_t cols, int64_t x_stride, int32_t fmt, const void* weight,
                             const void* bias, int32_t w_fmt, float eps, void* y, int64_t y_stride, float* mean,
                             float* rstd, void* stream) {
    if (!rows_ok(rows, cols, x_stride, fmt) || !rows_ok(rows, cols, y_stride, fmt) || cols > kNormMaxCols) return CS_EINVAL;
    if ((w_fmt != fmt && w_fmt != CS_FMT_F32) || !(eps >= 0.f) || (mean == nullptr) != (rstd == nullptr)) return CS_EINVAL;
    if (rows == 0) return CS_OK;
    if (!x || !y || !apart_or_same(y, y_stride, x, x_stride, rows, cols, fmt)) return CS_EINVAL;
    for (const void* w : {weight, bias})
        if (w && span_in_rows(w, cols * fmt_bytes(w_fmt), y, y_stride, rows, cols, fmt)) return CS_EINVAL;
    for (const void* s : {static_cast<const void*>(mean), static_cast<const void*>(rstd)})
        if (s && (span_in_rows(s, 4 * rows, y, y_stride, rows, cols, fmt) ||
                  span_in_rows(s, 4 * rows, x, x_stride, rows, cols, fmt) ||
                  spans_meet(s, 4 * rows, weight, cols * fmt_bytes(w_fmt)) || spans_meet(s, 4 * rows, bias, cols * fmt_bytes(w_fmt))))
            return CS_EINVAL;
    if (spans_meet(mean, 4 * rows, rstd, 4 * rows)) return CS_EINVAL;
    NormArgs a = {};
    a.x = x, a.weight = weight, a.bias = bias, a.rows = rows, a.cols = cols, a.x_stride = x_stride;
    a.eps = eps, a.out = y, a.out_stride = y_stride, a.mean = mean, a.rstd = rstd, a.stream = stream_of(stream);
    return by_type<Forward>(fmt, w_fmt, a);
}

extern "C" int cs_layer_norm_grad_workspace_bytes(int64_t rows, int64_t cols, size_t* bytes) {
    if (rows < 0 || cols < 1 || cols > kNormMaxCols || !bytes) return CS_EINVAL;
    // (of either width of the rows' type)
    const int a = norm_shares(rows, cols, CS_FMT_F32), b = norm_shares(rows, cols, CS_FMT_BF16);
    *bytes = static_cast<size_t>(a > b ? a : b) * 2 * cols * sizeof(float);
    return CS_OK;
}

extern "C" int cs_layer_norm_grad(const void* dy, int64_t dy_stride, const void* x, int64_t x_stride, int64_t rows,
                                  int64_t cols, int32_t fmt, const void* weight, int32_t w_fmt, const float* mean,
                                  const float* rstd, void* dx, int64_t dx_stride, void* dweight, void* dbias,
                                  void* workspace, size_t ws_bytes, void* stream) {
    if (!rows_ok(rows, cols, x_stride, fmt) || !rows_ok(rows, cols, dy_stride, fmt) || cols > kNormMaxCols) return CS_EINVAL;
    if (w_fmt != fmt && w_fmt != CS_FMT_F32) return CS_EINVAL;
    if (dx && !rows_ok(rows, cols, dx_stride, fmt)) return CS_EINVAL;
    if (rows && (!dy || !x || !mean || !rstd)) return CS_EINVAL;
    const int64_t wb = cols * fmt_bytes(w_fmt);
    if (dx && (!apart_or_same(dx, dx_stride, dy, dy_stride, rows, cols, fmt) ||
               !apart_or_same(dx, dx_stride, x, x_stride, rows, cols, fmt)))
        return CS_EINVAL;
    if (spans_meet(dweight, wb, dbias, wb)) return CS_EINVAL;
    size_t need = 0;
    cs_layer_norm_grad_workspace_bytes(rows, cols, &need);
    const bool sums = dweight || dbias;
    if (sums && ws_bytes < need) return CS_EWORKSPACE;
    if (sums && need && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 3))) return CS_EINVAL;
    // what is written must not lie in what is still to be read
    const void* written[] = {dweight, dbias, sums ? workspace : nullptr};
    const int64_t size[] = {wb, wb, static_cast<int64_t>(need)};
    for (int k = 0; k < 3; ++k) {
        if (!written[k]) continue;
        if (span_in_rows(written[k], size[k], dy, dy_stride, rows, cols, fmt) ||
            span_in_rows(written[k], size[k], x, x_stride, rows, cols, fmt) ||
            (dx && span_in_rows(written[k], size[k], dx, dx_stride, rows, cols, fmt)) ||
            spans_meet(written[k], size[k], weight, wb) || spans_meet(written[k], size[k], mean, 4 * rows) ||
            spans_meet(written[k], size[k], rstd, 4 * rows))
            return CS_EINVAL;
        for (int j = 0; j < k; ++j)
            if (spans_meet(written[k], size[k], written[j], size[j])) return CS_EINVAL;
    }
    if (dx && (span_in_rows(weight, weight ? wb : 0, dx, dx_stride, rows, cols, fmt) ||
               span_in_rows(mean, 4 * rows, dx, dx_stride, rows, cols, fmt) ||
               span_in_rows(rstd, 4 * rows, dx, dx_stride, rows, cols, fmt)))
        return CS_EINVAL;
    if (!dx && !sums) return CS_OK;
    NormArgs a = {};
    a.x = x, a.dy = dy, a.weight = weight, a.rows = rows, a.cols = cols, a.x_stride = x_stride, a.dy_stride = dy_stride;
    a.out = dx, a.out_stride = dx_stride, a.mean = const_cast<float*>(mean), a.rstd = const_cast<float*>(rstd);
    a.dweight = dweight, a.dbias = dbias, a.partials = static_cast<float*>(workspace), a.stream = stream_of(stream);
    return by_type<Backward>(fmt, w_fmt, a);
}

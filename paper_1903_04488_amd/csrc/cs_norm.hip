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
// Rows of any length, a value at a time: the forms for what the packed kernels below do not take.
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
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 64 + lane;
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
}

// dweight and dbias from the shares' partial sums, in a fixed order: 16 columns a workgroup, 16 shares at a time
template <typename W>
__global__ void __launch_bounds__(kNormBlock)
k_norm_weights(const float* partials, int shares, int64_t cols, W* dweight, W* dbias) {
    __shared__ float lds[16][17];
    W* out = blockIdx.y ? dbias : dweight;
    if (!out) return;
    const int at = threadIdx.x & 15, part = threadIdx.x >> 4;
    const int64_t c = static_cast<int64_t>(blockIdx.x) * 16 + at;
    float s = 0.f;
    if (c < cols)
        for (int g = part; g < shares; g += 16) s += partials[(static_cast<int64_t>(g) * 2 + blockIdx.y) * cols + c];
    lds[part][at] = s;
    __syncthreads();
    if (part == 0 && c < cols) {
        s = 0.f;
#pragma unroll
        for (int k = 0; k < 16; ++k) s += lds[k][at];
        out[c] = static_cast<W>(s);
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

// shares of the rows whose partial sums of the weights' gradients are added up at the end
int norm_shares(int64_t rows, int64_t cols) {
    const int64_t blocks = (cols + 63) / 64;
    int64_t want = blocks >= 1024 ? 1 : (1024 + blocks - 1) / blocks;
    if (want > (rows + 15) / 16) want = (rows + 15) / 16;
    return static_cast<int>(want < 1 ? 1 : want);
}

unsigned norm_grid(int64_t rows) { return static_cast<unsigned>(rows < 4096 ? rows : 4096); }

template <typename T, typename W>
int norm_forward(const NormArgs& a) {
    k_norm_any<T, W><<<norm_grid(a.rows), kNormBlock, 0, a.stream>>>(
        static_cast<const T*>(a.x), a.x_stride, a.rows, a.cols, static_cast<const W*>(a.weight),
        static_cast<const W*>(a.bias), a.eps, static_cast<T*>(a.out), a.out_stride, a.mean, a.rstd);
    return launched();
}

template <typename T, typename W>
int norm_backward(const NormArgs& a) {
    const T *dy = static_cast<const T*>(a.dy), *x = static_cast<const T*>(a.x);
    if (a.dweight || a.dbias) {
        int shares = 0;
        if (a.rows) {
            shares = norm_shares(a.rows, a.cols);
            const dim3 grid(static_cast<unsigned>((a.cols + 63) / 64), shares);
            k_norm_columns_any<T><<<grid, kNormBlock, 0, a.stream>>>(dy, a.dy_stride, x, a.x_stride, a.rows, a.cols, a.mean,
                                                                     a.rstd, a.partials);
            if (int rc = launched()) return rc;
        }
        const dim3 grid(static_cast<unsigned>((a.cols + 15) / 16), 2);
        k_norm_weights<W><<<grid, kNormBlock, 0, a.stream>>>(a.partials, shares, a.cols, static_cast<W*>(a.dweight),
                                                             static_cast<W*>(a.dbias));
        if (int rc = launched()) return rc;
    }
    if (a.out && a.rows) {
        k_norm_grad_any<T, W><<<norm_grid(a.rows), kNormBlock, 0, a.stream>>>(
            dy, a.dy_stride, x, a.x_stride, a.rows, a.cols, static_cast<const W*>(a.weight), a.mean, a.rstd,
            static_cast<T*>(a.out), a.out_stride);
        return launched();
    }
    return CS_OK;
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
                  span_in_rows(s, 4 * rows, x, x_stride, rows, cols, fmt)))
            return CS_EINVAL;
    if (spans_meet(mean, 4 * rows, rstd, 4 * rows)) return CS_EINVAL;
    NormArgs a = {};
    a.x = x, a.weight = weight, a.bias = bias, a.rows = rows, a.cols = cols, a.x_stride = x_stride;
    a.eps = eps, a.out = y, a.out_stride = y_stride, a.mean = mean, a.rstd = rstd, a.stream = stream_of(stream);
    return by_type<Forward>(fmt, w_fmt, a);
}

extern "C" int cs_layer_norm_grad_workspace_bytes(int64_t rows, int64_t cols, size_t* bytes) {
    if (rows < 0 || cols < 1 || cols > kNormMaxCols || !bytes) return CS_EINVAL;
    *bytes = static_cast<size_t>(norm_shares(rows, cols)) * 2 * cols * sizeof(float);
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
    if (sums && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 3))) return CS_EINVAL;
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
    NormArgs a = {};
    a.x = x, a.dy = dy, a.weight = weight, a.rows = rows, a.cols = cols, a.x_stride = x_stride, a.dy_stride = dy_stride;
    a.out = dx, a.out_stride = dx_stride, a.mean = const_cast<float*>(mean), a.rstd = const_cast<float*>(rstd);
    a.dweight = dweight, a.dbias = dbias, a.partials = static_cast<float*>(workspace), a.stream = stream_of(stream);
    return by_type<Backward>(fmt, w_fmt, a);
}

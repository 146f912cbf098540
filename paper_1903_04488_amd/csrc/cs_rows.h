// What the kernels over rows of a model's tensors share: 16-byte packs of the three floating types, sums and
// maxima over a wavefront or a workgroup, and the checks of row-wise arguments.  gfx950 only.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "csketch.h"

namespace cs {

using bf16 = __bf16;
using f16 = _Float16;

// values of a 16-byte pack
template <typename T>
constexpr int kPack = 16 / static_cast<int>(sizeof(T));

// N values of type T from an address that is aligned to T alone: one 16-byte (or shorter) request, also where a row begins
// off a 16-byte boundary (global memory is read and written at any alignment).
template <typename T, int N>
struct Raw {
    T v[N];
    __device__ __forceinline__ void load(const T* __restrict__ p) { __builtin_memcpy(v, p, sizeof(v)); }
    __device__ __forceinline__ float operator[](int e) const { return static_cast<float>(v[e]); }
};
template <typename T, int N, bool PAST = false>
__device__ __forceinline__ void load_pack(const T* __restrict__ p, float (&v)[N]) {
    typedef uint32_t Words __attribute__((ext_vector_type(N * sizeof(T) / 4), aligned(sizeof(T))));
    Raw<T, N> raw;
    if (PAST) {
        const Words w = __builtin_nontemporal_load(reinterpret_cast<const Words*>(p));
        __builtin_memcpy(raw.v, &w, sizeof(raw.v));
    } else {
        raw.load(p);
    }
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = raw[e];
}
// rounded to nearest, ties to even, once.  PAST: written past the caches
template <bool PAST, typename T, int N>
__device__ __forceinline__ void store_pack(T* __restrict__ p, const float (&v)[N]) {
    typedef uint32_t Words __attribute__((ext_vector_type(N * sizeof(T) / 4), aligned(sizeof(T))));
    T raw[N];
#pragma unroll
    for (int e = 0; e < N; ++e) raw[e] = static_cast<T>(v[e]);
    Words w;
    __builtin_memcpy(&w, raw, sizeof(raw));
    if (PAST) __builtin_nontemporal_store(w, reinterpret_cast<Words*>(p));
    else *reinterpret_cast<Words*>(p) = w;
}

template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, ROWS, 0xf, false));
}
// the sum of a wavefront's 64 values, the same in every lane: four exchanges within rows of 16 lanes, two broadcasts of a
// row's last lane to the next rows
__device__ __forceinline__ float wave_sum(float v) {
    v += dpp<0xB1, 0xf>(v);      // lanes 1, 0, 3, 2
    v += dpp<0x4E, 0xf>(v);      // lanes 2, 3, 0, 1
    v += dpp<0x141, 0xf>(v);     // half a row mirrored
    v += dpp<0x140, 0xf>(v);     // a row mirrored
    v += dpp<0x142, 0xa>(v);     // into rows 1 and 3
    v += dpp<0x143, 0xc>(v);     // into rows 2 and 3
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp_or_self(float v) {
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(v), __float_as_int(v), CTRL, ROWS, 0xf, false));
}
// (fmaxf: a NaN only where there is nothing else)
__device__ __forceinline__ float wave_max(float v) {
    v = fmaxf(v, dpp_or_self<0xB1, 0xf>(v));
    v = fmaxf(v, dpp_or_self<0x4E, 0xf>(v));
    v = fmaxf(v, dpp_or_self<0x141, 0xf>(v));
    v = fmaxf(v, dpp_or_self<0x140, 0xf>(v));
    v = fmaxf(v, dpp_or_self<0x142, 0xa>(v));
    v = fmaxf(v, dpp_or_self<0x143, 0xc>(v));
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// Sums over groups of THREADS threads of a workgroup, the same in every thread of a group; `turn` counts the calls of a kernel
// (two buffers take turns, so that one barrier a call is enough; every group of the workgroup makes the same calls).
// THREADS = 64 and 16: a wavefront, or a quarter, no barrier.
template <int THREADS, int N>
__device__ __forceinline__ void block_sums(float (&v)[N], float (&lds)[2][N][16], int& turn) {
    static_assert(THREADS == 16 || THREADS % 64 == 0, "");
    if (THREADS == 16) {
#pragma unroll
        for (int k = 0; k < N; ++k) {
            v[k] += dpp<0xB1, 0xf>(v[k]);
            v[k] += dpp<0x4E, 0xf>(v[k]);
            v[k] += dpp<0x141, 0xf>(v[k]);
            v[k] += dpp<0x140, 0xf>(v[k]);
        }
        return;
    }
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = wave_sum(v[k]);
    if (THREADS == 64) return;
    float(&buf)[N][16] = lds[turn & 1];
    ++turn;
    const int wave = threadIdx.x >> 6, first = threadIdx.x / THREADS * (THREADS / 64);
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int k = 0; k < N; ++k) buf[k][wave] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
        float s = 0.f;
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) s += buf[k][first + w];
        v[k] = s;
    }
}

inline bool fmt_ok(int32_t fmt) { return fmt == CS_FMT_BF16 || fmt == CS_FMT_F16 || fmt == CS_FMT_F32; }
inline int64_t fmt_bytes(int32_t fmt) { return fmt == CS_FMT_F32 ? 4 : 2; }

// True when `rows` rows of `bytes` bytes, `step` bytes apart, cannot be told to lie apart from as many rows of another
// array: the spans meet, and they are not two slices of the same wider rows.
inline bool rows_meet(const void* a, int64_t a_step, const void* b, int64_t b_step, int64_t rows, int64_t bytes) {
    if (rows <= 0 || bytes <= 0) return false;
    const uintptr_t pa = reinterpret_cast<uintptr_t>(a), pb = reinterpret_cast<uintptr_t>(b);
    const uintptr_t ea = pa + (rows - 1) * a_step + bytes, eb = pb + (rows - 1) * b_step + bytes;
    if (ea <= pb || eb <= pa) return false;
    if (a_step != b_step || rows == 1) return true;
    const uintptr_t off = (pa < pb ? pb - pa : pa - pb) % static_cast<uintptr_t>(a_step);
    return off < static_cast<uintptr_t>(bytes) || off + bytes > static_cast<uintptr_t>(a_step);
}
inline bool spans_meet(const void* a, int64_t a_bytes, const void* b, int64_t b_bytes) {
    const uintptr_t pa = reinterpret_cast<uintptr_t>(a), pb = reinterpret_cast<uintptr_t>(b);
    return a && b && a_bytes > 0 && b_bytes > 0 && pa < pb + b_bytes && pb < pa + a_bytes;
}
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
// rows x cols values of `fmt` whose rows are `stride` values apart: sizes in range and every address in 63 bits
inline bool rows_ok(int64_t rows, int64_t cols, int64_t stride, int32_t fmt) {
    return rows >= 0 && cols >= 1 && stride >= cols && fmt_ok(fmt) &&
           (rows <= 1 || stride <= (static_cast<int64_t>(1) << 59) / rows);
}

// Outputs that the memory-side cache cannot keep whole are written past the caches: whoever reads them next begins at the
// front, which their end would have pushed out, and what the caches hold of the inputs stays (us a pass: norm 32768 x 4096
// bf16 309 / 296, gradients of 8192 x 34000 bf16 logits 292 / 257, of 4096 x 32001 f32 314 / 285).
inline bool past_caches(int64_t bytes) { return bytes >= (static_cast<int64_t>(256) << 20); }

inline hipStream_t stream_of(void* s) { return reinterpret_cast<hipStream_t>(s); }
inline int launched() { return hipGetLastError() == hipSuccess ? CS_OK : CS_EHIP; }

}  // namespace cs

// AdamW over many tensors in one launch, with moments in 32 or 8 bits, and the gradients' global norm.
//     m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g g,  p = p (1 - lr wd) - lr c1 (m / (sqrt(v) c2 + eps))
//     c1 = 1 / (1 - b1^t),  c2 = 1 / sqrt(1 - b2^t)
// Every product and sum is rounded by itself, in the order above (no fused multiply-add), so that a plain program
// gives the same bits: a moment held in 8 bits then never falls to the other side of a rounding boundary.
//
// Moments in 8 bits: a block of 256 values of a tensor keeps the exponent field ex of its largest magnitude (at least 16), which
// stands for 2^(ex - 127); a code's bits are the top bits of the value's own binary32 pattern, its exponent counted from ex - 15.
// First moment: sign, 4 exponent bits, 3 fraction bits.  Root of the second moment: 4 and 4.  (The
// root, as its square has twice the range; and a root that is not 0 never becomes code 0, as m / eps would be a leap.)
// Rounded to nearest, halves away from 0: half a step is 1/16 of a first moment, 1/32 of a root.  By that alone a moving average stands
// still: a step of decay changes a root by 1 - sqrt(beta2), 1 % at 0.98, which nearest undoes every time (after 5000 steps of gradients of
// one size the roots were 1.9 times too large at 0.98, half as large as they should be at 0.999).  So, with a seed, a change that
// nearest would undo is made with the probability of its share of a step: such a change is right on average.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "cs_rows.h"
#include "csketch.h"

namespace cs {
namespace {

constexpr int kThreads = 256;
constexpr int kBlock8 = CS_ADAMW_BLOCK;              // values that share an exponent
constexpr int kChunk = 4096;                         // values that a workgroup takes
constexpr int kBatch = 56;                           // tensors that one launch writes into a list (4 KB of arguments)

// A list in device memory: this, then Tensor[count], then Chunk[chunks].
struct Tensor {
    void* p;
    const void* g;
    void *m, *v;
    uint8_t *m_exp, *v_exp;
    int64_t n;
    int64_t first_chunk;
};
struct Chunk {
    int32_t tensor, part;
};
struct Batch {
    Tensor t[kBatch];
};
static_assert(sizeof(Batch) < 3800, "kernel arguments are limited to 4 KB");

__global__ void __launch_bounds__(64) k_list_tensors(Batch b, Tensor* out, int count) {
    if (static_cast<int>(threadIdx.x) < count) out[threadIdx.x] = b.t[threadIdx.x];
}
// every chunk's tensor: the last that begins at or before it
__global__ void __launch_bounds__(kThreads) k_list_chunks(const Tensor* tensors, int count, Chunk* out, int64_t chunks) {
    const int64_t c = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    if (c >= chunks) return;
    int lo = 0, hi = count - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (tensors[mid].first_chunk <= c) lo = mid;
        else hi = mid - 1;
    }
    out[c] = Chunk{lo, static_cast<int32_t>(c - tensors[lo].first_chunk)};
}

// ---------------------------------------------------------------------------------------
// 8 bits
// ---------------------------------------------------------------------------------------
__device__ __forceinline__ int32_t bits_of(float x) { return __float_as_int(x); }
__device__ __forceinline__ int32_t base_of(int32_t ex) { return (ex - 15) << 23; }

__device__ __forceinline__ float first_of(uint32_t code, int32_t base) {
    const uint32_t mag = code & 0x7f;
    const float x = __int_as_float(static_cast<int32_t>(mag << 20) + base);
    return mag ? (code & 0x80 ? -x : x) : 0.f;
}
__device__ __forceinline__ float root_of(uint32_t code, int32_t base) {
    return code ? __int_as_float(static_cast<int32_t>(code << 19) + base) : 0.f;
}
// (magnitudes are patterns of at most 31 bits and base is at least 1 << 23: no difference or sum leaves 32 bits)
__device__ __forceinline__ uint32_t code_of_first(float x, int32_t base) {
    const int32_t rel = (bits_of(x) & 0x7fffffff) - base;
    const int32_t c = (rel + (1 << 19)) >> 20;
    return static_cast<uint32_t>(min(max(c, 0), 127)) | (static_cast<uint32_t>(bits_of(x)) >> 24 & 0x80u);
}
__device__ __forceinline__ uint32_t code_of_root(float x, int32_t base) {
    const int32_t mag = bits_of(x) & 0x7fffffff;
    const int32_t c = (mag - base + (1 << 18)) >> 19;
    return mag ? static_cast<uint32_t>(min(max(c, 1), 255)) : 0u;
}
// Codes of a wavefront's four values a lane, which were `old` before, by chance where nearest would undo the change; `ex` becomes the
// block's exponent.  random: 16 bits a value.  A largest value that is rounded up beyond the last code belongs to the next exponent, and 8
// (16) codes less are the same values there.
template <bool FIRST>
__device__ __forceinline__ uint32_t codes_by_chance(const float (&x)[4], const float (&old)[4], const uint32_t (&random)[4], int32_t& ex) {
    constexpr int DROP = FIRST ? 20 : 19, BINADE = FIRST ? 8 : 16, MOST = FIRST ? 127 : 255;
    int32_t c[4];
    bool beyond = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int32_t base = base_of(ex), mag = bits_of(x[e]) & 0x7fffffff, before = bits_of(old[e]) & 0x7fffffff;
        const int32_t half = 1 << (DROP - 1), near = (mag - base + half) >> DROP;
        if (before && (before - base + half) >> DROP == near) {
            c[e] = (mag - base + static_cast<int32_t>(random[e] << (DROP - 16) | 1u << (DROP - 17))) >> DROP;
            beyond |= c[e] > MOST;
        } else {
            c[e] = min(near, MOST);
        }
    }
    if (ex < 254 && __ballot(beyond)) {
        ++ex;
#pragma unroll
        for (int e = 0; e < 4; ++e) c[e] -= BINADE;
    }
    uint32_t codes = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int32_t code = min(max(c[e], FIRST ? 0 : 1), MOST);
        if (FIRST) codes |= (static_cast<uint32_t>(code) | (static_cast<uint32_t>(bits_of(x[e])) >> 24 & 0x80u)) << (8 * e);
        else codes |= (bits_of(x[e]) & 0x7fffffff ? static_cast<uint32_t>(code) : 0u) << (8 * e);
    }
    return codes;
}
__device__ __forceinline__ int32_t wave_max_bits(int32_t v) {
#pragma unroll
    for (int d = 32; d; d >>= 1) v = max(v, __shfl_xor(v, d));
    return v;
}
__device__ __forceinline__ int32_t exponent_of(int32_t most_bits) { return max(most_bits >> 23, 16); }

// ---------------------------------------------------------------------------------------
// the step
// ---------------------------------------------------------------------------------------
struct Coefs {
    float b1, one_b1, b2, one_b2, keep, c2, rate, eps;
    uint32_t chance[2];                               // where the step's random numbers begin, low half first
};
// the n-th output (from 1) of SplitMix64 begun at `state`
__host__ __device__ __forceinline__ uint64_t splitmix(uint64_t state, uint64_t n) {
    uint64_t z = state + n * 0x9E3779B97F4A7C15ull;
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}
// b^t by squaring: products alone, so that the host and the GPU give the same bits
__host__ __device__ __forceinline__ double power(double b, int64_t t) {
#pragma clang fp contract(off)
    double r = 1.;
    for (; t; t >>= 1, b *= b)
        if (t & 1) r *= b;
    return r;
}
__host__ __device__ __forceinline__ Coefs coefs_of(const cs_adamw& h, double lr, int64_t t) {
#pragma clang fp contract(off)
    const double c1 = 1. / (1. - power(h.beta1, t)), c2 = 1. / sqrt(1. - power(h.beta2, t));
    const uint64_t chance = splitmix(h.seed, static_cast<uint64_t>(t));
    return Coefs{static_cast<float>(h.beta1), static_cast<float>(1. - h.beta1), static_cast<float>(h.beta2),
                 static_cast<float>(1. - h.beta2), static_cast<float>(1. - lr * h.weight_decay), static_cast<float>(c2),
                 static_cast<float>(lr * c1), static_cast<float>(h.eps),
                 {static_cast<uint32_t>(chance), static_cast<uint32_t>(chance >> 32)}};
}

struct Moved {
    float p, m, v, root;
};
__device__ __forceinline__ Moved move(float p, float g, float m, float v, const Coefs& c) {
#pragma clang fp contract(off)
    Moved r;
    r.m = m * c.b1 + g * c.one_b1;
    r.v = v * c.b2 + g * g * c.one_b2;
    r.root = sqrtf(r.v);
    r.p = p * c.keep - (r.m / (r.root * c.c2 + c.eps)) * c.rate;
    return r;
}

// four values of a lane, the first of them at `at`; beyond n: 0
template <bool PAST = false, typename T>
__device__ __forceinline__ void load4(const T* x, int64_t at, int64_t n, float (&v)[4]) {
    if (at + 4 <= n) {
        load_pack<T, 4, PAST>(x + at, v);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = at + e < n ? static_cast<float>(x[at + e]) : 0.f;
    }
}
template <bool PAST = false, typename T>
__device__ __forceinline__ void store4(T* x, int64_t at, int64_t n, const float (&v)[4]) {
    if (at + 4 <= n) {
        store_pack<PAST>(x + at, v);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (at + e < n) x[at + e] = static_cast<T>(v[e]);
    }
}
__device__ __forceinline__ uint32_t load4_codes(const uint8_t* x, int64_t at, int64_t n) {
    uint32_t c = 0;
    if (at + 4 <= n) {
        __builtin_memcpy(&c, x + at, 4);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (at + e < n) c |= static_cast<uint32_t>(x[at + e]) << (8 * e);
    }
    return c;
}
__device__ __forceinline__ void store4_codes(uint8_t* x, int64_t at, int64_t n, uint32_t c) {
    if (at + 4 <= n) {
        __builtin_memcpy(x + at, &c, 4);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (at + e < n) x[at + e] = static_cast<uint8_t>(c >> (8 * e));
    }
}

// A wavefront takes blocks of 256 values, four a lane, so that a block's largest magnitude is a reduction of one wavefront; a workgroup
// a chunk of 4096 values of one tensor, found in the list (all tensors in one launch: a small model is launch and latency, 4.9 us
// for 35 tensors of 0.2 M parameters).  Bound by memory: 90 M parameters with moments in 32 bits 394 us, 2465 MB as counted at 6.3
// TB/s; in 8 bits 212 us, 1245 MB at 5.9, and there the vector ALU is busy too (95 %: a square root and a quotient, both rounded
// correctly, and two encodings a value).  By chance 33 us more (90 M, bf16 gradients, 235 / 267 a step): the vector ALU.  With a
// number of its own for either moment 278.
enum { kThirtyTwo, kNearest, kChance };               // moments: in 32 bits, in 8 to nearest, in 8 by chance
template <typename P, typename G, int MOMENTS, bool PAST>
__global__ void __launch_bounds__(kThreads)
k_adamw(const Tensor* tensors, const Chunk* chunks, int split, Coefs c, const Coefs* coefs, const float* grad_scale) {
    constexpr bool EIGHT = MOMENTS != kThirtyTwo;
    float scale = 1.f;
    if (grad_scale) {
        scale = *grad_scale;
        if (!(fabsf(scale) < INFINITY)) return;       // gradients that are not finite: no step
    }
    if (coefs) c = *coefs;
    // (from the last chunk down: the gradients' norm has just read them upwards, and the caches hold the end of them)
    const unsigned place = gridDim.x - 1 - blockIdx.x;
    const Chunk ch = chunks[place / split];
    const Tensor t = tensors[ch.tensor];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, each = kChunk / kBlock8 / split, from = place % split * each;
    const int64_t begin = static_cast<int64_t>(ch.part) * kChunk;
    for (int k = from + wave; k < from + each; k += kThreads / 64) {
        const int64_t block = begin + k * kBlock8, at = block + lane * 4;
        if (block >= t.n) return;                     // (the whole wavefront)
        float p[4], g[4], m[4], v[4], root[4], old_m[4], old_root[4];
        load4<PAST>(static_cast<const P*>(t.p), at, t.n, p);
        load4(static_cast<const G*>(t.g), at, t.n, g);
        if (EIGHT) {
            const int32_t mb = base_of(t.m_exp[block / kBlock8]), vb = base_of(t.v_exp[block / kBlock8]);
            const uint32_t mc = load4_codes(static_cast<const uint8_t*>(t.m), at, t.n);
            const uint32_t vc = load4_codes(static_cast<const uint8_t*>(t.v), at, t.n);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                m[e] = first_of(mc >> (8 * e) & 0xff, mb);
                const float r = root_of(vc >> (8 * e) & 0xff, vb);
                v[e] = r * r;
                old_m[e] = m[e], old_root[e] = r;
            }
        } else {
            load4<PAST>(static_cast<const float*>(t.m), at, t.n, m);
            load4<PAST>(static_cast<const float*>(t.v), at, t.n, v);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const Moved r = move(p[e], grad_scale ? g[e] * scale : g[e], m[e], v[e], c);
            p[e] = r.p, m[e] = r.m, v[e] = r.v, root[e] = r.root;
        }
        store4<PAST>(static_cast<P*>(t.p), at, t.n, p);
        if (EIGHT) {
            // (values beyond n are 0 all along)
            int32_t mm = 0, vm = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                mm = max(mm, bits_of(m[e]) & 0x7fffffff);
                vm = max(vm, bits_of(root[e]) & 0x7fffffff);
            }
            int32_t me = exponent_of(wave_max_bits(mm)), ve = exponent_of(wave_max_bits(vm));
            uint32_t mc = 0, vc = 0;
            if constexpr (MOMENTS == kChance) {
                // four values' numbers come from one output, 16 bits each (the same ones for both moments)
                const uint64_t state = static_cast<uint64_t>(c.chance[1]) << 32 | c.chance[0];
                const uint64_t z = splitmix(state, static_cast<uint64_t>(place / split) * (kChunk / 4) + static_cast<uint32_t>(k * kBlock8 / 4 + lane) + 1);
                const uint32_t low = static_cast<uint32_t>(z), high = static_cast<uint32_t>(z >> 32);
                const uint32_t r[4] = {low & 0xffff, low >> 16, high & 0xffff, high >> 16};
                mc = codes_by_chance<true>(m, old_m, r, me);
                vc = codes_by_chance<false>(root, old_root, r, ve);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    mc |= code_of_first(m[e], base_of(me)) << (8 * e);
                    vc |= code_of_root(root[e], base_of(ve)) << (8 * e);
                }
            }
            store4_codes(static_cast<uint8_t*>(t.m), at, t.n, mc);
            store4_codes(static_cast<uint8_t*>(t.v), at, t.n, vc);
            if (lane == 0) {
                t.m_exp[block / kBlock8] = static_cast<uint8_t>(me);
                t.v_exp[block / kBlock8] = static_cast<uint8_t>(ve);
            }
        } else {
            store4<PAST>(static_cast<float*>(t.m), at, t.n, m);
            store4<PAST>(static_cast<float*>(t.v), at, t.n, v);
        }
    }
}

// Memory: 90 M parameters read back in 86 us, 540 MB at 6.3 TB/s.
// The list's p and g take the moments' values: 8 bits into bf16 (exactly), or (WRITE) binary32 values p, g into 8 bits.
template <bool WRITE, bool PAST>
__global__ void __launch_bounds__(kThreads) k_moments(const Tensor* tensors, const Chunk* chunks, int split) {
    const Chunk ch = chunks[blockIdx.x / split];
    const Tensor t = tensors[ch.tensor];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, each = kChunk / kBlock8 / split, from = blockIdx.x % split * each;
    const int64_t begin = static_cast<int64_t>(ch.part) * kChunk;
    for (int k = from + wave; k < from + each; k += kThreads / 64) {
        const int64_t block = begin + k * kBlock8, at = block + lane * 4;
        if (block >= t.n) return;
        float m[4], v[4];
        if (WRITE) {
            load4(static_cast<const float*>(t.p), at, t.n, m);
            load4(static_cast<const float*>(t.g), at, t.n, v);
            int32_t mm = 0, vm = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                mm = max(mm, bits_of(m[e]) & 0x7fffffff);
                vm = max(vm, bits_of(v[e]) & 0x7fffffff);
            }
            const int32_t me = exponent_of(wave_max_bits(mm)), ve = exponent_of(wave_max_bits(vm));
            uint32_t mc = 0, vc = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                mc |= code_of_first(m[e], base_of(me)) << (8 * e);
                vc |= code_of_root(v[e], base_of(ve)) << (8 * e);
            }
            store4_codes(static_cast<uint8_t*>(t.m), at, t.n, mc);
            store4_codes(static_cast<uint8_t*>(t.v), at, t.n, vc);
            if (lane == 0) {
                t.m_exp[block / kBlock8] = static_cast<uint8_t>(me);
                t.v_exp[block / kBlock8] = static_cast<uint8_t>(ve);
            }
        } else {
            const int32_t mb = base_of(t.m_exp[block / kBlock8]), vb = base_of(t.v_exp[block / kBlock8]);
            const uint32_t mc = load4_codes(static_cast<const uint8_t*>(t.m), at, t.n);
            const uint32_t vc = load4_codes(static_cast<const uint8_t*>(t.v), at, t.n);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                m[e] = first_of(mc >> (8 * e) & 0xff, mb);
                v[e] = root_of(vc >> (8 * e) & 0xff, vb);
            }
            store4<PAST>(static_cast<bf16*>(t.p), at, t.n, m);
            store4<PAST>(static_cast<bf16*>(const_cast<void*>(t.g)), at, t.n, v);
        }
    }
}

__device__ __forceinline__ double block_sum(double s, double* lds) {
#pragma unroll
    for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
    __syncthreads();
    return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

// Squares and their sums in binary64: no overflow, and nothing lost between large and small tensors.  Workgroup w takes chunks
// w, w + workers, ...; a thread's four requests of a chunk are under way together.  90 M gradients in 32 bits 59 us (360 MB at 6.1
// TB/s), in bf16 37 (4.9).
// ADVANCE: one workgroup more, the first, makes the coefficients of the step that these gradients are for, if it is taken.  (By a thread of
// k_grad_norm, which nothing hides, 2 us a step.)
constexpr int kSquares = 2048;                       // workgroups, and partial sums
struct Counted {
    cs_adamw h;
    int64_t* step;
    const double* lr;
    Coefs* coefs;
};
template <typename G, bool ADVANCE>
__global__ void __launch_bounds__(kThreads)
k_grad_squares(const Tensor* tensors, const Chunk* chunks, int64_t count, double* partials, Counted counted) {
    __shared__ double lds[4];
    if (ADVANCE && blockIdx.x == 0) {
        if (threadIdx.x == 0) *counted.coefs = coefs_of(counted.h, counted.lr ? *counted.lr : counted.h.lr, *counted.step + 1);
        return;
    }
    const unsigned worker = blockIdx.x - ADVANCE, workers = gridDim.x - ADVANCE;
    double s = 0.;
    // (where the next chunk lies is looked up while this one's values are on their way)
    Chunk ch = chunks[worker];
    int64_t n = tensors[ch.tensor].n, begin = static_cast<int64_t>(ch.part) * kChunk;
    const G* g = static_cast<const G*>(tensors[ch.tensor].g);
    for (int64_t c = worker; c < count;) {
        constexpr int PER = kChunk / kThreads / 4;
        float v[PER][4];
        if (begin + kChunk <= n) {
#pragma unroll
            for (int k = 0; k < PER; ++k) load_pack<G, 4>(g + begin + (k * kThreads + threadIdx.x) * 4, v[k]);
        } else {
#pragma unroll
            for (int k = 0; k < PER; ++k) load4(g, begin + (k * kThreads + threadIdx.x) * 4, n, v[k]);
        }
        c += workers;
        if (c < count) {
            ch = chunks[c];
            n = tensors[ch.tensor].n;
            begin = static_cast<int64_t>(ch.part) * kChunk;
            g = static_cast<const G*>(tensors[ch.tensor].g);
        }
#pragma unroll
        for (int k = 0; k < PER; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) s = fma(static_cast<double>(v[k][e]), static_cast<double>(v[k][e]), s);
    }
    s = block_sum(s, lds);
    if (threadIdx.x == 0) partials[worker] = s;
}
// step (may be null): counted up where the norm is finite
__global__ void __launch_bounds__(kThreads) k_grad_norm(const double* partials, int count, double max_norm, float* out, int64_t* step) {
    __shared__ double lds[4];
    const int64_t steps = step && threadIdx.x == 0 ? *step : 0;
    double v[kSquares / kThreads], s = 0.;
#pragma unroll
    for (int k = 0; k < kSquares / kThreads; ++k) {
        const int i = k * kThreads + threadIdx.x;
        v[k] = i < count ? partials[i] : 0.;
    }
#pragma unroll
    for (int k = 0; k < kSquares / kThreads; ++k) s += v[k];
    s = block_sum(s, lds);
    if (threadIdx.x) return;
    // (finite as it is told, in binary32)
    const double norm = sqrt(s), c = max_norm / (norm + 1e-6);
    const bool finite = static_cast<float>(norm) < INFINITY;
    if (step && finite) *step = steps + 1;
    out[0] = static_cast<float>(norm);
    out[1] = finite ? static_cast<float>(c < 1. ? c : 1.) : NAN;
}

__global__ void k_adamw_coefs(cs_adamw h, int64_t* step, const double* lr, const float* grad_scale, Coefs* out) {
    if (grad_scale && !(fabsf(*grad_scale) < INFINITY)) return;
    const int64_t t = ++*step;
    *out = coefs_of(h, lr ? *lr : h.lr, t);
}
static_assert(sizeof(Coefs) == 4 * CS_ADAMW_COEFS, "csketch.h");

// ---------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------
// Chunks from which moments are read back by one workgroup a chunk (52 M, 8 bits: 212 us a pass, with four 226).
constexpr int64_t kReadWhole = 8192;
constexpr int64_t kMaxValues = static_cast<int64_t>(1) << 40, kMaxChunks = static_cast<int64_t>(1) << 24;   // (2^32 threads a launch)

int64_t chunks_of(const int64_t* n, int32_t count, int64_t& values, bool& ok) {
    int64_t chunks = 0;
    values = 0;
    ok = true;
    for (int32_t i = 0; i < count; ++i) {
        if (n[i] < 0 || n[i] > kMaxValues || (values += n[i]) > kMaxValues) {
            ok = false;
            return 0;
        }
        chunks += (n[i] + kChunk - 1) / kChunk;
    }
    return chunks;
}

// what a cs_tensor_list says of its device memory
struct List {
    const Tensor* tensors;
    const Chunk* chunks;
};
List list_of(const cs_tensor_list* l) {
    const Tensor* t = static_cast<const Tensor*>(l->memory);
    return List{t, reinterpret_cast<const Chunk*>(t + l->count)};
}
// Workgroups that share a chunk: four, a block of 256 values a wavefront, so that none waits for memory four times in a row; but of
// moments in 8 bits that go past the caches one (us a step, one / four: 0.64 M parameters, 8 bits 15.1 / 11.7; 11.5 M, 32 bits 69 / 63;
// 90 M, 32 bits with clipping 474 / 462; 30 M, 8 bits 141 / 132; 52 M, 8 bits, past the caches 212 / 234).
// A launch has fewer than 2^32 threads: a list of 2^22 chunks or more is not split.
int split_of(int64_t chunks, bool one) { return one || chunks * 4 >= kMaxChunks ? 1 : 4; }
int partials_of(const cs_tensor_list* l) { return static_cast<int>(l->chunks < kSquares ? l->chunks : kSquares); }
int64_t list_bytes(const cs_tensor_list* l) {
    return l->count * static_cast<int64_t>(sizeof(Tensor)) + l->chunks * static_cast<int64_t>(sizeof(Chunk));
}
bool list_ok(const cs_tensor_list* l) {
    return l && l->count >= 0 && l->chunks >= 0 && l->chunks < kMaxChunks && (l->chunks == 0 || l->memory);
}

template <typename P, typename G>
int adamw(const cs_tensor_list* l, const Coefs& c, bool chance, const Coefs* coefs, const float* grad_scale, hipStream_t stream) {
    const List at = list_of(l);
    // Parameters and moments that the memory-side cache cannot keep are read and written past it: what it keeps is
    // the gradients that their norm has just read.
    const int64_t each = fmt_bytes(l->p_fmt) + (l->bits == 8 ? 2 : 8);
    const bool past = past_caches(l->values * each);
    const int split = split_of(l->chunks, past && l->bits == 8);
    const unsigned grid = static_cast<unsigned>(l->chunks * split);
    const auto kernel = l->bits == 32 ? (past ? k_adamw<P, G, kThirtyTwo, true> : k_adamw<P, G, kThirtyTwo, false>)
                        : chance      ? (past ? k_adamw<P, G, kChance, true> : k_adamw<P, G, kChance, false>)
                                      : (past ? k_adamw<P, G, kNearest, true> : k_adamw<P, G, kNearest, false>);
    kernel<<<grid, kThreads, 0, stream>>>(at.tensors, at.chunks, split, c, coefs, grad_scale);
    return launched();
}
template <typename P>
int adamw_p(const cs_tensor_list* l, const Coefs& c, bool chance, const Coefs* coefs, const float* grad_scale, hipStream_t stream) {
    if (l->g_fmt == CS_FMT_F32) return adamw<P, float>(l, c, chance, coefs, grad_scale, stream);
    if (l->g_fmt == CS_FMT_BF16) return adamw<P, bf16>(l, c, chance, coefs, grad_scale, stream);
    return adamw<P, f16>(l, c, chance, coefs, grad_scale, stream);
}

bool hyper_ok(const cs_adamw* h) {
    return h && h->lr >= 0. && h->lr < INFINITY && h->beta1 >= 0. && h->beta1 < 1. && h->beta2 >= 0. && h->beta2 < 1. &&
           h->eps >= 0. && h->eps < INFINITY && h->weight_decay >= 0. && h->weight_decay < INFINITY;
}

}  // namespace
}  // namespace cs

using namespace cs;

extern "C" int cs_tensor_list_bytes(const int64_t* n, int32_t count, size_t* bytes) {
    bool ok = false;
    int64_t values = 0;
    if (count < 0 || (count && !n) || !bytes) return CS_EINVAL;
    const int64_t chunks = chunks_of(n, count, values, ok);
    if (!ok || chunks >= kMaxChunks) return CS_EINVAL;
    *bytes = static_cast<size_t>(count) * sizeof(Tensor) + static_cast<size_t>(chunks) * sizeof(Chunk);
    return CS_OK;
}

extern "C" int cs_tensor_list_build(const int64_t* n, int32_t count, void* const* p, int32_t p_fmt, const void* const* g,
                                    int32_t g_fmt, void* const* m, void* const* v, int32_t bits, uint8_t* const* m_exp,
                                    uint8_t* const* v_exp, void* memory, size_t bytes, cs_tensor_list* list, void* stream) {
    size_t need = 0;
    if (int rc = cs_tensor_list_bytes(n, count, &need)) return rc;
    if (!list || !fmt_ok(p_fmt) || !fmt_ok(g_fmt) || (bits != 8 && bits != 32)) return CS_EINVAL;
    if (count && (!p || !g || !m || !v || (bits == 8 && (!m_exp || !v_exp)))) return CS_EINVAL;
    if (bytes < need) return CS_EWORKSPACE;
    if (need && (!memory || (reinterpret_cast<uintptr_t>(memory) & 7))) return CS_EINVAL;
    const int64_t pb = fmt_bytes(p_fmt), gb = fmt_bytes(g_fmt), sb = bits / 8;
    for (int32_t i = 0; i < count; ++i) {
        if (n[i] == 0) continue;
        const uintptr_t all[] = {reinterpret_cast<uintptr_t>(p[i]), reinterpret_cast<uintptr_t>(g[i]),
                                 reinterpret_cast<uintptr_t>(m[i]), reinterpret_cast<uintptr_t>(v[i])};
        if (!all[0] || !all[1] || !all[2] || !all[3] || all[0] % pb || all[1] % gb || (bits == 32 && (all[2] % 4 || all[3] % 4)))
            return CS_EINVAL;
        if (bits == 8 && (!m_exp[i] || !v_exp[i])) return CS_EINVAL;
        // what a step writes of one tensor lies apart from the rest of it
        const int64_t blocks = (n[i] + kBlock8 - 1) / kBlock8;
        const void* at[] = {p[i], m[i], v[i], bits == 8 ? m_exp[i] : nullptr, bits == 8 ? v_exp[i] : nullptr, g[i]};
        const int64_t size[] = {pb * n[i], sb * n[i], sb * n[i], blocks, blocks, gb * n[i]};
        for (int a = 0; a < 6; ++a)
            for (int b = 0; b < a; ++b)
                if (spans_meet(at[a], size[a], at[b], size[b])) return CS_EINVAL;
    }
    bool ok = false;
    int64_t values = 0;
    const int64_t chunks = chunks_of(n, count, values, ok);
    *list = cs_tensor_list{memory, chunks, count, p_fmt, g_fmt, bits, values};
    if (count == 0) return CS_OK;
    Tensor* tensors = static_cast<Tensor*>(memory);
    int64_t chunk = 0;
    for (int32_t i = 0; i < count; i += kBatch) {
        Batch b = {};
        const int k = count - i < kBatch ? count - i : kBatch;
        for (int j = 0; j < k; ++j) {
            b.t[j] = Tensor{p[i + j], g[i + j], m[i + j], v[i + j], bits == 8 ? m_exp[i + j] : nullptr,
                            bits == 8 ? v_exp[i + j] : nullptr, n[i + j], chunk};
            chunk += (n[i + j] + kChunk - 1) / kChunk;
        }
        k_list_tensors<<<1, 64, 0, stream_of(stream)>>>(b, tensors + i, k);
        if (int rc = launched()) return rc;
    }
    if (chunk == 0) return CS_OK;
    k_list_chunks<<<static_cast<unsigned>((chunk + kThreads - 1) / kThreads), kThreads, 0, stream_of(stream)>>>(
        tensors, count, reinterpret_cast<Chunk*>(tensors + count), chunk);
    return launched();
}

extern "C" int cs_grad_norm_workspace_bytes(const cs_tensor_list* list, size_t* bytes) {
    if (!list_ok(list) || !bytes) return CS_EINVAL;
    *bytes = static_cast<size_t>(partials_of(list)) * sizeof(double);
    return CS_OK;
}

namespace cs {
namespace {

int grad_norm(const cs_tensor_list* list, double max_norm, float* out, void* workspace, size_t ws_bytes, const cs_adamw* h,
              int64_t* step, const double* lr, float* coefs, void* stream) {
    if (!list_ok(list) || !out || !(max_norm > 0.)) return CS_EINVAL;
    const size_t need = static_cast<size_t>(partials_of(list)) * sizeof(double);
    if (ws_bytes < need) return CS_EWORKSPACE;
    if (need && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 7))) return CS_EINVAL;
    const Span written[] = {{out, 8}, {need ? workspace : nullptr, static_cast<int64_t>(need)}, {step, 8}, {coefs, 4 * CS_ADAMW_COEFS}};
    const Span read[] = {{list->memory, list_bytes(list)}, {lr, 8}};
    if (!spans_apart(written, read)) return CS_EINVAL;
    const List at = list_of(list);
    double* partials = static_cast<double*>(workspace);
    const int grid = partials_of(list);
    const hipStream_t s = stream_of(stream);
    if (grid || step) {
        const auto kernel = list->g_fmt == CS_FMT_F32    ? (step ? k_grad_squares<float, true> : k_grad_squares<float, false>)
                            : list->g_fmt == CS_FMT_BF16 ? (step ? k_grad_squares<bf16, true> : k_grad_squares<bf16, false>)
                                                         : (step ? k_grad_squares<f16, true> : k_grad_squares<f16, false>);
        kernel<<<grid + (step != nullptr), kThreads, 0, s>>>(
            at.tensors, at.chunks, list->chunks, partials,
            step ? Counted{*h, step, lr, reinterpret_cast<Coefs*>(coefs)} : Counted{});
        if (int rc = launched()) return rc;
    }
    k_grad_norm<<<1, kThreads, 0, s>>>(partials, grid, max_norm, out, step);
    return launched();
}

}  // namespace
}  // namespace cs

extern "C" int cs_grad_norm(const cs_tensor_list* list, double max_norm, float* out, void* workspace, size_t ws_bytes, void* stream) {
    return grad_norm(list, max_norm, out, workspace, ws_bytes, nullptr, nullptr, nullptr, nullptr, stream);
}

extern "C" int cs_grad_norm_advance(const cs_tensor_list* list, double max_norm, float* out, void* workspace, size_t ws_bytes,
                                    const cs_adamw* h, int64_t* step, const double* lr_or_null, float* coefs, void* stream) {
    if (!hyper_ok(h) || !step || !coefs) return CS_EINVAL;
    return grad_norm(list, max_norm, out, workspace, ws_bytes, h, step, lr_or_null, coefs, stream);
}

extern "C" int cs_adamw_advance_scaled(const cs_adamw* h, int64_t* step, const double* lr_or_null, const float* grad_scale_or_null,
                                       float* coefs, void* stream) {
    if (!hyper_ok(h) || !step || !coefs) return CS_EINVAL;
    const Span written[] = {{step, 8}, {coefs, 4 * CS_ADAMW_COEFS}}, read[] = {{lr_or_null, 8}, {grad_scale_or_null, 4}};
    if (!spans_apart(written, read)) return CS_EINVAL;
    k_adamw_coefs<<<1, 1, 0, stream_of(stream)>>>(*h, step, lr_or_null, grad_scale_or_null, reinterpret_cast<Coefs*>(coefs));
    return launched();
}

extern "C" int cs_adamw_advance(const cs_adamw* h, int64_t* step, const double* lr_or_null, float* coefs, void* stream) {
    return cs_adamw_advance_scaled(h, step, lr_or_null, nullptr, coefs, stream);
}

extern "C" int cs_adamw_step(const cs_adamw* h, int64_t step, const cs_tensor_list* list, const float* coefs_or_null,
                             const float* grad_scale_or_null, void* stream) {
    if (!hyper_ok(h) || !list_ok(list) || (!coefs_or_null && step < 1)) return CS_EINVAL;
    if (list->chunks == 0) return CS_OK;
    const Coefs c = coefs_or_null ? Coefs{} : coefs_of(*h, h->lr, step);
    const Coefs* dc = reinterpret_cast<const Coefs*>(coefs_or_null);
    const hipStream_t s = stream_of(stream);
    const bool chance = h->seed != 0;
    if (list->p_fmt == CS_FMT_F32) return adamw_p<float>(list, c, chance, dc, grad_scale_or_null, s);
    if (list->p_fmt == CS_FMT_BF16) return adamw_p<bf16>(list, c, chance, dc, grad_scale_or_null, s);
    return adamw_p<f16>(list, c, chance, dc, grad_scale_or_null, s);
}

extern "C" int cs_moments_read(const cs_tensor_list* list, void* stream) {
    if (!list_ok(list) || list->bits != 8 || list->p_fmt != CS_FMT_BF16 || list->g_fmt != CS_FMT_BF16) return CS_EINVAL;
    if (list->chunks == 0) return CS_OK;
    const List at = list_of(list);
    const bool past = past_caches(list->values * 4);
    const auto kernel = past ? k_moments<false, true> : k_moments<false, false>;
    const int split = split_of(list->chunks, list->chunks >= kReadWhole);
    kernel<<<static_cast<unsigned>(list->chunks * split), kThreads, 0, stream_of(stream)>>>(at.tensors, at.chunks, split);
    return launched();
}

extern "C" int cs_moments_write(const cs_tensor_list* list, void* stream) {
    if (!list_ok(list) || list->bits != 8 || list->p_fmt != CS_FMT_F32 || list->g_fmt != CS_FMT_F32) return CS_EINVAL;
    if (list->chunks == 0) return CS_OK;
    const List at = list_of(list);
    const int split = split_of(list->chunks, false);
    k_moments<true, false><<<static_cast<unsigned>(list->chunks * split), kThreads, 0, stream_of(stream)>>>(at.tensors, at.chunks, split);
    return launched();
}

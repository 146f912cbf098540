// Log probabilities of given tokens under rows of logits, with the entropy and the largest alternatives of every row,
// and the gradient of log probability and entropy.  With z = scale x:
//     lse = ln sum exp z,  logp = z_t - lse,  H = lse - sum p z,  p = exp(z - lse)
//     dx_v = scale (g ([v = t] - p_v) - h p_v (ln p_v + H))
// One pass over a row keeps a running reference B, s = sum 2^d and u = sum 2^d d with d = x k - B, k = scale log2(e): one
// fused multiply-add, one exponential and two accumulations a value, all in binary32.  B is a binary32 number that is at
// least k times the largest value so far (up to rounding), so d is exact up to one rounding of its own size however
// large the logits are.
#pragma once

#include <hip/hip_runtime.h>
#include <float.h>
#include <stdint.h>

#include "cs_rows.h"
#include "cs_token.h"
#include "csketch.h"

namespace cs {
namespace {

constexpr int kThreads = 256;                // of a row among many, and of the kernels that go by packs
constexpr int kFewThreads = 1024;            // of a row among few, or of its part
constexpr int kList = 1024;                  // candidates for the alternatives of a part
constexpr float kLog2e = 1.44269504088896341f, kLn2 = 0.69314718055994531f;
constexpr float kFar = -200.f;               // 2^kFar is 0 beside any sum
constexpr float kPlain = -1e30f;             // values above this leave no product in the infinite

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// Values in order as whole numbers; -0 is 0, a NaN counts as -inf.  With the index below it, what is larger comes first
// among alternatives; 0 is none.
__device__ __forceinline__ uint32_t order_of(float v) {
    v = v == v ? v + 0.0f : -INFINITY;
    const uint32_t u = __float_as_uint(v);
    return u ^ (static_cast<uint32_t>(static_cast<int32_t>(u) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float ranked(float v) { return v == v ? v : -INFINITY; }
__device__ __forceinline__ float value_of(uint32_t order) {
    return __uint_as_float(order & 0x80000000u ? order ^ 0x80000000u : ~order);
}
__device__ __forceinline__ uint64_t key_of(float v, int64_t at) {
    return static_cast<uint64_t>(order_of(v)) << 32 | (0xffffffffu - static_cast<uint32_t>(at));
}
__device__ __forceinline__ int64_t index_of(uint64_t key) { return 0xffffffffu - static_cast<uint32_t>(key); }
// bits at the lower end of an order that a type's values have alike
template <typename T>
constexpr int kAlike = sizeof(T) == 4 ? 0 : sizeof(T) == 2 && static_cast<float>(static_cast<T>(65536.f)) == 65536.f ? 16 : 13;

// THREADS threads hold or share a row; 64: a wavefront, which needs no barrier
template <int THREADS>
struct TokenShared {
    static constexpr int UNIT = THREADS == 64 ? 1 : 4, LIST = THREADS == 64 ? 256 : kList;
    float f[3][16];
    int32_t order[THREADS / UNIT], pack[THREADS / UNIT];
    uint64_t list[LIST];
    static constexpr int HITS = THREADS == 64 ? 64 : 256;
    int32_t chosen[kMaxTop * UNIT];
    uint32_t hit[HITS][4];                   // packs that reach the bound, and which they are
    int32_t hit_pack[HITS];
    int32_t n, chosen_n;
    uint64_t best[16];
};
template <int THREADS>
__device__ __forceinline__ int thread_of_row() { return threadIdx.x % THREADS; }
template <int THREADS>
__device__ __forceinline__ void row_sync() {
    if (THREADS == 64) {
        // (a wavefront's accesses to LDS are served in order)
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    } else {
        __syncthreads();
    }
}

template <int THREADS>
__device__ __forceinline__ float block_max(float v, float (&buf)[16]) {
    v = wave_max(v);
    if (THREADS == 64) return v;
    if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
    __syncthreads();
    v = buf[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) v = fmaxf(v, buf[w]);
    return v;
}
// (buffers of its own: no barrier before)
template <int THREADS>
__device__ __forceinline__ void block_add2(float& a, float& b, float (&ba)[16], float (&bb)[16]) {
    a = wave_sum(a);
    b = wave_sum(b);
    if (THREADS == 64) return;
    if ((threadIdx.x & 63) == 0) {
        ba[threadIdx.x >> 6] = a;
        bb[threadIdx.x >> 6] = b;
    }
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        a += ba[w];
        b += bb[w];
    }
}

// What a thread has seen of its part of a row: packs first, first + THREADS, ...
template <typename T, bool TOP>
struct Scan {
    static constexpr int P = kPack<T>;
    float B = -FLT_MAX, s = 0.f, u = 0.f, most = -INFINITY;
    int32_t most_pack = INT32_MAX;           // TOP: the first pack with that value

    // a pack's largest and lowest value into top and low
    __device__ __forceinline__ void look(const float (&v)[P], int32_t pack, float& top, float& low) {
        float t = fmaxf(v[0], v[1]);
#pragma unroll
        for (int e = 2; e < P; e += 2) t = fmaxf(fmaxf(v[e], v[e + 1]), t);
#pragma unroll
        for (int e = 0; e < P; e += 2) low = fminf(fminf(v[e], v[e + 1]), low);
        if (TOP) {
            // (the first pack counts also where it holds nothing above -inf)
            if (t > most || most_pack == INT32_MAX) {
                most = t == t ? t : -INFINITY;
                most_pack = pack;
            }
        }
        top = fmaxf(top, t);
    }
    // the largest value yet: sums relative to it
    __device__ __forceinline__ void raise(float top, float k) {
        if (!TOP) most = fmaxf(most, top);
        const float b = top * k;
        if (b > B) {
            const float f = exp2_of(B - b);
            u = f * fmaf(s, fmaxf(B - b, kFar), u);
            s *= f;
            B = b;
        }
    }
    // GUARDED: values may be -inf
    template <bool GUARDED>
    __device__ __forceinline__ void add(const float (&v)[P], float k) {
#pragma unroll
        for (int e = 0; e < P; ++e) {
            const float d = fmaf(v[e], k, -B), x = exp2_of(d);
            s += x;
            u = fmaf(x, GUARDED ? fmaxf(d, kFar) : d, u);
        }
    }
    // N packs, the first `count` of which there are; number j is pack + j * step
    template <int N>
    __device__ __forceinline__ void meet(const float (&v)[N][P], int count, float k, int32_t pack, int32_t step) {
        float top = -INFINITY, low = INFINITY;
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (j < count) look(v[j], pack + j * step, top, low);
        raise(top, k);
        if (low > kPlain) {
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (j < count) add<false>(v[j], k);
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (j < count) add<true>(v[j], k);
        }
    }
};

// the last pack of a row, where the row ends inside it
template <typename T>
__device__ __forceinline__ void load_tail(const T* row, int64_t at, int64_t vocab, float (&v)[kPack<T>]) {
#pragma unroll
    for (int e = 0; e < kPack<T>; ++e) v[e] = at + e < vocab ? static_cast<float>(row[at + e]) : -INFINITY;
}

// Packs [first, last) of a row (`last` may be one that the row ends in): the thread's own sums.
template <typename T, bool TOP, int THREADS>
__device__ __forceinline__ void scan_packs(const T* row, int64_t vocab, int32_t first, int32_t last, float k, Scan<T, TOP>& scan) {
    constexpr int P = kPack<T>, N = sizeof(T) == 4 ? 4 : THREADS == kFewThreads ? 2 : 1;
    const int32_t whole = static_cast<int32_t>(vocab / P);         // packs before one that the row ends in
    const int32_t stop = last < whole ? last : whole;
    for (int32_t q = first + static_cast<int32_t>(threadIdx.x); q < stop; q += N * THREADS) {
        const int32_t count = min(N, (stop - q + THREADS - 1) / THREADS);
        Raw<T, P> raw[N];
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (j < count) raw[j].load(row + static_cast<int64_t>(q + j * THREADS) * P);
        float v[N][P];
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int e = 0; e < P; ++e) v[j][e] = raw[j][e];
        if (count == N) scan.template meet<N>(v, N, k, q, THREADS);
        else scan.template meet<N>(v, count, k, q, THREADS);
    }
    if (last > whole && first <= whole && (whole - first) % THREADS == static_cast<int32_t>(threadIdx.x)) {
        float v[1][P];
        load_tail(row, static_cast<int64_t>(whole) * P, vocab, v[0]);
        scan.template meet<1>(v, 1, k, whole, THREADS);
    }
}

// the sums of all threads
template <typename T, bool TOP, int THREADS>
__device__ __forceinline__ Sums join_threads(const T* row, int64_t vocab, int32_t first, int32_t last, float scale, float k,
                                             TokenShared<THREADS>& sh, const Scan<T, TOP>& scan) {
    constexpr int P = kPack<T>;
    Sums r;
    r.m = block_max<THREADS>(scan.most, sh.f[0]);
    const float B = block_max<THREADS>(scan.B, sh.f[1]);
    row_sync<THREADS>();
    const float f = exp2_of(scan.B - B);
    float s = scan.s * f, u = f * fmaf(scan.s, fmaxf(scan.B - B, kFar), scan.u);
    block_add2<THREADS>(s, u, sh.f[0], sh.f[2]);
    // from B to the largest value itself
    const float off = fmaf(r.m, k, -B), g = exp2_of(-off);
    r.S = s * g;
    r.U = g * fmaf(-off, s, u);
    // Where the reference or a product leaves binary32 (values beyond 2e38: masks of the type's lowest value in a row that has
    // nothing else; a scale beyond 1e8), where the row holds a NaN or +inf, and where the reference is that large (2^22) that it may be
    // more than 1/4 from the largest value's product (U would be a small difference of large numbers), once more with differences of the
    // values themselves (and the scale itself, as k may be infinite).  (The largest value adds 1 to S.)
    if (!(r.S >= 0.5f && r.S < INFINITY && fabsf(r.U) < INFINITY && fabsf(off) <= 0.25f) && r.m > -INFINITY) {
        row_sync<THREADS>();
        s = u = 0.f;
        const int64_t end = static_cast<int64_t>(last) * P < vocab ? static_cast<int64_t>(last) * P : vocab;
#pragma unroll 2
        for (int64_t i = static_cast<int64_t>(first) * P + thread_of_row<THREADS>(); i < end; i += THREADS) {
            const float d = (static_cast<float>(row[i]) - r.m) * scale * kLog2e, x = exp2_of(d);
            s += x;
            u = fmaf(x, fmaxf(d, kFar), u);
        }
        block_add2<THREADS>(s, u, sh.f[0], sh.f[2]);
        r.S = s;
        r.U = u;
    } else if (r.m == -INFINITY && !(s == s)) {      // NaN and -inf alone
        r.S = r.U = s;
    } else if (r.m == -INFINITY) {
        r.S = r.U = 0.f;
    }
    return r;
}

// `n` keys ranked by counting; those before `top` go to emit(rank, key)
template <int THREADS, typename Emit>
__device__ __forceinline__ void rank_list(const uint64_t* list, int32_t n, int top, Emit emit) {
    for (int32_t i = thread_of_row<THREADS>(); i < n; i += THREADS) {
        const uint64_t key = list[i];
        int32_t before = 0, j = 0;
        for (; j + 8 <= n; j += 8)
#pragma unroll
            for (int e = 0; e < 8; ++e) before += list[j + e] > key;
        for (; j < n; ++j) before += list[j] > key;
        if (before < top) emit(before, key);
    }
}

// The `top` largest of packs [first, last) of a row, in order, by emit(rank, key).  A thread (of a wavefront that has the row
// to itself) or four neighbouring ones are a unit; of the
// units' largest values the top-th in order (equal ones: lower pack first) is a bound that `top` values reach, so the
// largest are among the values of the `top` units before it that reach it too: few more than `top` values where `top` is well below the
// 64 units (at 48 and more a wavefront's row mostly has more than are listed), which
// those threads list and which are then ranked by counting.  The bound is found bit by bit, in every wavefront by itself, a
// unit (or four) a lane.
template <typename T, int THREADS, bool HELD, typename Row, typename Emit>
__device__ __forceinline__ void largest_of_part(const T* row, const Row& held, int64_t vocab, int32_t first, int32_t last, int top,
                                                const Scan<T, true>& scan, TokenShared<THREADS>& sh, Emit emit) {
    constexpr int P = kPack<T>, LOW = kAlike<T>, UNIT = TokenShared<THREADS>::UNIT, PER = THREADS / UNIT / 64;
    constexpr int32_t LIST = TokenShared<THREADS>::LIST;
    const int tid = thread_of_row<THREADS>(), lane = tid & 63;
    const auto pack_at = [&](int32_t q, float(&v)[P]) {
        if ((static_cast<int64_t>(q) + 1) * P <= vocab) load_pack<T, P>(row + static_cast<int64_t>(q) * P, v);
        else load_tail(row, static_cast<int64_t>(q) * P, vocab, v);
    };
    // (orders compare as signed numbers once the top bit is turned; packs too)
    int32_t most = static_cast<int32_t>(order_of(scan.most) ^ 0x80000000u) >> LOW, pack = scan.most_pack;
#pragma unroll
    for (int d = 1; d < UNIT; d <<= 1) {
        const int32_t m = __shfl_xor(most, d), q = __shfl_xor(pack, d);
        if (m > most || (m == most && q < pack)) {
            most = m;
            pack = q;
        }
    }
    if (tid % UNIT == 0) {
        sh.order[tid / UNIT] = most;
        sh.pack[tid / UNIT] = pack;
    }
    if (tid == 0) sh.n = sh.chosen_n = 0;
    row_sync<THREADS>();
    int32_t o[PER], q[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        o[k] = sh.order[lane + 64 * k];
        q[k] = sh.pack[lane + 64 * k];
    }
    // the largest bound that at least `top` units reach
    int32_t bound = INT32_MIN >> LOW;
#pragma unroll
    for (int bit = 31 - LOW; bit >= 0; --bit) {
        // (the sign's bit first: from the lowest number up to 0)
        const int32_t next = bit == 31 - LOW ? 0 : bound + (1 << bit);
        int reach = 0;
#pragma unroll
        for (int k = 0; k < PER; ++k) reach += __popcll(__ballot(o[k] >= next));
        if (reach >= top) bound = next;
    }
    int reach = 0, beyond = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        reach += __popcll(__ballot(o[k] >= bound));
        beyond += __popcll(__ballot(o[k] > bound));
    }
    // of units that are equal to the bound, those with the lowest packs
    int32_t bound_pack = INT32_MAX;
    if (reach > top) {
        bound_pack = 0;                                              // (never beyond twice the last pack; further ones are none)
#pragma unroll 1
        for (int bit = 31 - __clz(last | 1); bit >= 0; --bit) {
            const int32_t below = bound_pack + (1 << bit);           // are there enough below this pack?
            int n = beyond;
#pragma unroll
            for (int k = 0; k < PER; ++k) n += __popcll(__ballot(o[k] == bound && q[k] < below));
            if (n < top) bound_pack = below;
        }
    }
    const bool chosen = most > bound || (most == bound && pack <= bound_pack);
    const auto list = [&](float value, int32_t at_pack, int e) {
        const int64_t at = static_cast<int64_t>(at_pack) * P + e;
        const int32_t x = static_cast<int32_t>(order_of(value) ^ 0x80000000u) >> LOW;
        if (at < vocab && (x > bound || (x == bound && at_pack <= bound_pack))) {
            const int32_t slot = atomicAdd(&sh.n, 1);
            if (slot < LIST) sh.list[slot] = key_of(value, at);
        }
    };
    int32_t n = 0;
    if constexpr (HELD) {
        // the chosen threads hand out those packs that reach the bound
        constexpr int32_t HITS = TokenShared<THREADS>::HITS;
        if (chosen)
            held.each([&](int32_t at_pack, const uint32_t(&w)[4], const float(&v)[P]) {
                float t = ranked(v[0]);
#pragma unroll
                for (int e = 1; e < P; ++e) t = fmaxf(t, v[e]);
                const int32_t o = static_cast<int32_t>(order_of(t) ^ 0x80000000u) >> LOW;
                if (o < bound || (o == bound && at_pack > bound_pack)) return;
                const int32_t slot = atomicAdd(&sh.chosen_n, 1);
                if (slot >= HITS) return;
                sh.hit_pack[slot] = at_pack;
#pragma unroll
                for (int e = 0; e < 4; ++e) sh.hit[slot][e] = w[e];
            });
        row_sync<THREADS>();
        const int32_t hits = sh.chosen_n;
        if (hits > HITS) n = LIST + 1;
        else
            for (int32_t w = tid; w < hits * P; w += THREADS)
                list(static_cast<float>(reinterpret_cast<const T*>(sh.hit[w / P])[w % P]), sh.hit_pack[w / P], w % P);
    } else {
        // the chosen threads' packs are read again by all threads, two requests each under way
        if (chosen) sh.chosen[atomicAdd(&sh.chosen_n, 1)] = tid;
        __syncthreads();
        const uint32_t threads = sh.chosen_n, each = (last - first + THREADS - 1) / THREADS, all = threads * each;
        for (uint32_t w = tid; w < all; w += 2 * THREADS) {
            float v[2][P];
            int32_t at_pack[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint32_t i = w + j * THREADS;
                at_pack[j] = i < all ? first + sh.chosen[i % threads] + static_cast<int32_t>(i / threads) * THREADS : last;
                if (at_pack[j] < last) pack_at(at_pack[j], v[j]);
            }
#pragma unroll
            for (int j = 0; j < 2; ++j)
                if (at_pack[j] < last)
#pragma unroll
                    for (int e = 0; e < P; ++e) list(v[j][e], at_pack[j], e);
        }
    }
    row_sync<THREADS>();
    n = max(n, sh.n);
    if (n <= LIST) {
        rank_list<THREADS>(sh.list, n, top, emit);
        for (int32_t i = n + tid; i < top; i += THREADS) emit(i, 0);
        return;
    }
    // More than the list holds (long runs of equal values): one after the other, each the largest below the one before.
    uint64_t prev = ~0ull;
    for (int r = 0; r < top; ++r) {
        uint64_t best = 0;
        if (chosen)
            for (int32_t at_pack = first + tid; at_pack < last; at_pack += THREADS) {
                const int64_t at = static_cast<int64_t>(at_pack) * P;
                float v[P];
                pack_at(at_pack, v);
                for (int e = 0; e < P; ++e) {
                    const uint64_t key = at + e < vocab ? key_of(v[e], at + e) : 0;
                    if (key < prev && key > best) best = key;
                }
            }
#pragma unroll
        for (int d = 32; d; d >>= 1) {
            const uint64_t other = __shfl_xor(best, d);
            if (other > best) best = other;
        }
        if (THREADS > 64) {
            __syncthreads();
            if (lane == 0) sh.best[tid >> 6] = best;
            __syncthreads();
            for (int w = 0; w < THREADS / 64; ++w)
                if (sh.best[w] > best) best = sh.best[w];
        }
        prev = best;
        if (tid == 0) emit(r, best);
    }
}

// the first pack of a part: parts are alike but for one pack
__host__ __device__ __forceinline__ int32_t part_begin(int64_t part, int32_t packs, int parts) {
    return static_cast<int32_t>(part * packs / parts);
}
// log probability of value x in a row with sums r; `log_sum` = ln S
__device__ __forceinline__ float logp_of(float x, const Sums& r, float log_sum, float scale) {
    // (x = m = -inf: a row with nothing in it gives nothing any probability)
    return r.m == -INFINITY && r.S == r.S ? -INFINITY : fmaf(x - r.m, scale, -log_sum);
}

// the logit of a row's target; counts: there is one
template <typename T>
struct Target {
    float x = 0.f;
    bool counts = false;
    __device__ __forceinline__ void load(const T* row, int64_t vocab, int64_t t) {
        counts = t >= 0 && t < vocab;
        if (counts) x = static_cast<float>(row[t]);
    }
};

// (an empty row's is 0)
__device__ __forceinline__ float entropy_of(const Sums& r, float log_sum) {
    return r.m == -INFINITY && r.S == r.S ? 0.f : log_sum - kLn2 * (r.U / r.S);
}

template <typename T>
__device__ __forceinline__ void row_results(int64_t row, const Target<T>& target, float scale, const Sums& r, float log_sum,
                                            const TokenOut& out) {
    const bool empty = r.m == -INFINITY && r.S == r.S;
    if (out.lse) {
        // (-inf says that a row is empty: a number below binary32 is the lowest there is)
        const float lse = fmaf(r.m, scale, log_sum);
        out.lse[row] = empty ? -INFINITY : lse < -FLT_MAX ? -FLT_MAX : lse;
    }
    if (out.entropy) out.entropy[row] = entropy_of(r, log_sum);
    if (out.logp) out.logp[row] = target.counts ? logp_of(target.x, r, log_sum, scale) : 0.f;
}

// Rows as a stream, for what is not held: one read, online sums.  kThreads a row where there are rows enough to fill the chip: 2047 x
// 50021 f16 41 us, 205 MB at 5.0 TB/s (vector ALU 55 % busy; one round of workgroups, whose beginning and end nothing hides),
// 4096 x 32001 f32 93 us, 524 MB at 5.6.  Of few rows kFewThreads each, and parts of long ones, for latency.
template <typename T, bool TOP, int THREADS>
__global__ void __launch_bounds__(THREADS)
k_token(const T* logits, int64_t vocab, int64_t stride, float scale, const int64_t* target, TokenOut out, int top, int parts,
        int32_t packs, Parts ws) {
    __shared__ TokenShared<THREADS> sh;
    const int64_t row = blockIdx.x / static_cast<unsigned>(parts);
    const int part = blockIdx.x % static_cast<unsigned>(parts);
    const T* x = logits + row * stride;
    const int32_t first = part_begin(part, packs, parts), last = part_begin(part + 1, packs, parts);
    const float k = scale * kLog2e;
    const bool results = parts == 1 && threadIdx.x == 0;
    const int64_t t = results && out.logp ? target[row] : -1;
    Scan<T, TOP> scan;
    scan_packs<T, TOP, THREADS>(x, vocab, first, last, k, scan);
    Target<T> hit;
    hit.load(x, vocab, t);
    const Sums r = join_threads<T, TOP, THREADS>(x, vocab, first, last, scale, k, sh, scan);
    const float log_sum = logf(r.S);
    const int64_t at = row * parts + part;
    if (results) row_results(row, hit, scale, r, log_sum, out);
    else if (threadIdx.x == 0) ws.sums[at] = r;
    if constexpr (TOP) {
        largest_of_part<T, THREADS, false>(x, x, vocab, first, last, top, scan, sh, [&](int rank, uint64_t key) {
            if (parts > 1) {
                ws.key[at * top + rank] = key;
            } else {
                out.top_idx[row * top + rank] = index_of(key);
                out.top_logp[row * top + rank] = logp_of(value_of(static_cast<uint32_t>(key >> 32)), r, log_sum, scale);
            }
        });
    }
}

// A row's parts joined: every address is known from the start, so that there is one wait for memory and one for the target's
// logit.  Latency: 4 us for 64 rows of 4 parts with 8 alternatives each.
template <typename T, bool TOP>
__global__ void __launch_bounds__(kThreads)
k_token_join(const T* logits, int64_t vocab, int64_t stride, float scale, const int64_t* target, TokenOut out, int top,
             int parts, Parts ws) {
    __shared__ uint64_t list[TOP ? kMaxParts * kMaxTop : 1];
    __shared__ int32_t n;
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x & 63;
    // every wavefront joins the sums for itself: a part a lane
    Sums p = {-INFINITY, 0.f, 0.f};
    uint64_t bound = 0, key = 0;
    const int keys = parts * top;
    const int64_t t = out.logp ? target[row] : -1;
    if (lane < parts) {
        p = ws.sums[row * parts + lane];
        // `top` values reach the last one of any part's list
        if (TOP) bound = ws.key[(row * parts + lane) * top + top - 1];
    }
    if (TOP && static_cast<int>(threadIdx.x) < keys) key = ws.key[row * keys + threadIdx.x];
    Target<T> hit;
    hit.load(logits + row * stride, vocab, t);
    Sums r;
    r.m = wave_max(p.m);
    const float d = p.m == r.m ? 0.f : (p.m - r.m) * scale * kLog2e, f = exp2_of(d);
    r.S = wave_sum(p.S * f);
    r.U = wave_sum(f * fmaf(p.S, fmaxf(d, kFar), p.U));
    const float log_sum = logf(r.S);
    if (threadIdx.x == 0) {
        row_results(row, hit, scale, r, log_sum, out);
        n = 0;
    }
    if constexpr (TOP) {
#pragma unroll
        for (int s = 32; s; s >>= 1) {
            const uint64_t other = __shfl_xor(bound, s);
            if (other > bound) bound = other;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < keys; i += kThreads) {
            if (i >= kThreads) key = ws.key[row * keys + i];
            if (key && key >= bound) list[atomicAdd(&n, 1)] = key;
        }
        __syncthreads();
        rank_list<kThreads>(list, n, top, [&](int rank, uint64_t best) {
            out.top_idx[row * top + rank] = index_of(best);
            out.top_logp[row * top + rank] = logp_of(value_of(static_cast<uint32_t>(best >> 32)), r, log_sum, scale);
        });
    }
}

// Gradient of a row's values: p (a + b max(l, far)), with what scale, g, h, entropy and the target make of a and b.
//   kLogs, from a log of p:   l = x mul - add = ln p, p = 2^(l log2(e)):       a = -scale (g + h H),               b = -scale h
//   kSums, from the sums:     l = x mul - add = log2 p + log2 s, p = 2^l / s:  a = -scale (g + h (H - ln s)) / s,  b = -scale h ln2 / s
//   kDiffs, from differences: l = (x - add) mul = ln p + ln S, p = e^l / S:    a = -scale (g + h (H - ln S)) / S,  b = -scale h / S
// (a value with no probability has p = 0, l = -inf and the gradient 0).  The target's value has hot = scale g more.
enum { kLogs, kSums, kDiffs };
struct PolicyRows {
    PolicyIn in;
    float* loss;
    PolicyTerms* terms;
};
struct RowGrad {
    float mul, add, a, b, hot;
    int32_t target;                  // -1: none
    bool empty;                      // the row has no probabilities, or a policy loss leaves it out: gradient 0

    __device__ __forceinline__ void coefficients(int64_t row, int64_t vocab, float scale, int64_t t, const float* g_logp,
                                                  const float* g_entropy) {
        target = t >= 0 && t < vocab ? static_cast<int32_t>(t) : -1;
        const float g = target >= 0 && g_logp ? g_logp[row] : 0.f;
        hot = scale * g;
        a = -hot;
        b = g_entropy ? -scale * g_entropy[row] : 0.f;
    }
    // the same from the policy loss of a row's token; writes: that thread leaves the loss and what sums are taken of.  True: the row is left out,
    // and its logits may be anything (0 times a NaN would not be 0)
    __device__ __forceinline__ bool coefficients(int64_t row, int64_t vocab, float scale, int64_t t, const PolicyRows& rows,
                                                 const PolicyRow& given, float logp, float entropy, bool writes) {
        target = t >= 0 && t < vocab ? static_cast<int32_t>(t) : -1;
        const PolicyToken token = policy_token(rows.in.h, given, logp, entropy, target >= 0);
        if (writes) {
            if (rows.loss) rows.loss[row] = token.loss;
            if (rows.terms) rows.terms[row] = PolicyTerms{token.loss, token.kl, token.cut, target >= 0 ? given.weight : 0.f};
        }
        hot = scale * token.g_logp;
        a = -hot;
        b = -scale * token.g_entropy;
        return left_out(target, given.weight);
    }
    static __device__ __forceinline__ bool left_out(int32_t target, float weight) { return target < 0 || weight == 0.f; }
    // ENTROPY: b is not 0
    template <int FROM, bool ENTROPY>
    __device__ __forceinline__ float of(float x) const {
        const float l = FROM == kDiffs ? (x - add) * mul : fmaf(x, mul, -add), p = exp2_of(FROM == kSums ? l : l * kLog2e);
        return ENTROPY ? p * fmaf(fmaxf(l, kFar), b, a) : p * a;
    }
};

// A row's gradient from its sums and differences to its largest value.
__device__ __forceinline__ void grad_from_diffs(RowGrad& g, const Sums& r, float log_sum, float scale) {
    const float H = log_sum - kLn2 * (r.U / r.S), one = 1.f / r.S;
    g.empty = r.m == -INFINITY && r.S == r.S;
    g.mul = scale;
    g.add = r.m;
    g.a = one * fmaf(g.b, H - log_sum, g.a);
    g.b *= one;
}

// What a row's gradient is computed from, with its sums at hand: relative to a binary32 number next to m k, for which s is S
// but for what that is off; where m k is 2^22 or more, so that it may be off by more than 1/4 (and s, a power of 2 of that, out of range
// soon), from differences to m itself: finite masks in a row that has nothing else, logits with a large offset.  True: the former.
__device__ __forceinline__ bool grad_from_sums(RowGrad& g, const Sums& r, float log_sum, float scale) {
    g.mul = scale * kLog2e;
    g.add = r.m * g.mul;
    if (!(fabsf(g.add) < 4194304.f)) {
        grad_from_diffs(g, r, log_sum, scale);
        return false;
    }
    const float H = log_sum - kLn2 * (r.U / r.S), s = r.S * exp2_of(fmaf(r.m, g.mul, -g.add)), one = 1.f / s;
    g.empty = r.m == -INFINITY && r.S == r.S;
    g.a = one * fmaf(g.b, H - logf(s), g.a);
    g.b *= one * kLn2;
    return true;
}

// pack q of a row with the values v
template <bool PAST, int FROM, bool ENTROPY, typename T, int P>
__device__ __forceinline__ void grad_pack(float (&v)[P], T* dx, int32_t vocab, int32_t q, const RowGrad& row) {
    const int32_t at = q * P;
#pragma unroll
    for (int e = 0; e < P; ++e) v[e] = row.template of<FROM, ENTROPY>(v[e]);
    // (none: -1 lies in no pack)
    if (static_cast<uint32_t>(row.target - at) < static_cast<uint32_t>(P))
#pragma unroll
        for (int e = 0; e < P; ++e) v[e] += at + e == row.target ? row.hot : 0.f;
    if (row.empty)
#pragma unroll
        for (int e = 0; e < P; ++e) v[e] = 0.f;
    if (at + P <= vocab) {
        store_pack<PAST>(dx + at, v);
    } else {
#pragma unroll
        for (int e = 0; e < P; ++e)
            if (at + e < vocab) dx[at + e] = static_cast<T>(v[e]);
    }
}

// packs [first, last) of a row
template <bool PAST, int FROM, bool ENTROPY, int THREADS, typename T>
__device__ __forceinline__ void grad_packs(const T* x, T* dx, int64_t vocab, int32_t first, int32_t last, const RowGrad& row) {
    constexpr int P = kPack<T>;
    for (int32_t q = first + static_cast<int32_t>(threadIdx.x); q < last; q += THREADS) {
        const int32_t at = q * P;
        float v[P];
        if (at + P <= vocab) load_pack<T, P>(x + at, v);
        else load_tail(x, at, vocab, v);
        grad_pack<PAST, FROM, ENTROPY>(v, dx, static_cast<int32_t>(vocab), q, row);
    }
}

// A row's sums by a workgroup, four packs a thread under way: with the gradient 4096 x 32001 f32 in 627 us, 1 x 262144 in 129 (187 and 7 where
// the lse will do).
template <typename T>
__device__ __forceinline__ Sums sums_of_row(const T* x, int64_t vocab, int32_t packs, float scale, float (&buf)[3][16]) {
    constexpr int P = kPack<T>;
    Sums r = {-INFINITY, 0.f, 0.f};
    const auto each = [&](auto f) {
#pragma unroll 4
        for (int32_t q = threadIdx.x; q < packs; q += kThreads) {
            float v[P];
            if ((static_cast<int64_t>(q) + 1) * P <= vocab) load_pack<T, P>(x + static_cast<int64_t>(q) * P, v);
            else load_tail(x, static_cast<int64_t>(q) * P, vocab, v);
#pragma unroll
            for (int e = 0; e < P; ++e) f(v[e]);
        }
    };
    each([&](float v) { r.m = fmaxf(r.m, v); });
    r.m = block_max<kThreads>(r.m, buf[0]);
    each([&](float v) {
        const float d = (v - r.m) * scale * kLog2e, e = exp2_of(d);
        r.S += e;
        r.U = fmaf(e, fmaxf(d, kFar), r.U);
    });
    block_add2<kThreads>(r.S, r.U, buf[1], buf[2]);
    return r;
}

// From here on a row's gradient is not taken from its lse, which in binary32 is off by up to 2^-24 of itself, and so is every p: up to here
// 1.5e-5 of p, but 1e-3 at 3e4 and all of it in a row of a finite mask alone.  One of the row's workgroups (another one from row to row, as
// neighbours of a launch are on different dies) sums it again and writes all of it, the others leave it alone (dlogits may be the logits).
constexpr float kFarLse = 256.f;

// The gradient that is asked for later: a pass over the logits, four packs a thread, many workgroups a row.  4096 x 32001 f32
// in 187 us, 1049 MB at 5.6 TB/s (a copy: 4.8): memory.  policy_weight: of a policy loss, whose rows of weight 0 or without a target are
// left out; null otherwise.
template <typename T, bool PAST>
__global__ void __launch_bounds__(kThreads)
k_token_grad(const T* logits, int64_t vocab, int64_t stride, float scale, const int64_t* target, const float* lse,
             const float* entropy, const float* g_logp, const float* g_entropy, const float* policy_weight, T* dlogits, int64_t d_stride,
             int pieces, int32_t packs) {
    const int64_t row = blockIdx.x / static_cast<unsigned>(pieces);
    const int32_t each = (packs + pieces - 1) / pieces, piece = static_cast<int32_t>(blockIdx.x % static_cast<unsigned>(pieces));
    const int32_t first = min(each * piece, packs);
    RowGrad r;
    r.coefficients(row, vocab, scale, target ? target[row] : -1, g_logp, g_entropy);
    r.mul = scale;
    r.add = lse[row];
    r.empty = r.add == -INFINITY || (policy_weight && RowGrad::left_out(r.target, policy_weight[row]));
    if (fabsf(r.add) >= kFarLse && !r.empty) {
        __shared__ float buf[3][16];
        if (piece != row % pieces) return;
        const Sums sums = sums_of_row(logits + row * stride, vocab, packs, scale, buf);
        grad_from_diffs(r, sums, logf(sums.S), scale);
        grad_packs<PAST, kDiffs, true, kThreads>(logits + row * stride, dlogits + row * d_stride, vocab, 0, packs, r);
        return;
    }
    if (g_entropy) {
        r.a = fmaf(r.b, entropy[row], r.a);
        grad_packs<PAST, kLogs, true, kThreads>(logits + row * stride, dlogits + row * d_stride, vocab, first, min(first + each, packs), r);
    } else {
        grad_packs<PAST, kLogs, false, kThreads>(logits + row * stride, dlogits + row * d_stride, vocab, first, min(first + each, packs), r);
    }
}

enum { kForward, kAlternatives, kLoss, kPolicy };

// A row held in registers by THREADS threads, up to ITEMS packs each: one read of it for everything.  All but the last EITHER
// packs of a thread there are.
template <typename T, int THREADS, int ITEMS>
struct HeldRow {
    static constexpr int P = kPack<T>, EITHER = THREADS == 64 ? 1 : 4;
    uint32_t word[ITEMS][4];
    int32_t packs;
    __device__ __forceinline__ static int32_t pack(int i) { return thread_of_row<THREADS>() + i * THREADS; }
    __device__ __forceinline__ bool has(int i) const { return i < ITEMS - EITHER || pack(i) < packs; }
    __device__ __forceinline__ void load(const T* x, int32_t vocab, int32_t n) {
        const int32_t t = thread_of_row<THREADS>(), whole = vocab / P;
        packs = n;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
            if (i < ITEMS - EITHER || pack(i) < whole) __builtin_memcpy(word[i], x + i * THREADS * P + t * P, 16);
        if (packs > whole && t == whole % THREADS) {         // the pack that the row ends in
            T v[P];
            uint32_t last[4];
#pragma unroll
            for (int e = 0; e < P; ++e) v[e] = whole * P + e < vocab ? x[whole * P + e] : static_cast<T>(-INFINITY);
            __builtin_memcpy(last, v, 16);
#pragma unroll
            for (int i = ITEMS - EITHER; i < ITEMS; ++i)
                if (pack(i) == whole) __builtin_memcpy(word[i], last, 16);
        }
    }
    // (The empty statement has the values made from the words each time: kept in binary32 they would take twice the registers,
    // and registers are rows of other workgroups.)
    __device__ __forceinline__ void values(int i, float (&v)[P]) const {
        T raw[P];
        uint32_t w[4] = {word[i][0], word[i][1], word[i][2], word[i][3]};
        asm volatile("" : "+v"(w[0]), "+v"(w[1]), "+v"(w[2]), "+v"(w[3]));
        __builtin_memcpy(raw, w, 16);
#pragma unroll
        for (int e = 0; e < P; ++e) v[e] = static_cast<float>(raw[e]);
    }
    // of every pack: which, its words, its values
    template <typename F>
    __device__ __forceinline__ void each(F f) const {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
            if (has(i)) {
                float v[P];
                values(i, v);
                f(pack(i), word[i], v);
            }
    }
    template <bool TOP>
    __device__ __forceinline__ void scan(Scan<T, TOP>& scan, float k) const {
        float top = -INFINITY, low = INFINITY;
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
            if (has(i)) {
                float v[P];
                values(i, v);
                scan.look(v, pack(i), top, low);
            }
        scan.raise(top, k);
        if (low > kPlain) add<false>(scan, k);
        else add<true>(scan, k);
    }
    template <bool GUARDED, bool TOP>
    __device__ __forceinline__ void add(Scan<T, TOP>& scan, float k) const {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i)
            if (has(i)) {
                float v[P];
                values(i, v);
                scan.template add<GUARDED>(v, k);
            }
    }
};

template <bool PAST, int FROM, bool ENTROPY, int THREADS, int ITEMS, typename T>
__device__ __forceinline__ void grad_held(const HeldRow<T, THREADS, ITEMS>& held, T* dx, int32_t vocab, const RowGrad& row) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
        if (held.has(i)) {
            float v[kPack<T>];
            held.values(i, v);
            grad_pack<PAST, FROM, ENTROPY>(v, dx, vocab, held.pack(i), row);
        }
}

// Loss and gradient: one read and one write of the logits.  8192 x 34000 bf16 in 205 us, 1114 MB at 5.4 TB/s, vector ALU 59 %
// busy: memory (from the stream and the caches, k_token_loss, 258).  Registers are what counts, as they are rows under way:
// 512 threads and 84 registers are three rows a CU, 1024 threads and 82 one (329 us).
// Alternatives: no second read.  64 x 131072 bf16, in 4 parts each, 15 us; 1 x 32768 f32 with 20 alternatives 10 us: a
// chain of the row's read (3), the sums (2) and five steps with a barrier each.
// A wavefront a short row: 16000 x 200 f32 in 9 us.
template <typename T, int MODE, int THREADS, int ITEMS, bool PAST>
__global__ void __launch_bounds__(THREADS == 64 ? kThreads : THREADS)
k_token_held(const T* logits, int64_t rows, int32_t vocab, int64_t stride, float scale, const int64_t* target, TokenOut out, int top,
             const float* g_logp, const float* g_entropy, T* dlogits, int64_t d_stride, int32_t packs, int parts, Parts ws, PolicyRows policy) {
    constexpr int ROWS = THREADS == 64 ? kThreads / 64 : 1, P = kPack<T>;
    __shared__ TokenShared<THREADS> shared[ROWS];
    int64_t row = static_cast<int64_t>(blockIdx.x) * ROWS + (THREADS == 64 ? threadIdx.x >> 6 : 0);
    if (row >= rows * parts) return;                  // (a wavefront: nothing waits for it)
    TokenShared<THREADS>& sh = shared[THREADS == 64 ? threadIdx.x >> 6 : 0];
    // of a row in parts its own part, as a row of that length
    int32_t first = 0;
    const int64_t place = row;
    if (MODE == kAlternatives && parts > 1) {
        const int64_t part = row % parts;
        row /= parts;
        first = part_begin(part, packs, parts);
        packs = part_begin(part + 1, packs, parts) - first;
        vocab = min(packs * P, vocab - first * P);
    }
    const bool results = parts == 1;
    const T* x = logits + row * stride + first * P;
    const int64_t t = MODE == kLoss || MODE == kPolicy || (out.logp && results) ? target[row] : -1;
    const PolicyRow given = MODE == kPolicy ? policy_row(policy.in, row) : PolicyRow{};       // (under way while the row is read)
    const float k = scale * kLog2e;
    HeldRow<T, THREADS, ITEMS> held;
    held.load(x, vocab, packs);
    Target<T> hit;
    hit.load(x, vocab, t);
    Scan<T, MODE == kAlternatives> scan;
    held.scan(scan, k);
    const Sums r = join_threads<T, MODE == kAlternatives, THREADS>(x, vocab, 0, packs, scale, k, sh, scan);
    const float log_sum = logf(r.S);
    if (thread_of_row<THREADS>() == 0) {
        if (results) row_results(row, hit, scale, r, log_sum, out);
        else ws.sums[place] = r;
    }
    if constexpr (MODE == kAlternatives) {
        largest_of_part<T, THREADS, true>(x, held, vocab, 0, packs, top, scan, sh, [&](int rank, uint64_t key) {
            if (results) {
                out.top_idx[row * top + rank] = index_of(key);
                out.top_logp[row * top + rank] = logp_of(value_of(static_cast<uint32_t>(key >> 32)), r, log_sum, scale);
            } else {
                // (the index counts down in the key; none is 0)
                ws.key[place * top + rank] = key ? key - static_cast<uint32_t>(first * P) : 0;
            }
        });
    }
    if constexpr (MODE == kLoss || MODE == kPolicy) {
        T* dx = dlogits + row * d_stride;
        RowGrad g;
        bool bonus, out_of_it = false;
        if constexpr (MODE == kPolicy) {
            out_of_it = g.coefficients(row, vocab, scale, t, policy, given, hit.counts ? logp_of(hit.x, r, log_sum, scale) : 0.f, entropy_of(r, log_sum),
                           thread_of_row<THREADS>() == 0);
            bonus = policy.in.h.entropy != 0.f;
        } else {
            g.coefficients(row, vocab, scale, t, g_logp, g_entropy);
            bonus = g_entropy;
        }
        const bool from_sums = grad_from_sums(g, r, log_sum, scale);
        g.empty |= out_of_it;
        if (!from_sums) grad_held<PAST, kDiffs, true, THREADS, ITEMS>(held, dx, vocab, g);
        else if (bonus) grad_held<PAST, kSums, true, THREADS, ITEMS>(held, dx, vocab, g);
        else grad_held<PAST, kSums, false, THREADS, ITEMS>(held, dx, vocab, g);
    }
}

// Forward and gradient of a row in one workgroup, for rows that no workgroup holds (more than 131 072 values of 16 bits, 65 536 of 32): the
// second read comes from the caches.  1024 x 131072 bf16 as this 137 us, held 120.
template <typename T, bool PAST, int MODE>
__global__ void __launch_bounds__(kThreads)
k_token_loss(const T* logits, int64_t vocab, int64_t stride, float scale, const int64_t* target, TokenOut out,
             const float* g_logp, const float* g_entropy, T* dlogits, int64_t d_stride, int32_t packs, PolicyRows policy) {
    __shared__ TokenShared<kThreads> sh;
    const int64_t row = blockIdx.x;
    const T* x = logits + row * stride;
    T* dx = dlogits + row * d_stride;
    const int64_t t = target[row];
    const PolicyRow given = MODE == kPolicy ? policy_row(policy.in, row) : PolicyRow{};
    const float k = scale * kLog2e;
    Scan<T, false> scan;
    scan_packs<T, false, kThreads>(x, vocab, 0, packs, k, scan);
    Target<T> hit;
    hit.load(x, vocab, t);
    const Sums r = join_threads<T, false, kThreads>(x, vocab, 0, packs, scale, k, sh, scan);
    const float log_sum = logf(r.S);
    if (threadIdx.x == 0) row_results(row, hit, scale, r, log_sum, out);
    __syncthreads();                                  // (dlogits may be the logits, whose target has been read)
    RowGrad g;
    bool bonus, out_of_it = false;
    if constexpr (MODE == kPolicy) {
        out_of_it = g.coefficients(row, vocab, scale, t, policy, given, hit.counts ? logp_of(hit.x, r, log_sum, scale) : 0.f, entropy_of(r, log_sum),
                       threadIdx.x == 0);
        bonus = policy.in.h.entropy != 0.f;
    } else {
        g.coefficients(row, vocab, scale, t, g_logp, g_entropy);
        bonus = g_entropy;
    }
    const bool from_sums = grad_from_sums(g, r, log_sum, scale);
    g.empty |= out_of_it;
    if (!from_sums) grad_packs<PAST, kDiffs, true, kThreads>(x, dx, vocab, 0, packs, g);
    else if (bonus) grad_packs<PAST, kSums, true, kThreads>(x, dx, vocab, 0, packs, g);
    else grad_packs<PAST, kSums, false, kThreads>(x, dx, vocab, 0, packs, g);
}

// ---------------------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------------------
// rows (or their parts) that are held in registers: threads a row and packs a thread (threads = 0: they are not)
struct Held {
    int threads, items;
};
// Rows (or parts) up to which each has 1024 threads.  A policy loss has 512 from a row a CU on, where two rounds of 1024 would be needed (us a call,
// 1024 / 512 threads: 257 x 32001 f32 22.2 / 18.0, 300 x 32001 23.3 / 19.1, 511 x 32001 29.7 / 23.9, 300 x 8200 10.0 / 8.4, 500 x 34000 bf16 22.3 / 17.9,
// 270 x 65000 f16 28.8 / 25.0, 300 x 60000 f32, which needs 1024, 36.5).  The plain loss would gain as much (300 x 32001 22.0 / 18.0); it has the bits
// that it always gave.
constexpr int64_t kFewHeldRows = 512, kFewPolicyRows = 257;
Held held(int64_t rows, int64_t vocab, int32_t fmt, int parts, int64_t few = kFewHeldRows) {
    const int32_t all = packs_of(vocab, fmt), packs = (all + parts - 1) / parts;
    if (packs <= 256 && parts == 1) return {64, (packs + 63) / 64};
    // as many threads as there are for few rows; for many as few as have the registers, so that more rows are under way
    for (const int threads : {256, 512, 1024}) {
        if (threads < 1024 && rows * parts < few) continue;
        const int items = (packs + 4 * threads - 1) / (4 * threads) * 4;
        // (a part that is a pack shorter still has all but the last four packs of every thread whole)
        if (parts > 1 && all / parts <= threads * (items - 4) + 1) return {0, 0};
        if (items <= (threads == 256 ? 8 : 16)) return {threads, items};
    }
    return {0, 0};
}
template <typename T, int MODE, int THREADS, int ITEMS>
int token_held_as(const TokenArgs& a, int parts) {
    constexpr bool GRAD = MODE == kLoss || MODE == kPolicy;
    const auto kernel = GRAD && past_caches(a.rows * a.vocab * sizeof(T)) ? k_token_held<T, MODE, THREADS, ITEMS, GRAD>
                                                                          : k_token_held<T, MODE, THREADS, ITEMS, false>;
    const int64_t grid = THREADS == 64 ? (a.rows + 3) / 4 : a.rows * parts;
    kernel<<<static_cast<unsigned>(grid), THREADS == 64 ? kThreads : THREADS, 0, a.stream>>>(
        static_cast<const T*>(a.logits), a.rows, static_cast<int32_t>(a.vocab), a.stride, a.scale, a.target, a.out, a.top, a.g_logp,
        a.g_entropy, static_cast<T*>(a.dlogits), a.d_stride, packs_of(a.vocab, a.fmt), parts,
        parts > 1 ? parts_in(a.ws, a.rows, parts, a.top) : Parts{},
        PolicyRows{a.policy, a.policy_out.loss, a.policy_terms});
    return launched();
}
template <typename T, int MODE>
int token_held(const TokenArgs& a, const Held& h, int parts) {
#define CS_CASE(THREADS, ITEMS) \
    case THREADS * 32 + ITEMS: return token_held_as<T, MODE, THREADS, ITEMS>(a, parts);
    switch (h.threads * 32 + h.items) {
        CS_CASE(64, 1) CS_CASE(64, 2) CS_CASE(64, 3) CS_CASE(64, 4)
    }
    if constexpr (MODE != kForward) switch (h.threads * 32 + h.items) {
        CS_CASE(256, 4) CS_CASE(256, 8) CS_CASE(512, 8) CS_CASE(512, 12) CS_CASE(512, 16)
        CS_CASE(1024, 4) CS_CASE(1024, 8) CS_CASE(1024, 12) CS_CASE(1024, 16)
    }
#undef CS_CASE
    return CS_EINVAL;
}

template <typename T, bool TOP>
int token_forward(const TokenArgs& a) {
    const int parts = parts_of(a.rows, a.vocab);
    const Held h = held(a.rows, a.vocab, a.fmt, parts);
    const T* x = static_cast<const T*>(a.logits);
    const Parts ws = parts > 1 ? parts_in(a.ws, a.rows, parts, a.top) : Parts{};
    // (without alternatives nothing is wanted of a row a second time: only rows of a wavefront are held)
    if (h.threads == 64 || (TOP && h.threads)) {
        if (int rc = token_held<T, TOP ? kAlternatives : kForward>(a, h, parts)) return rc;
    } else {
        const bool few = few_rows(a.rows);
        const auto kernel = few ? k_token<T, TOP, kFewThreads> : k_token<T, TOP, kThreads>;
        kernel<<<static_cast<unsigned>(a.rows * parts), few ? kFewThreads : kThreads, 0, a.stream>>>(
            x, a.vocab, a.stride, a.scale, a.target, a.out, a.top, parts, packs_of(a.vocab, a.fmt), ws);
        if (int rc = launched()) return rc;
    }
    if (parts == 1) return CS_OK;
    k_token_join<T, TOP><<<static_cast<unsigned>(a.rows), kThreads, 0, a.stream>>>(x, a.vocab, a.stride, a.scale, a.target,
                                                                                  a.out, a.top, parts, ws);
    return launched();
}
template <typename T>
int token_grad(const TokenArgs& a) {
    const int32_t packs = packs_of(a.vocab, a.fmt);
    const int64_t most = kTokenMaxRows / a.rows;
    int64_t pieces = (packs + 4 * kThreads - 1) / (4 * kThreads);
    if (pieces > most) pieces = most;
    const auto kernel = past_caches(a.rows * a.vocab * sizeof(T)) ? k_token_grad<T, true> : k_token_grad<T, false>;
    kernel<<<static_cast<unsigned>(a.rows * pieces), kThreads, 0, a.stream>>>(
        static_cast<const T*>(a.logits), a.vocab, a.stride, a.scale, a.target, a.lse, a.entropy, a.g_logp, a.g_entropy,
        a.policy.weight, static_cast<T*>(a.dlogits), a.d_stride, static_cast<int>(pieces), packs);
    return launched();
}
// (kPolicy: the sums too)
template <typename T, int MODE>
int token_loss(TokenArgs a) {
    const auto sums = [&] {
        if (MODE != kPolicy || !a.policy_terms) return static_cast<int>(CS_OK);
        return launch_policy_sums(a.policy_terms, a.rows, a.policy_out.sums, a.policy_out.partials, a.stream);
    };
    const Held h = held(a.rows, a.vocab, a.fmt, 1, MODE == kPolicy ? kFewPolicyRows : kFewHeldRows);
    if (h.threads && parts_of(a.rows, a.vocab) == 1) {
        if (int rc = token_held<T, MODE>(a, h, 1)) return rc;
        return sums();
    }
    if (few_rows(a.rows)) {
        if (int rc = token_forward<T, false>(a)) return rc;
        if (MODE == kPolicy) {
            if (a.policy.h.entropy == 0.f) a.policy_out.g_entropy = nullptr;
            if (int rc = launch_policy(a.policy, a.rows, a.out.logp, a.out.entropy, a.target, a.vocab, a.policy_out, a.stream)) return rc;
            a.g_logp = a.policy_out.g_logp, a.g_entropy = a.policy_out.g_entropy;
        }
        a.lse = a.out.lse, a.entropy = a.out.entropy;
        return token_grad<T>(a);
    }
    const auto kernel = past_caches(a.rows * a.vocab * sizeof(T)) ? k_token_loss<T, true, MODE> : k_token_loss<T, false, MODE>;
    kernel<<<static_cast<unsigned>(a.rows), kThreads, 0, a.stream>>>(
        static_cast<const T*>(a.logits), a.vocab, a.stride, a.scale, a.target, a.out, a.g_logp, a.g_entropy,
        static_cast<T*>(a.dlogits), a.d_stride, packs_of(a.vocab, a.fmt),
        PolicyRows{a.policy, a.policy_out.loss, a.policy_terms});
    if (int rc = launched()) return rc;
    return sums();
}

template <typename T>
int token(TokenCall call, const TokenArgs& a) {
    if (call == kTokenForward) return a.top ? token_forward<T, true>(a) : token_forward<T, false>(a);
    if (call == kTokenPolicy) return token_loss<T, kPolicy>(a);
    return call == kTokenGrad ? token_grad<T>(a) : token_loss<T, kLoss>(a);
}

}  // namespace
}  // namespace cs

// Losses of answers from their tokens' log probabilities, with the gradients: the clipped policy loss, and the loss of pairs.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "cs_policy.h"
#include "cs_rows.h"
#include "csketch.h"

namespace cs {
namespace {

constexpr int kMost = 1024;                  // threads of a workgroup

// Sums of N binary64 numbers over a workgroup, in a fixed order; the first wavefront has them
template <int N>
__device__ __forceinline__ void workgroup_sums(double (&v)[N], double (&buf)[N][kMost / 64]) {
    const int lane = threadIdx.x & 63, waves = blockDim.x / 64;
#pragma unroll
    for (int k = 0; k < N; ++k) {
#pragma unroll
        for (int d = 32; d; d >>= 1) v[k] += __shfl_xor(v[k], d);
        if (lane == 0) buf[k][threadIdx.x >> 6] = v[k];
    }
    __syncthreads();
    if (threadIdx.x >= 64) return;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        v[k] = lane < waves ? buf[k][lane] : 0.;
#pragma unroll
        for (int d = kMost / 128; d; d >>= 1) v[k] += __shfl_xor(v[k], d);
    }
}

// A token a thread and turn; partials (one workgroup: the sums themselves) by workgroup
__global__ void __launch_bounds__(kMost)
k_policy(PolicyIn in, int64_t rows, const float* logp, const float* entropy, const int64_t* target, int64_t vocab, PolicyOut out) {
    __shared__ double buf[4][kMost / 64];
    double sums[4] = {0., 0., 0., 0.};
    const int64_t step = static_cast<int64_t>(gridDim.x) * blockDim.x;
    for (int64_t row = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; row < rows; row += step) {
        const int64_t at = target ? target[row] : 0;
        const bool counts = !target || (at >= 0 && at < vocab);
        const PolicyRow given = policy_row(in, row);
        const PolicyToken t = policy_token(in.h, given, logp[row], in.h.entropy != 0.f ? entropy[row] : 0.f, counts);
        if (out.loss) out.loss[row] = t.loss;
        if (out.g_logp) out.g_logp[row] = t.g_logp;
        if (out.g_entropy) out.g_entropy[row] = t.g_entropy;
        sums[0] += t.loss, sums[1] += t.kl, sums[2] += t.cut, sums[3] += counts ? given.weight : 0.f;
    }
    if (!out.sums) return;
    workgroup_sums(sums, buf);
    if (threadIdx.x == 0)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (gridDim.x == 1) out.sums[k] = static_cast<float>(sums[k]);
            else out.partials[blockIdx.x * 4 + k] = sums[k];
        }
}
constexpr int kAtOnce = 8;                   // loads of a thread that are under way together, where few threads wait for them
__global__ void __launch_bounds__(kMost) k_policy_sums(const PolicyTerms* terms, int64_t rows, float* out, double* partials) {
    __shared__ double buf[4][kMost / 64];
    double sums[4] = {0., 0., 0., 0.};
    const int64_t step = static_cast<int64_t>(gridDim.x) * blockDim.x;
    for (int64_t row = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; row < rows; row += kAtOnce * step) {
        PolicyTerms t[kAtOnce];
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) t[i] = row + i * step < rows ? terms[row + i * step] : PolicyTerms{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < kAtOnce; ++i) sums[0] += t[i].loss, sums[1] += t[i].kl, sums[2] += t[i].cut, sums[3] += t[i].weight;
    }
    workgroup_sums(sums, buf);
    if (threadIdx.x == 0)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (gridDim.x == 1) out[k] = static_cast<float>(sums[k]);
            else partials[blockIdx.x * 4 + k] = sums[k];
        }
}
template <int N>
__global__ void __launch_bounds__(kMost) k_join_sums(const double* partials, int count, float* sums) {
    __shared__ double buf[N][kMost / 64];
    double v[N] = {};
    for (int i = threadIdx.x; i < count; i += blockDim.x)
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += partials[i * N + k];
    workgroup_sums(v, buf);
    if (threadIdx.x == 0)
#pragma unroll
        for (int k = 0; k < N; ++k) sums[k] = static_cast<float>(v[k]);
}

// What a batch of nothing leaves: sums of 0, and no token has a gradient
__global__ void __launch_bounds__(kMost) k_nothing(float* sums, int count, float* g, int64_t tokens) {
    const int64_t first = static_cast<int64_t>(blockIdx.x) * kMost + threadIdx.x;
    if (sums && first < count) sums[first] = 0.f;
    for (int64_t i = first; i < tokens; i += static_cast<int64_t>(gridDim.x) * kMost) g[i] = 0.f;
}

// One workgroup is a launch less (5000 tokens 7.6 us, in five 10.1), but slower than many from about 8000 tokens on (10 000: 11.5 and 10.1).
int policy_grid(int64_t rows) {
    const int64_t grid = (rows + kMost - 1) / kMost;
    return static_cast<int>(grid <= 8 ? 1 : grid < 256 ? grid : 256);
}

// ---------------------------------------------------------------------------------------
// pairs of answers
// ---------------------------------------------------------------------------------------
// Answers have very different lengths, so work goes by pieces of kPiece tokens, whatever answers they belong to: one launch for the sums of each
// answer's part of each piece, one that joins an answer's parts and takes the loss of every pair, one that writes the gradients.  The part of answer a in
// piece t is number a + t: along the tokens either a or t goes up by 1, so no two are the same.
constexpr int kPieceThreads = 256, kEach = 8, kPiece = kPieceThreads * kEach;
constexpr int kPairsEach = 4;                // pairs of a workgroup, a wavefront each

// a token's log ratio: equal infinities are 0 apart (a token that neither allows), as in the policy loss
__device__ __forceinline__ double log_ratio(float l, float l1) { return l == l1 ? 0. : static_cast<double>(l) - static_cast<double>(l1); }

struct Part {
    double sum;
    int64_t count;
};
struct Preference {
    cs_preference h;
    int64_t tokens, pairs, pieces;
    const float *logp, *ref_logp;
    const uint8_t* counts;
    const int64_t* begin;
    const float* weight;
    float *loss, *reward, *g_logp, *sums;
    // workspace
    Part* parts;                             // 2 pairs + pieces
    double* partials;                        // of 4 pairs each, 3
    int32_t* first;                          // of every piece: the answer that its first token belongs to
    float* slope;                            // of every answer's tokens
};
__device__ __forceinline__ int64_t begin_of(const Preference& k, int64_t answer) {
    return min(max(k.begin[answer], static_cast<int64_t>(0)), k.tokens);
}

// The last answer (2 pairs: behind the last, -1: before the first) that begins at or before token `at`: 256 of the rest are looked at at a time.
__device__ __forceinline__ int64_t answer_at(const Preference& k, int64_t at) {
    int64_t lo = -1, hi = 2 * k.pairs + 1;   // it is in [lo, hi)
    while (hi - lo > 1) {
        const int64_t step = (hi - lo - 1 + kPieceThreads - 1) / kPieceThreads, mine = lo + step * (threadIdx.x + 1);
        const int n = __syncthreads_count(mine < hi && begin_of(k, mine) <= at);
        hi = min(hi, lo + step * (n + 1));
        lo += step * n;
    }
    return lo;
}
// Which answer begins at each of a piece's tokens, as a number from `first` on (0: none); begins in (at, at + kPiece)
__device__ __forceinline__ void mark_begins(const Preference& k, int64_t at, int64_t first, int32_t (&mark)[kPiece]) {
#pragma unroll
    for (int i = 0; i < kPiece; i += kPieceThreads) mark[i + threadIdx.x] = 0;
    __syncthreads();
    for (int64_t a = first + 1;; a += kPieceThreads) {
        const int64_t mine = a + threadIdx.x;
        bool in = false;
        if (mine <= 2 * k.pairs) {
            const int64_t b = begin_of(k, mine) - at;
            in = b < kPiece;
            // (of answers that begin at the same token the last one has it, the others are empty)
            if (in && b > 0) atomicMax(&mark[b], static_cast<int32_t>(mine - first));
        }
        if (!__syncthreads_and(in)) break;
    }
}

// What lies before a thread's tokens: the answer, and its sums in this piece
struct Run {
    int32_t answer;                          // from the first one of the piece on; 0: no other begins
    int32_t count;
    double sum;
};
__device__ __forceinline__ Run after(const Run& left, const Run& right) {
    return right.answer ? right : Run{left.answer, left.count + right.count, left.sum + right.sum};
}
__device__ __forceinline__ Run before_me(Run r, Run (&buf)[kPieceThreads / 64]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const Run left = {__shfl_up(r.answer, d), __shfl_up(r.count, d), __shfl_up(r.sum, d)};
        if (lane >= d) r = after(left, r);
    }
    if (lane == 63) buf[wave] = r;
    __syncthreads();
    Run all = {0, 0, 0.};
    for (int w = 0; w < wave; ++w) all = after(all, buf[w]);
    const Run left = {__shfl_up(r.answer, 1), __shfl_up(r.count, 1), __shfl_up(r.sum, 1)};
    return lane ? after(all, left) : all;
}

// kEach neighbouring values, 0 behind the last
template <typename T>
__device__ __forceinline__ void load_each(const T* p, int64_t at, int64_t n, T (&v)[kEach]) {
    if (at + kEach <= n) {
        __builtin_memcpy(v, p + at, sizeof(v));
    } else {
#pragma unroll
        for (int e = 0; e < kEach; ++e) v[e] = at + e < n ? p[at + e] : T(0);
    }
}

__global__ void __launch_bounds__(kPieceThreads) k_preference_parts(Preference k) {
    __shared__ int32_t mark[kPiece];
    __shared__ Run buf[kPieceThreads / 64];
    const int64_t at = static_cast<int64_t>(blockIdx.x) * kPiece;
    const int mine = threadIdx.x * kEach;
    float l[kEach], l1[kEach] = {};
    uint8_t counts[kEach];
    load_each(k.logp, at + mine, k.tokens, l);
    if (k.ref_logp) load_each(k.ref_logp, at + mine, k.tokens, l1);
#pragma unroll
    for (int e = 0; e < kEach; ++e) counts[e] = 1;
    if (k.counts) load_each(k.counts, at + mine, k.tokens, counts);
    const int64_t first = answer_at(k, at);
    if (threadIdx.x == 0) k.first[blockIdx.x] = static_cast<int32_t>(first);
    mark_begins(k, at, first, mark);
    double v[kEach];
    Run own = {0, 0, 0.};
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        v[e] = counts[e] ? log_ratio(l[e], l1[e]) : 0.;
        const Run one = {mark[mine + e], counts[e] != 0, v[e]};
        own = after(own, one);
    }
    Run r = before_me(own, buf);
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        if (mark[mine + e]) r = Run{mark[mine + e], 0, 0.};
        r.sum += v[e];
        r.count += counts[e] != 0;
        const bool last = mine + e + 1 == kPiece || at + mine + e + 1 == k.tokens || mark[min(mine + e + 1, kPiece - 1)];
        const int64_t answer = first + r.answer;
        if (last && answer >= 0 && answer < 2 * k.pairs && at + mine + e < k.tokens)
            k.parts[answer + blockIdx.x] = Part{r.sum, r.count};
    }
}

// loss and its slope at z
__device__ __forceinline__ void pair_loss(const cs_preference& h, double z, double& loss, double& slope) {
    if (h.kind == CS_PREFERENCE_LOGISTIC) {
        // ln(1 + e^-z) = max(-z, 0) + ln(1 + e^-|z|), and z more for the other answer
        const double e = exp(-fabs(z)), soft = log1p(e), p = (z >= 0. ? e : 1.) / (1. + e);        // p = 1 / (1 + e^z)
        const double s = h.smoothing;
        // (an answer that cannot be makes z infinite: what has no share in the loss adds 0, not 0 times that)
        loss = (s == 1. ? 0. : (1. - s) * (fmax(-z, 0.) + soft)) + (s == 0. ? 0. : s * (fmax(z, 0.) + soft));
        slope = s - p;
        if (!(z == z)) loss = z;             // (a maximum drops a NaN)
    } else if (h.kind == CS_PREFERENCE_HINGE) {
        loss = z < 1. ? 1. - z : z == z ? 0. : z;
        slope = z < 1. ? -1. : z == z ? 0. : z;
    } else {
        const double d = (z - 0.5) / h.beta;
        loss = d * d;
        slope = 2. * d / h.beta;
    }
}

// A pair from its answers' sums, each in one half of a wavefront: results, what the sums over the pairs get (in every lane), and the gradient of
// the lane's answer's tokens
__device__ __forceinline__ float finish_pair(const Preference& k, int64_t pair, double sum, double count, double (&out)[3]) {
    const int lane = threadIdx.x & 63, side = lane >> 5;
    const double each = k.h.beta / (k.h.mean ? fmax(count, 1.) : 1.), mine = each * sum, other = __shfl_xor(mine, 32);
    const double better = side ? other : mine, worse = side ? mine : other;
    double loss, slope;
    pair_loss(k.h, better - worse - k.h.margin, loss, slope);
    const double w = k.weight ? static_cast<double>(k.weight[pair]) : 1.;
    if ((lane & 31) == 0) k.reward[pair + side * k.pairs] = static_cast<float>(mine);
    if (lane == 0) k.loss[pair] = static_cast<float>(loss);
    out[0] += w == 0. ? 0. : w * loss;
    out[1] += better > worse ? w : 0.;
    out[2] += w == 0. ? 0. : w * (better - worse);
    return w == 0. ? 0.f : static_cast<float>((side ? -w : w) * slope * each);
}

// A pair a wavefront
__global__ void __launch_bounds__(kPairsEach * 64) k_preference_pairs(Preference k) {
    __shared__ double buf[3][kPairsEach];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, side = lane >> 5;
    const int64_t pair = static_cast<int64_t>(blockIdx.x) * kPairsEach + wave;
    double out[3] = {0., 0., 0.};
    if (pair < k.pairs) {
        const int64_t answer = pair + side * k.pairs, begin = begin_of(k, answer), end = begin_of(k, answer + 1);
        double sum = 0., count = 0.;
        if (end > begin)
            for (int64_t t = begin / kPiece + (lane & 31); t <= (end - 1) / kPiece; t += 32) {
                const Part p = k.parts[answer + t];
                sum += p.sum;
                count += static_cast<double>(p.count);
            }
#pragma unroll
        for (int d = 16; d; d >>= 1) {
            sum += __shfl_xor(sum, d);
            count += __shfl_xor(count, d);
        }
        const float slope = finish_pair(k, pair, sum, count, out);
        if ((lane & 31) == 0) k.slope[answer] = slope;
    }
    if (lane == 0)
#pragma unroll
        for (int i = 0; i < 3; ++i) buf[i][wave] = out[i];
    __syncthreads();
    if (threadIdx.x < 3) {
        double all = 0.;
        for (int w = 0; w < kPairsEach; ++w) all += buf[threadIdx.x][w];
        k.partials[blockIdx.x * 3 + threadIdx.x] = all;
    }
}

// Few pairs of few tokens in one launch, a pair a wavefront and turn, eight tokens of a lane under way together (16 pairs of up to 400 tokens: 13.4 us in
// pieces, 9.0 with a token after the other, 7.8)
constexpr int64_t kFewPairs = 32, kFewTokens = 8192;
__global__ void __launch_bounds__(kMost) k_preference_few(Preference k) {
    __shared__ double buf[3][kMost / 64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, side = lane >> 5;
    double out[3] = {0., 0., 0.};
    for (int64_t pair = wave; pair < k.pairs; pair += kMost / 64) {
        int64_t begin[2], end[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            begin[s] = begin_of(k, pair + s * k.pairs);
            end[s] = begin_of(k, pair + s * k.pairs + 1);
        }
        double sum[2] = {0., 0.}, count[2] = {0., 0.};
#pragma unroll
        for (int s = 0; s < 2; ++s)
            for (int64_t i = begin[s] + lane; i < end[s]; i += 64 * kAtOnce) {
                float l[kAtOnce], l1[kAtOnce];
                uint8_t counts[kAtOnce];
#pragma unroll
                for (int e = 0; e < kAtOnce; ++e) {
                    const int64_t at = i + 64 * e;
                    counts[e] = at < end[s];
                    l[e] = l1[e] = 0.f;
                    if (!counts[e]) continue;
                    l[e] = k.logp[at];
                    if (k.ref_logp) l1[e] = k.ref_logp[at];
                    if (k.counts) counts[e] = k.counts[at];
                }
#pragma unroll
                for (int e = 0; e < kAtOnce; ++e) {
                    sum[s] += counts[e] ? log_ratio(l[e], l1[e]) : 0.;
                    count[s] += counts[e] != 0;
                }
            }
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int d = 32; d; d >>= 1) {
                sum[s] += __shfl_xor(sum[s], d);
                count[s] += __shfl_xor(count[s], d);
            }
        const float slope = finish_pair(k, pair, sum[side], count[side], out);
        if (!k.g_logp) continue;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const float g = __shfl(slope, s * 32);
            for (int64_t i = begin[s] + lane; i < end[s]; i += 64) k.g_logp[i] = !k.counts || k.counts[i] ? g : 0.f;
        }
    }
    if (k.g_logp) {                          // tokens of no answer
        const int64_t first = begin_of(k, 0), last = begin_of(k, 2 * k.pairs);
        for (int64_t i = threadIdx.x; i < first; i += kMost) k.g_logp[i] = 0.f;
        for (int64_t i = last + threadIdx.x; i < k.tokens; i += kMost) k.g_logp[i] = 0.f;
    }
    if (lane == 0)
#pragma unroll
        for (int i = 0; i < 3; ++i) buf[i][wave] = out[i];
    __syncthreads();
    if (threadIdx.x < 3) {
        double all = 0.;
        for (int w = 0; w < kMost / 64; ++w) all += buf[threadIdx.x][w];
        k.sums[threadIdx.x] = static_cast<float>(all);
    }
}

// Gradients, a piece a workgroup; the last workgroup sums over the pairs
__global__ void __launch_bounds__(kPieceThreads) k_preference_gradient(Preference k, int groups) {
    if (blockIdx.x == gridDim.x - 1) {
        __shared__ double sums[3][kMost / 64];
        double v[3] = {0., 0., 0.};
        for (int i = threadIdx.x; i < groups; i += kPieceThreads)
#pragma unroll
            for (int e = 0; e < 3; ++e) v[e] += k.partials[i * 3 + e];
        workgroup_sums(v, sums);
        if (threadIdx.x == 0)
#pragma unroll
            for (int e = 0; e < 3; ++e) k.sums[e] = static_cast<float>(v[e]);
        return;
    }
    __shared__ int32_t mark[kPiece];
    __shared__ Run buf[kPieceThreads / 64];
    const int64_t at = static_cast<int64_t>(blockIdx.x) * kPiece, first = k.first[blockIdx.x];
    const int mine = threadIdx.x * kEach;
    uint8_t counts[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) counts[e] = 1;
    if (k.counts) load_each(k.counts, at + mine, k.tokens, counts);
    mark_begins(k, at, first, mark);
    Run own = {0, 0, 0.};
#pragma unroll
    for (int e = 0; e < kEach; ++e) own.answer = max(own.answer, mark[mine + e]);
    int64_t answer = first + before_me(own, buf).answer;
    float slope = answer >= 0 && answer < 2 * k.pairs ? k.slope[answer] : 0.f, g[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        if (mark[mine + e]) {
            answer = first + mark[mine + e];
            slope = answer < 2 * k.pairs ? k.slope[answer] : 0.f;
        }
        g[e] = counts[e] ? slope : 0.f;
    }
    float* const to = k.g_logp + at + mine;
    if (at + mine + kEach <= k.tokens) {
        __builtin_memcpy(to, g, sizeof(g));
    } else {
#pragma unroll
        for (int e = 0; e < kEach; ++e)
            if (at + mine + e < k.tokens) to[e] = g[e];
    }
}

// (pieces: workgroups of 256 threads of a launch, which has fewer than 2^32)
constexpr int64_t kMaxTokens = static_cast<int64_t>(1) << 40, kMaxPacked = static_cast<int64_t>(1) << 34, kMaxPairs = (static_cast<int64_t>(1) << 22) - 1;
int64_t pieces_of(int64_t tokens) { return (tokens + kPiece - 1) / kPiece; }
int64_t groups_of(int64_t pairs) { return (pairs + kPairsEach - 1) / kPairsEach; }
size_t preference_bytes(int64_t tokens, int64_t pairs) {
    const size_t pieces = static_cast<size_t>(pieces_of(tokens)), n = static_cast<size_t>(pairs);
    return pairs ? (2 * n + pieces) * sizeof(Part) + static_cast<size_t>(groups_of(pairs)) * 3 * sizeof(double) + pieces * 4 + 2 * n * 4 : 0;
}

}  // namespace

int policy_partials(int64_t rows) { return policy_grid(rows); }
bool policy_ok(const cs_policy* h) {
    const auto fine = [](float x) { return x >= 0.f && x < INFINITY; };
    return h && fine(h->clip_low) && h->clip_low <= 1.f && fine(h->clip_high) && fine(h->kl) && fabsf(h->entropy) < INFINITY;
}
int launch_policy(const PolicyIn& in, int64_t rows, const float* logp, const float* entropy, const int64_t* target, int64_t vocab,
                  const PolicyOut& out, hipStream_t stream) {
    const int grid = policy_grid(rows);
    const int64_t need = (rows + 63) / 64 * 64;
    k_policy<<<grid, static_cast<unsigned>(need < kMost ? need : kMost), 0, stream>>>(in, rows, logp, entropy, target, vocab, out);
    if (int rc = launched()) return rc;
    if (grid == 1 || !out.sums) return CS_OK;
    k_join_sums<4><<<1, 256, 0, stream>>>(out.partials, grid, out.sums);
    return launched();
}

int launch_nothing(float* sums, int count, float* g, int64_t tokens, hipStream_t stream) {
    const int64_t grid = tokens ? (tokens + kMost - 1) / kMost : 1;
    k_nothing<<<static_cast<unsigned>(grid < 1024 ? grid : 1024), kMost, 0, stream>>>(sums, count, g, tokens);
    return launched();
}

int launch_policy_sums(const PolicyTerms* terms, int64_t rows, float* sums, double* partials, hipStream_t stream) {
    const int grid = policy_grid(rows);
    const int64_t need = (rows + 63) / 64 * 64;
    k_policy_sums<<<grid, static_cast<unsigned>(need < kMost ? need : kMost), 0, stream>>>(terms, rows, sums, partials);
    if (int rc = launched()) return rc;
    if (grid == 1) return CS_OK;
    k_join_sums<4><<<1, 256, 0, stream>>>(partials, grid, sums);
    return launched();
}

}  // namespace cs

using namespace cs;

extern "C" int cs_policy_workspace_bytes(int64_t rows, size_t* bytes) {
    if (rows < 0 || rows > kMaxTokens || !bytes) return CS_EINVAL;
    *bytes = rows ? static_cast<size_t>(policy_partials(rows)) * 4 * sizeof(double) : 0;
    return CS_OK;
}

extern "C" int cs_policy_loss(const cs_policy* h, int64_t rows, const float* logp, const float* entropy, const float* old_logp,
                              const float* ref_logp, const float* advantage, const float* weight, float* loss, float* g_logp, float* g_entropy,
                              float* sums, void* workspace, size_t ws_bytes, void* stream) {
    if (!policy_ok(h) || rows < 0 || rows > kMaxTokens) return CS_EINVAL;
    if (rows == 0) return sums && workspace ? launch_nothing(sums, 4, nullptr, 0, stream_of(stream)) : CS_OK;
    if (!logp || !old_logp || !advantage || !weight || (h->kl != 0.f && !ref_logp) || (h->entropy != 0.f && !entropy)) return CS_EINVAL;
    const size_t need = static_cast<size_t>(policy_partials(rows)) * 4 * sizeof(double);
    if (ws_bytes < need) return CS_EWORKSPACE;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 7)) return CS_EINVAL;
    const Span written[] = {{loss, 4 * rows}, {g_logp, 4 * rows}, {g_entropy, 4 * rows}, {sums, 16}, {workspace, static_cast<int64_t>(need)}};
    const Span read[] = {{logp, 4 * rows}, {h->entropy != 0.f ? entropy : nullptr, 4 * rows}, {old_logp, 4 * rows},
                         {h->kl != 0.f ? ref_logp : nullptr, 4 * rows}, {advantage, 4 * rows}, {weight, 4 * rows}};
    if (!spans_apart(written, read)) return CS_EINVAL;
    return launch_policy(PolicyIn{*h, old_logp, ref_logp, advantage, weight}, rows, logp, entropy, nullptr, 0,
                         PolicyOut{loss, g_logp, g_entropy, sums, static_cast<double*>(workspace)}, stream_of(stream));
}

extern "C" int cs_preference_workspace_bytes(int64_t tokens, int64_t pairs, size_t* bytes) {
    if (tokens < 0 || tokens > kMaxPacked || pairs < 0 || pairs > kMaxPairs || !bytes) return CS_EINVAL;
    *bytes = preference_bytes(tokens, pairs);
    return CS_OK;
}

extern "C" int cs_preference_loss(const cs_preference* h, int64_t tokens, int64_t pairs, const float* logp, const float* ref_logp,
                                  const uint8_t* counts, const int64_t* begin, const float* weight, float* loss, float* reward,
                                  float* g_logp, float* sums, void* workspace, size_t ws_bytes, void* stream) {
    if (!h || h->kind < 0 || h->kind > CS_PREFERENCE_SQUARE || !(h->beta > 0.f && h->beta < INFINITY) || !(h->smoothing >= 0.f && h->smoothing <= 1.f) ||
        !(fabsf(h->margin) < INFINITY) || tokens < 0 || tokens > kMaxPacked || pairs < 0 || pairs > kMaxPairs)
        return CS_EINVAL;
    if (pairs == 0) {
        if (!workspace) return CS_OK;
        const Span nothing[] = {{g_logp, 4 * tokens}, {sums, 12}}, given[] = {{logp, 4 * tokens}, {ref_logp, 4 * tokens}, {counts, tokens}, {begin, 8}};
        if (!spans_apart(nothing, given)) return CS_EINVAL;
        return sums || (g_logp && tokens) ? launch_nothing(sums, 3, g_logp, g_logp ? tokens : 0, stream_of(stream)) : CS_OK;
    }
    if ((tokens && !logp) || !begin || !loss || !reward || !sums) return CS_EINVAL;
    const size_t need = preference_bytes(tokens, pairs);
    if (ws_bytes < need) return CS_EWORKSPACE;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 7)) return CS_EINVAL;
    const Span written[] = {{loss, 4 * pairs}, {reward, 8 * pairs}, {g_logp, 4 * tokens}, {sums, 12}, {workspace, static_cast<int64_t>(need)}};
    const Span read[] = {{logp, 4 * tokens}, {ref_logp, 4 * tokens}, {counts, tokens}, {begin, 8 * (2 * pairs + 1)}, {weight, 4 * pairs}};
    if (!spans_apart(written, read)) return CS_EINVAL;
    Preference k = {*h, tokens, pairs, pieces_of(tokens), logp, ref_logp, counts, begin, weight, loss, reward, g_logp, sums, nullptr, nullptr, nullptr, nullptr};
    const int64_t groups = groups_of(pairs);
    k.parts = static_cast<Part*>(workspace);
    k.partials = reinterpret_cast<double*>(k.parts + 2 * pairs + k.pieces);
    k.slope = reinterpret_cast<float*>(k.partials + groups * 3);
    k.first = reinterpret_cast<int32_t*>(k.slope + 2 * pairs);
    const hipStream_t s = stream_of(stream);
    if (pairs <= kFewPairs && tokens <= kFewTokens) {
        k_preference_few<<<1, kMost, 0, s>>>(k);
        return launched();
    }
    if (k.pieces) k_preference_parts<<<static_cast<unsigned>(k.pieces), kPieceThreads, 0, s>>>(k);
    k_preference_pairs<<<static_cast<unsigned>(groups), kPairsEach * 64, 0, s>>>(k);
    k_preference_gradient<<<static_cast<unsigned>((g_logp ? k.pieces : 0) + 1), kPieceThreads, 0, s>>>(k, static_cast<int>(groups));
    return launched();
}

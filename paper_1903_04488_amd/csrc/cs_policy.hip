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

// Sums of N binary64 numbers over a workgroup, in a fixed order; thread 0 has them
template <int N>
__device__ __forceinline__ void workgroup_sums(double (&v)[N], double (&buf)[N][kMost / 64]) {
#pragma unroll
    for (int k = 0; k < N; ++k) {
#pragma unroll
        for (int d = 32; d; d >>= 1) v[k] += __shfl_xor(v[k], d);
        if ((threadIdx.x & 63) == 0) buf[k][threadIdx.x >> 6] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < N; ++k) {
        v[k] = 0.;
        for (unsigned w = 0; w < blockDim.x / 64; ++w) v[k] += buf[k][w];
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
        const PolicyToken t = policy_token(in, row, logp[row], in.h.entropy != 0.f ? entropy[row] : 0.f, counts);
        if (out.loss) out.loss[row] = t.loss;
        if (out.g_logp) out.g_logp[row] = t.g_logp;
        if (out.g_entropy) out.g_entropy[row] = t.g_entropy;
        sums[0] += t.loss, sums[1] += t.kl, sums[2] += t.cut, sums[3] += counts ? in.weight[row] : 0.f;
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

int policy_grid(int64_t rows) {
    const int64_t grid = (rows + kMost - 1) / kMost;
    return static_cast<int>(grid < 8 ? 1 : grid < 256 ? grid : 256);
}

// ---------------------------------------------------------------------------------------
// pairs of answers
// ---------------------------------------------------------------------------------------
struct Preference {
    cs_preference h;
    int64_t tokens, pairs;
    const float *logp, *ref_logp;
    const uint8_t* counts;
    const int64_t* begin;
    const float* weight;
    float *loss, *reward, *g_logp;
    double* partials;                        // pairs x 3
};

// loss and its slope at z
__device__ __forceinline__ void pair_loss(const cs_preference& h, double z, double& loss, double& slope) {
    if (h.kind == CS_PREFERENCE_LOGISTIC) {
        // ln(1 + e^-z) = max(-z, 0) + ln(1 + e^-|z|), and z more for the other answer
        const double e = exp(-fabs(z)), soft = log1p(e), p = (z >= 0. ? e : 1.) / (1. + e);        // p = 1 / (1 + e^z)
        const double s = h.smoothing;
        loss = (1. - s) * (fmax(-z, 0.) + soft) + s * (fmax(z, 0.) + soft);
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

// tokens [first, last) of an answer, whatever the offsets say
__device__ __forceinline__ void answer_at(const Preference& k, int64_t answer, int64_t& first, int64_t& last) {
    first = min(max(k.begin[answer], static_cast<int64_t>(0)), k.tokens);
    last = min(max(k.begin[answer + 1], first), k.tokens);
}

// A pair a workgroup
__global__ void __launch_bounds__(kMost) k_preference(Preference k) {
    __shared__ double buf[4][kMost / 64];
    const int64_t pair = blockIdx.x;
    int64_t first[2], last[2];
    double v[4] = {0., 0., 0., 0.};          // sums, then how many count
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        answer_at(k, pair + side * k.pairs, first[side], last[side]);
        for (int64_t i = first[side] + threadIdx.x; i < last[side]; i += blockDim.x) {
            if (k.counts && !k.counts[i]) continue;
            v[side] += static_cast<double>(k.logp[i]) - (k.ref_logp ? static_cast<double>(k.ref_logp[i]) : 0.);
            v[2 + side] += 1.;
        }
    }
    workgroup_sums(v, buf);
    double each[2], reward[2], loss, slope;
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        each[side] = k.h.beta / (k.h.mean ? fmax(v[2 + side], 1.) : 1.);
        reward[side] = each[side] * v[side];
    }
    pair_loss(k.h, reward[0] - reward[1] - k.h.margin, loss, slope);
    const double w = k.weight ? static_cast<double>(k.weight[pair]) : 1.;
    if (threadIdx.x == 0) {
        k.loss[pair] = static_cast<float>(loss);
        k.reward[pair] = static_cast<float>(reward[0]);
        k.reward[pair + k.pairs] = static_cast<float>(reward[1]);
        k.partials[pair * 3] = w == 0. ? 0. : w * loss;
        k.partials[pair * 3 + 1] = reward[0] > reward[1] ? w : 0.;
        k.partials[pair * 3 + 2] = w == 0. ? 0. : w * (reward[0] - reward[1]);
    }
    if (!k.g_logp) return;
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        const float g = w == 0. ? 0.f : static_cast<float>((side ? -w : w) * slope * each[side]);
        for (int64_t i = first[side] + threadIdx.x; i < last[side]; i += blockDim.x) k.g_logp[i] = k.counts && !k.counts[i] ? 0.f : g;
    }
}

constexpr int64_t kMaxTokens = static_cast<int64_t>(1) << 40, kMaxPairs = (static_cast<int64_t>(1) << 22) - 1;
size_t preference_bytes(int64_t pairs) { return static_cast<size_t>(pairs) * 3 * sizeof(double); }

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
    if (rows == 0) return CS_OK;
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
    if (tokens < 0 || tokens > kMaxTokens || pairs < 0 || pairs > kMaxPairs || !bytes) return CS_EINVAL;
    *bytes = preference_bytes(pairs);
    return CS_OK;
}

extern "C" int cs_preference_loss(const cs_preference* h, int64_t tokens, int64_t pairs, const float* logp, const float* ref_logp,
                                  const uint8_t* counts, const int64_t* begin, const float* weight, float* loss, float* reward,
                                  float* g_logp, float* sums, void* workspace, size_t ws_bytes, void* stream) {
    if (!h || h->kind < 0 || h->kind > CS_PREFERENCE_SQUARE || !(h->beta > 0.f && h->beta < INFINITY) || !(h->smoothing >= 0.f && h->smoothing <= 1.f) ||
        !(fabsf(h->margin) < INFINITY) || tokens < 0 || tokens > kMaxTokens || pairs < 0 || pairs > kMaxPairs)
        return CS_EINVAL;
    if (pairs == 0) return CS_OK;
    if ((tokens && !logp) || !begin || !loss || !reward || !sums) return CS_EINVAL;
    const size_t need = preference_bytes(pairs);
    if (ws_bytes < need) return CS_EWORKSPACE;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 7)) return CS_EINVAL;
    const Span written[] = {{loss, 4 * pairs}, {reward, 8 * pairs}, {g_logp, 4 * tokens}, {sums, 12}, {workspace, static_cast<int64_t>(need)}};
    const Span read[] = {{logp, 4 * tokens}, {ref_logp, 4 * tokens}, {counts, tokens}, {begin, 8 * (2 * pairs + 1)}, {weight, 4 * pairs}};
    if (!spans_apart(written, read)) return CS_EINVAL;
    const Preference k = {*h, tokens, pairs, logp, ref_logp, counts, begin, weight, loss, reward, g_logp, static_cast<double*>(workspace)};
    const hipStream_t s = stream_of(stream);
    k_preference<<<static_cast<unsigned>(pairs), pairs < 256 ? kMost : 256, 0, s>>>(k);
    if (int rc = launched()) return rc;
    k_join_sums<3><<<1, kMost, 0, s>>>(static_cast<const double*>(workspace), static_cast<int>(pairs), sums);
    return launched();
}

// The clipped policy loss of one token, for the kernels that have log probabilities and for those that have logits.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "csketch.h"

namespace cs {

struct PolicyIn {
    cs_policy h;
    const float *old_logp, *ref_logp, *advantage, *weight;
};
struct PolicyToken {
    float loss, g_logp, g_entropy, kl, cut;  // loss, gradients and kl times the weight; cut: the weight where clipping decides
};

// a - b of log probabilities: equal infinities are 0 apart (a token that neither allows)
__device__ __forceinline__ float apart(float a, float b) { return a == b ? 0.f : a - b; }

// e^x - x - 1 without the cancellation near 0 (the ninth term is below 2^-28 of the first there)
__device__ __forceinline__ float beyond_line(float x) {
    if (fabsf(x) >= 0.5f) return expm1f(x) - x;
    float s = 1.f / 362880.f;
    s = fmaf(s, x, 1.f / 40320.f);
    s = fmaf(s, x, 1.f / 5040.f);
    s = fmaf(s, x, 1.f / 720.f);
    s = fmaf(s, x, 1.f / 120.f);
    s = fmaf(s, x, 1.f / 24.f);
    s = fmaf(s, x, 1.f / 6.f);
    s = fmaf(s, x, 0.5f);
    return s * x * x;
}

// A token of weight 0 is left out whatever its values are.  In binary32, as the log probabilities are: their own rounding, 2^-24 of them, mostly moves the
// ratio by more than all that is rounded here (777 tokens: 5.7e-8 of the whole off, in 64 bits and rounded once 2.8e-8).
__device__ __forceinline__ PolicyToken policy_token(const cs_policy& h, float logp, float entropy, float old_logp, float ref_logp, float a,
                                                    float w) {
    if (w == 0.f) return PolicyToken{0.f, 0.f, 0.f, 0.f, 0.f};
    const float r = expf(apart(logp, old_logp));
    // (a ratio beyond binary32 times no advantage is 0; one that is not a number stays one)
    const float plain = a == 0.f && r == r ? 0.f : r * a, bounded = fminf(fmaxf(r, 1.f - h.clip_low), 1.f + h.clip_high) * a;
    const bool cut = plain > bounded;        // (at the border the ratio still counts)
    PolicyToken t;
    float loss = -(cut ? bounded : plain), g = cut ? 0.f : -plain;
    t.kl = 0.f;
    if (h.kl != 0.f) {
        const float e = apart(ref_logp, logp), k = beyond_line(e);
        loss = fmaf(h.kl, k, loss);
        g = fmaf(-h.kl, expm1f(e), g);
        t.kl = w * k;
    }
    if (h.entropy != 0.f) loss = fmaf(-h.entropy, entropy, loss);
    t.loss = w * loss;
    t.g_logp = w * g;
    t.g_entropy = -h.entropy * w;
    t.cut = cut ? w : 0.f;
    return t;
}
// a row's inputs, and its token
struct PolicyRow {
    float old_logp, ref_logp, advantage, weight;
};
__device__ __forceinline__ PolicyRow policy_row(const PolicyIn& in, int64_t row) {
    return PolicyRow{in.old_logp[row], in.h.kl != 0.f ? in.ref_logp[row] : 0.f, in.advantage[row], in.weight[row]};
}
__device__ __forceinline__ PolicyToken policy_token(const cs_policy& h, const PolicyRow& row, float logp, float entropy, bool counts) {
    return policy_token(h, logp, entropy, row.old_logp, row.ref_logp, row.advantage, counts ? row.weight : 0.f);
}

// What sums are taken of, a row
struct PolicyTerms {
    float loss, kl, cut, weight;
};

// Losses (or null), gradients (or null) and sums (or null) of `rows` tokens; target and vocab say which rows have a token
// (target null: all).  partials: policy_partials(rows) x 4 binary64.
struct PolicyOut {
    float *loss, *g_logp, *g_entropy, *sums;
    double* partials;
};
int policy_partials(int64_t rows);
int launch_policy(const PolicyIn& in, int64_t rows, const float* logp, const float* entropy, const int64_t* target, int64_t vocab,
                  const PolicyOut& out, hipStream_t stream);
// The sums alone, of rows whose terms are known, in the same order
int launch_policy_sums(const PolicyTerms* terms, int64_t rows, float* sums, double* partials, hipStream_t stream);
// `count` sums (or null) and `tokens` gradients of nothing: 0
int launch_nothing(float* sums, int count, float* g, int64_t tokens, hipStream_t stream);
bool policy_ok(const cs_policy* h);

}  // namespace cs

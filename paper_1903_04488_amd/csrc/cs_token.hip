// The entry points of token log probabilities: checks of their arguments.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cs_rows.h"
#include "cs_token.h"
#include "csketch.h"

namespace cs {
namespace {

int by_type(TokenCall call, const TokenArgs& a) {
    return a.fmt == CS_FMT_F32 ? token_f32(call, a) : a.fmt == CS_FMT_BF16 ? token_bf16(call, a) : token_f16(call, a);
}

int64_t row_span(int64_t rows, int64_t vocab, int64_t stride, int32_t fmt) {
    return rows > 0 ? ((rows - 1) * stride + vocab) * fmt_bytes(fmt) : 0;
}
// dlogits may be the logits themselves, value for value, and must not meet them otherwise
bool dlogits_ok(const TokenArgs& a) {
    if (!a.dlogits || !rows_ok(a.rows, a.vocab, a.d_stride, a.fmt)) return false;
    if (a.dlogits == a.logits && (a.d_stride == a.stride || a.rows == 1)) return true;
    const int64_t b = fmt_bytes(a.fmt);
    return !rows_meet(a.dlogits, a.d_stride * b, a.logits, a.stride * b, a.rows, a.vocab * b);
}

// The parts of rows (a multiple of 8), then partial sums, then what sums are taken of, or for rows in parts the gradients of log probabilities
// and entropies, 16 bytes a row
size_t parts_bytes8(int64_t rows, int64_t vocab) { return (token_bytes(rows, vocab, 0) + 7) / 8 * 8; }
size_t policy_bytes(int64_t rows, int64_t vocab) {
    if (rows == 0) return 0;
    return parts_bytes8(rows, vocab) + static_cast<size_t>(policy_partials(rows)) * 4 * sizeof(double) + sizeof(PolicyTerms) * static_cast<size_t>(rows);
}

}  // namespace
}  // namespace cs

using namespace cs;

extern "C" int cs_token_workspace_bytes(int64_t rows, int64_t vocab, int32_t top, size_t* bytes) {
    if (rows < 0 || rows > kTokenMaxRows || vocab < 1 || vocab > kTokenMaxVocab || top < 0 || top > kMaxTop || top > vocab || !bytes)
        return CS_EINVAL;
    *bytes = token_bytes(rows, vocab, top);
    return CS_OK;
}

extern "C" int cs_token_logprobs(const void* logits, int64_t rows, int64_t vocab, int64_t stride, int32_t fmt, float scale,
                                 const int64_t* target, float* logp, float* entropy, float* lse, int32_t top,
                                 int64_t* top_idx, float* top_logp, void* workspace, size_t ws_bytes, void* stream) {
    if (!token_ok(rows, vocab, stride, fmt, scale) || top < 0 || top > kMaxTop || top > vocab) return CS_EINVAL;
    if ((logp && !target) || (top && (!top_idx || !top_logp))) return CS_EINVAL;
    if (rows == 0) return CS_OK;
    if (!logits) return CS_EINVAL;
    const size_t need = token_bytes(rows, vocab, top);
    if (ws_bytes < need) return CS_EWORKSPACE;
    if (need && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 7))) return CS_EINVAL;
    const Span written[] = {{logp, 4 * rows}, {entropy, 4 * rows}, {lse, 4 * rows}, {top ? top_idx : nullptr, 8 * rows * top},
                            {top ? top_logp : nullptr, 4 * rows * top}, {need ? workspace : nullptr, static_cast<int64_t>(need)}};
    const Span read[] = {{logits, row_span(rows, vocab, stride, fmt)}, {logp ? target : nullptr, 8 * rows}};
    if (!spans_apart(written, read)) return CS_EINVAL;
    TokenArgs a = {};
    a.logits = logits, a.rows = rows, a.vocab = vocab, a.stride = stride, a.fmt = fmt, a.scale = scale, a.target = target;
    a.out = TokenOut{logp, entropy, lse, top_idx, top_logp}, a.top = top, a.ws = workspace, a.stream = stream_of(stream);
    return by_type(kTokenForward, a);
}

extern "C" int cs_token_logprobs_grad(const void* logits, int64_t rows, int64_t vocab, int64_t stride, int32_t fmt,
                                      float scale, const int64_t* target, const float* lse, const float* entropy,
                                      const float* g_logp, const float* g_entropy, void* dlogits, int64_t d_stride,
                                      void* stream) {
    if (!token_ok(rows, vocab, stride, fmt, scale) || (g_logp && !target) || (g_entropy && !entropy)) return CS_EINVAL;
    if (rows == 0) return CS_OK;
    TokenArgs a = {};
    a.logits = logits, a.rows = rows, a.vocab = vocab, a.stride = stride, a.fmt = fmt, a.scale = scale, a.target = target;
    a.lse = lse, a.entropy = g_entropy ? entropy : nullptr, a.g_logp = g_logp, a.g_entropy = g_entropy;
    a.dlogits = dlogits, a.d_stride = d_stride, a.stream = stream_of(stream);
    if (!logits || !lse || !dlogits_ok(a)) return CS_EINVAL;
    const Span written[] = {{dlogits, row_span(rows, vocab, d_stride, fmt)}};
    const Span read[] = {{target, 8 * rows}, {lse, 4 * rows}, {a.entropy, 4 * rows}, {g_logp, 4 * rows}, {g_entropy, 4 * rows}};
    if (!spans_apart(written, read)) return CS_EINVAL;
    return by_type(kTokenGrad, a);
}

extern "C" int cs_token_loss(const void* logits, int64_t rows, int64_t vocab, int64_t stride, int32_t fmt, float scale,
                             const int64_t* target, const float* g_logp, const float* g_entropy, float* logp,
                             float* entropy, float* lse, void* dlogits, int64_t d_stride, void* workspace, size_t ws_bytes,
                             void* stream) {
    if (!token_ok(rows, vocab, stride, fmt, scale)) return CS_EINVAL;
    if (rows == 0) return CS_OK;
    if (!logits || !target || !g_logp || !logp || !entropy || !lse) return CS_EINVAL;
    const size_t need = token_bytes(rows, vocab, 0);
    if (ws_bytes < need) return CS_EWORKSPACE;
    if (need && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 7))) return CS_EINVAL;
    TokenArgs a = {};
    a.logits = logits, a.rows = rows, a.vocab = vocab, a.stride = stride, a.fmt = fmt, a.scale = scale, a.target = target;
    a.out = TokenOut{logp, entropy, lse, nullptr, nullptr}, a.ws = workspace, a.g_logp = g_logp, a.g_entropy = g_entropy;
    a.dlogits = dlogits, a.d_stride = d_stride, a.stream = stream_of(stream);
    if (!dlogits_ok(a)) return CS_EINVAL;
    const Span written[] = {{logp, 4 * rows}, {entropy, 4 * rows}, {lse, 4 * rows}, {need ? workspace : nullptr, static_cast<int64_t>(need)}};
    const Span read[] = {{logits, row_span(rows, vocab, stride, fmt)}, {dlogits, row_span(rows, vocab, d_stride, fmt)},
                         {target, 8 * rows}, {g_logp, 4 * rows}, {g_entropy, 4 * rows}};
    const Span grad[] = {{dlogits, row_span(rows, vocab, d_stride, fmt)}};
    const Span rest[] = {{target, 8 * rows}, {g_logp, 4 * rows}, {g_entropy, 4 * rows}};
    if (!spans_apart(written, read) || !spans_apart(grad, rest)) return CS_EINVAL;
    return by_type(kTokenLoss, a);
}

extern "C" int cs_token_policy_workspace_bytes(int64_t rows, int64_t vocab, size_t* bytes) {
    if (rows < 0 || rows > kTokenMaxRows || vocab < 1 || vocab > kTokenMaxVocab || !bytes) return CS_EINVAL;
    *bytes = policy_bytes(rows, vocab);
    return CS_OK;
}

extern "C" int cs_token_policy_loss(const cs_policy* h, const void* logits, int64_t rows, int64_t vocab, int64_t stride, int32_t fmt,
                                    float scale, const int64_t* target, const float* old_logp, const float* ref_logp,
                                    const float* advantage, const float* weight, float* logp, float* entropy, float* lse, float* loss,
                                    float* sums, void* dlogits, int64_t d_stride, void* workspace, size_t ws_bytes, void* stream) {
    if (!policy_ok(h) || !token_ok(rows, vocab, stride, fmt, scale)) return CS_EINVAL;
    if (rows == 0) return sums && workspace ? launch_nothing(sums, 4, nullptr, 0, stream_of(stream)) : CS_OK;
    if (!logits || !target || !old_logp || (h->kl != 0.f && !ref_logp) || !advantage || !weight || !logp || !entropy || !lse) return CS_EINVAL;
    const size_t need = policy_bytes(rows, vocab);
    if (ws_bytes < need) return CS_EWORKSPACE;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 7)) return CS_EINVAL;
    const float* const ref = h->kl != 0.f ? ref_logp : nullptr;
    TokenArgs a = {};
    a.logits = logits, a.rows = rows, a.vocab = vocab, a.stride = stride, a.fmt = fmt, a.scale = scale, a.target = target;
    a.out = TokenOut{logp, entropy, lse, nullptr, nullptr}, a.ws = workspace;
    a.dlogits = dlogits, a.d_stride = d_stride, a.stream = stream_of(stream);
    a.policy = PolicyIn{*h, old_logp, ref, advantage, weight};
    char* const more = static_cast<char*>(workspace) + parts_bytes8(rows, vocab);
    a.policy_out = PolicyOut{loss, nullptr, nullptr, sums, reinterpret_cast<double*>(more)};
    char* const terms = more + static_cast<size_t>(policy_partials(rows)) * 4 * sizeof(double);
    a.policy_terms = sums ? reinterpret_cast<PolicyTerms*>(terms) : nullptr;
    a.policy_out.g_logp = reinterpret_cast<float*>(terms), a.policy_out.g_entropy = a.policy_out.g_logp + rows;
    if (!dlogits_ok(a)) return CS_EINVAL;
    const int64_t n = 4 * rows, dlogits_span = row_span(rows, vocab, d_stride, fmt);
    const Span written[] = {{logp, n}, {entropy, n}, {lse, n}, {loss, n}, {sums, 16}, {workspace, static_cast<int64_t>(need)}};
    const Span read[] = {{logits, row_span(rows, vocab, stride, fmt)}, {dlogits, dlogits_span}, {target, 8 * rows}, {old_logp, n}, {ref, n},
                         {advantage, n}, {weight, n}};
    const Span grad[] = {{dlogits, dlogits_span}};
    const Span rest[] = {{target, 8 * rows}, {old_logp, n}, {ref, n}, {advantage, n}, {weight, n}};
    if (!spans_apart(written, read) || !spans_apart(grad, rest)) return CS_EINVAL;
    return by_type(kTokenPolicy, a);
}

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

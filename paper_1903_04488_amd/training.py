"""A language model's training step on both sides of its gradient: layer norm, the loss over the vocabulary, AdamW.

Like the paths of pipeline.py these classes own tensors and the order of the library calls; every arithmetic step
runs inside libcsketch.so.  What they return are their own buffers, which the next call overwrites.
"""
from __future__ import annotations

import warnings

import torch

from . import binding as B


class LayerNorm:
    """Layer norm of up to `rows` vectors, with what the backward pass needs.  weight, bias: [cols] tensors of the rows' type
    or float32; their gradients go into dweight and dbias (given, or of this object)."""

    def __init__(self, weight, bias, rows: int, dtype=torch.float32, eps: float = 1e-5, dweight=None, dbias=None):
        self.weight, self.bias, self.eps = weight, bias, eps
        cols, dev = weight.numel(), weight.device
        self.y, self.dx = (torch.empty(rows, cols, dtype=dtype, device=dev) for _ in range(2))
        self.mean, self.rstd = (torch.empty(rows, dtype=torch.float32, device=dev) for _ in range(2))
        self.dweight = torch.empty_like(weight) if dweight is None else dweight
        self.dbias = torch.empty_like(bias) if dbias is None and bias is not None else dbias
        # (no number of rows up to `rows` needs more)
        self.workspace = torch.empty(B.cs_layer_norm_grad_workspace_bytes(rows, cols), dtype=torch.uint8, device=dev)
        self.x = None

    def forward(self, x):
        n = len(x)
        B.cs_layer_norm(x, self.weight, self.bias, self.y[:n], self.mean[:n], self.rstd[:n], self.eps)
        self.x = x
        return self.y[:n]

    def backward(self, dy):
        """dx; fills dweight and dbias"""
        if self.x is None:
            raise B.CsError("backward before forward")
        n = len(self.x)
        B.cs_layer_norm_grad(dy, self.x, self.weight, self.mean[:n], self.rstd[:n], self.dx[:n], self.dweight, self.dbias,
                             self.workspace)
        return self.dx[:n]


class TokenLogprobs:
    """Log probabilities of tokens under up to `rows` rows of logits, entropy, `top` alternatives, and gradients."""

    def __init__(self, rows: int, vocab: int, top: int = 0, scale: float = 1.0, device="cuda:0"):
        self.rows, self.vocab, self.scale = rows, vocab, scale
        f32 = dict(dtype=torch.float32, device=device)
        self.logp, self.entropy, self.lse = (torch.empty(rows, **f32) for _ in range(3))
        self.top_idx = torch.empty(rows, top, dtype=torch.int64, device=device) if top else None
        self.top_logp = torch.empty(rows, top, **f32) if top else None
        # (fewer rows are shared by more workgroups each, and take up to this much)
        need = max(B.cs_token_workspace_bytes(n, vocab, top) for n in range(1, min(rows, 512) + 1)) if rows else 0
        self.workspace = torch.empty(need, dtype=torch.uint8, device=device)

    def forward(self, logits, target):
        """(logp, entropy); lse, top_idx and top_logp are in the attributes"""
        n = len(logits)
        top = (None, None) if self.top_idx is None else (self.top_idx[:n], self.top_logp[:n])
        B.cs_token_logprobs(logits, target, self.logp[:n], self.entropy[:n], self.lse[:n], *top, self.workspace, self.scale)
        return self.logp[:n], self.entropy[:n]

    def backward(self, logits, target, g_logp, g_entropy=None, out=None):
        """the gradient of sum g_logp logp + g_entropy entropy, after forward of the same rows; `out` may be logits"""
        n = len(logits)
        out = torch.empty_like(logits) if out is None else out
        B.cs_token_logprobs_grad(logits, target, self.lse[:n], self.entropy[:n], g_logp, g_entropy, out, self.scale)
        return out

    def loss(self, logits, target, g_logp, g_entropy=None, out=None):
        """forward and that gradient in one call; `out` may be logits"""
        n = len(logits)
        out = torch.empty_like(logits) if out is None else out
        B.cs_token_loss(logits, target, g_logp, g_entropy, self.logp[:n], self.entropy[:n], self.lse[:n], out,
                        self.workspace, self.scale)
        return self.logp[:n], out


class AdamW:
    """AdamW over all tensors of a model in one launch, its moments in 32 or in 8 bits.

    params, grads: lists of tensors, updated and read where they are (`set_grads` after grads have moved).  max_norm: the
    gradients are clipped to this global norm, and a step whose norm is not finite changes nothing and does not count.  m, v
    (m_exp, v_exp): moments of a checkpoint after `steps` steps, kept and updated in place.  seed: of the rounding to 8 bits, which
    without one (0) is to nearest and does not follow the gradients over many steps; an optimizer that begins with moments of its own
    has a seed, one that goes on with others is told theirs.  capturable: step number and learning
    rate live on the GPU (`lr_now`, float64), so that a graph of step() can be replayed.  The constants may be changed between
    steps: opt.h.lr = ...  `steps` is the number of steps that were taken (with max_norm or capturable it is read from the GPU,
    which waits)."""

    def __init__(self, params, grads, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.01,
                 max_norm: float | None = None, bits: int = 32, m=None, v=None, m_exp=None, v_exp=None, steps: int = 0,
                 capturable: bool = False, seed: int | None = None):
        if bits not in (8, 32):
            raise B.CsError(f"moments have 8 or 32 bits, not {bits}")
        if not params:
            raise B.CsError("params must be a non-empty list")
        self.params, self.grads = list(params), list(grads)
        if seed is None:
            seed = 1 if bits == 8 and m is None and v is None else 0
        if not 0 <= seed < 1 << 64:
            raise B.CsError(f"seed must be a number of 64 bits, not {seed}")
        if bits == 8 and not seed and betas[1] > 0.938:
            warnings.warn("moments in 8 bits that are rounded to nearest (seed 0) do not follow the gradients over many steps",
                          stacklevel=2)
        self.h = B.CsAdamw(lr, *betas, eps, weight_decay, seed)
        self.max_norm, self.bits, self._steps = max_norm, bits, steps
        self.device = self.params[0].device
        kind = torch.uint8 if bits == 8 else torch.float32

        def zeros():
            return [torch.zeros(x.shape, dtype=kind, device=self.device) for x in self.params]

        def exponents():
            return [torch.full((-(-x.numel() // B.CS_ADAMW_BLOCK),), 16, dtype=torch.uint8, device=self.device)
                    for x in self.params]

        self.m, self.v = zeros() if m is None else list(m), zeros() if v is None else list(v)
        self.m_exp = self.v_exp = None
        if bits == 8:
            self.m_exp = exponents() if m_exp is None else list(m_exp)
            self.v_exp = exponents() if v_exp is None else list(v_exp)
        self.list = B.TensorList(self.params, self.grads, self.m, self.v, self.m_exp, self.v_exp)
        self._norm_and_scale = self._workspace = self.norm = self._scale = None
        if max_norm is not None:
            self._norm_and_scale = torch.zeros(2, dtype=torch.float32, device=self.device)
            self.norm, self._scale = self._norm_and_scale[0], self._norm_and_scale[1:]
            self._workspace = torch.empty(B.cs_grad_norm_workspace_bytes(self.list), dtype=torch.uint8, device=self.device)
        self.step_now = self.lr_now = self.coefs = None
        if capturable or max_norm is not None:           # (the host does not see whether a norm is finite)
            self.step_now = torch.full((1,), steps, dtype=torch.int64, device=self.device)
            self.coefs = torch.zeros(B.CS_ADAMW_COEFS, dtype=torch.float32, device=self.device)
        if capturable:
            self.lr_now = torch.full((1,), lr, dtype=torch.float64, device=self.device)

    @property
    def steps(self):
        return self._steps if self.step_now is None else int(self.step_now)

    @steps.setter
    def steps(self, n):
        self._steps = n
        if self.step_now is not None:
            self.step_now.fill_(n)

    def set_grads(self, grads):
        """other tensors with the gradients"""
        grads = list(grads)
        self.list.refresh(self.params, grads, self.m, self.v, self.m_exp, self.v_exp)
        self.grads = grads

    def step(self):
        """one update of params and moments; `norm` (with max_norm) is the gradients' norm, on the GPU"""
        if self.max_norm is not None:
            B.cs_grad_norm_advance(self.list, self.max_norm, self._norm_and_scale, self._workspace, self.h, self.step_now, self.coefs,
                                   self.lr_now)
        elif self.coefs is not None:
            B.cs_adamw_advance(self.h, self.step_now, self.coefs, self.lr_now)
        B.cs_adamw_step(self.h, self._steps + 1, self.list, self.coefs, self._scale)
        if self.coefs is None:
            self._steps += 1


class MomentReader:
    """The values of an optimizer's moments in 8 bits: first moment and ROOT of the second, in bf16, exactly."""

    def __init__(self, optimizer: AdamW, m=None, root_v=None):
        if optimizer.bits != 8:
            raise B.CsError("the optimizer's moments are not in 8 bits")

        def like():
            return [torch.empty(x.shape, dtype=torch.bfloat16, device=x.device) for x in optimizer.params]

        self.m, self.root_v = like() if m is None else list(m), like() if root_v is None else list(root_v)
        self.list = B.TensorList(self.m, self.root_v, optimizer.m, optimizer.v, optimizer.m_exp, optimizer.v_exp)

    def read(self):
        B.cs_moments_read(self.list)
        return self.m, self.root_v


def write_moments(optimizer: AdamW, m, root_v):
    """Puts first moments and roots of second moments, float32, into an optimizer's moments in 8 bits."""
    if optimizer.bits != 8:
        raise B.CsError("the optimizer's moments are not in 8 bits")
    B.cs_moments_write(B.TensorList(m, root_v, optimizer.m, optimizer.v, optimizer.m_exp, optimizer.v_exp))


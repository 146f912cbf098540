"""The binding's two ways through its checks, for calls whose tensors are all plain and for others, give the same calls: results are
the same bits, and a tensor that is not what it should be is refused wherever it stands."""
import pytest
import torch

import paper_1903_04488_amd as cs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def strided(t):
    """the same values in rows that lie further apart (for vectors: the same tensor)"""
    if t is None or t.dim() != 2 or t.dtype == torch.int64 or t.shape[1] < 8:
        return t
    wide = torch.zeros(t.shape[0], t.shape[1] + 8, dtype=t.dtype, device=DEV)
    wide[:, : t.shape[1]] = t
    return wide[:, : t.shape[1]]


def calls():
    gen = torch.Generator(device=DEV).manual_seed(1)

    def normal(*shape):
        return torch.randn(*shape, device=DEV, generator=gen)

    rows, cols, vocab = 6, 96, 500
    x, dy, w, b = normal(rows, cols), normal(rows, cols), normal(cols), normal(cols)
    mean, rstd = x.mean(1), 1 / x.std(1)
    ws = torch.empty(cs.cs_layer_norm_grad_workspace_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    logits, target = normal(rows, vocab), torch.randint(0, vocab, (rows,), device=DEV, generator=gen)
    tws = torch.empty(cs.cs_token_workspace_bytes(rows, vocab, 3), dtype=torch.uint8, device=DEV)
    v = [torch.zeros(rows, device=DEV) for _ in range(8)]
    lse = torch.logsumexp(logits, 1)
    H = torch.distributions.Categorical(logits=logits).entropy()
    z = torch.zeros_like
    # (call, arguments, which of them are written)
    return {
        "norm": (cs.cs_layer_norm, [x, w, b, z(x), v[0], v[1]], [3, 4, 5]),
        "norm alone": (cs.cs_layer_norm, [x, w, b, z(x), None, None], [3]),
        "norm gradient": (cs.cs_layer_norm_grad, [dy, x, w, mean, rstd, z(x), z(w), z(b), ws], [5, 6, 7]),
        "token": (cs.cs_token_logprobs, [logits, target, v[0], v[1], v[2], torch.zeros(rows, 3, dtype=torch.int64, device=DEV),
                                         torch.zeros(rows, 3, device=DEV), tws], [2, 3, 4, 5, 6]),
        "token alone": (cs.cs_token_logprobs, [logits, target, v[0], v[1], v[2], None, None, tws], [2, 3, 4]),
        "token gradient": (cs.cs_token_logprobs_grad, [logits, target, lse, H, mean.clone(), rstd.clone(), z(logits)], [6]),
        "loss": (cs.cs_token_loss, [logits, target, mean.clone(), None, v[3], v[4], v[5], z(logits), tws], [4, 5, 6, 7]),
        "loss with entropy": (cs.cs_token_loss, [logits, target, mean.clone(), rstd.clone(), v[3], v[4], v[5], z(logits), tws], [4, 5, 6, 7]),
    }


NAMES = ["norm", "norm alone", "norm gradient", "token", "token alone", "token gradient", "loss", "loss with entropy"]


@pytest.mark.parametrize("name", NAMES)
def test_plain_and_strided_tensors_give_the_same_bits(name):
    f, args, written = calls()[name]
    f(*args)
    plain = [args[i].clone() for i in written]
    apart = [strided(a) if isinstance(a, torch.Tensor) else a for a in args]
    for i in written:
        apart[i].zero_()
    f(*apart)
    assert all(torch.equal(apart[i], p) for i, p in zip(written, plain))


@pytest.mark.parametrize("name", NAMES)
def test_every_argument_is_checked(name):
    f, args, _ = calls()[name]
    for i, a in enumerate(args):
        if a is None:
            continue
        wrong = [a.cpu(), a.to(torch.float64), a[:-1], a.reshape(-1)[::2], 7]
        for bad in wrong:
            if a.dtype == torch.uint8 and isinstance(bad, torch.Tensor) and bad.dtype == torch.uint8 and bad.is_cuda:
                continue                                # (a workspace may have any size that is enough)
            with pytest.raises(cs.CsError):
                f(*args[:i], bad, *args[i + 1:])

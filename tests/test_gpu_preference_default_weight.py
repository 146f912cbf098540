"""The loss of pairs as an object, without a weight: a mean over the pairs, whatever torch makes tensors of by default."""
import pytest
import torch

from paper_1903_04488_amd.training import PreferenceLoss

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def batch(pairs, seed=1):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    begin = torch.arange(0, 10 * pairs + 1, 5, device=DEV)
    return -torch.rand(10 * pairs, device=DEV, generator=gen), -torch.rand(10 * pairs, device=DEV, generator=gen), begin


@pytest.mark.parametrize("pairs", [1, 3, 7, 64])
def test_a_mean_over_the_pairs_of_the_call(pairs):
    pl = PreferenceLoss(640, 64, beta=0.5)
    for n in (pairs, 64, pairs):                         # (fewer than there is room for, all, fewer again)
        logp, ref, begin = batch(n, seed=n)
        got = [x.clone() for x in pl.loss(logp, ref, begin)]
        want = pl.loss(logp, ref, begin, weight=torch.full((n,), 1.0 / n, device=DEV, dtype=torch.float32))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and got[1].any()


def test_any_default_type():
    logp, ref, begin = batch(8)
    pl = PreferenceLoss(80, 8, beta=0.5)
    want = [x.clone() for x in pl.loss(logp, ref, begin)]
    before = torch.get_default_dtype()
    try:
        for t in (torch.float64, torch.bfloat16):
            torch.set_default_dtype(t)
            for obj in (pl, PreferenceLoss(160, 16, beta=0.5)):
                sums, g = obj.loss(logp, ref, begin)
                assert torch.equal(sums, want[0]) and torch.equal(g, want[1]) and g.dtype is torch.float32
    finally:
        torch.set_default_dtype(before)


def test_two_graphs_of_different_numbers_of_pairs():
    """each has the mean over its own"""
    pl = PreferenceLoss(640, 64, beta=0.5)
    calls, graphs = [batch(n, seed=n) for n in (64, 5)], []
    want = [[x.clone() for x in pl.loss(*c)] for c in calls]
    for c in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            pl.loss(*c)
        graphs.append(g)
    for turn in range(3):
        for g, w, c in zip(graphs, want, calls):
            pl.sums.fill_(7.0)
            pl.g_logp.fill_(7.0)
            pl.loss(*calls[turn % 2])
            torch.cuda.synchronize()
            g.replay()
            assert torch.equal(pl.sums, w[0]) and torch.equal(pl.g_logp[:len(c[0])], w[1])

"""Token log probabilities where the number of threads, packs and workgroups that hold or share a row changes, with rows that end
inside a pack; alternatives among few, with all of a row's values in few threads' hands; and calls replayed from a graph."""
import pytest
import torch

import paper_1903_04488_amd as cs
from test_gpu_token_logprobs import TYPES, best, check_forward, check_gradients, forward, logits_of

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PACK = {"f32": 4, "bf16": 8, "f16": 8}


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("packs", [64, 128, 192, 256, 1024, 2048, 4096, 6144, 8192, 12288, 16384])
def test_around_a_step_of_held_rows(packs, dtype):
    """few rows (1024 threads each) and many (as few threads as hold them)"""
    for vocab in (packs * PACK[dtype] - 1, packs * PACK[dtype], packs * PACK[dtype] + 1):
        for rows in (3, 520) if packs <= 4096 else (3,):
            x, target = logits_of(rows, vocab, TYPES[dtype])
            check_forward(x, target, 6)
            check_gradients(x, target)


@pytest.mark.parametrize("rows", [515, 1030])
@pytest.mark.parametrize("vocab", [40_001, 70_000, 131_071])
def test_many_long_rows(rows, vocab):
    x, target = logits_of(rows, vocab, torch.bfloat16)
    check_forward(x, target, 12)
    check_gradients(x, target, 1.1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows", [1, 2, 5, 37, 200])
@pytest.mark.parametrize("vocab", [65_536, 65_537, 98_311, 262_144, 262_145])
def test_rows_in_parts(rows, vocab, dtype):
    x, target = logits_of(rows, vocab, TYPES[dtype], pad=3)
    x[0, vocab // 3:] = -float("inf")                    # parts with nothing in them
    check_forward(x, target, 0)
    check_forward(x, target, 64)


@pytest.mark.parametrize("rows,vocab", [(1, 1000), (600, 1000), (1, 30_000), (600, 9_000), (1, 200_000)])
def test_alternatives_of_rows_full_of_equal_values(rows, vocab):
    """whole rows of one value, of -inf, and of two kinds in stretches: everything is decided by the index"""
    x = torch.zeros(rows, vocab, dtype=torch.bfloat16, device=DEV)
    target = torch.zeros(rows, dtype=torch.int64, device=DEV)
    for change in (lambda: None, lambda: x.fill_(-float("inf")), lambda: x[:, vocab // 2:].fill_(1.0), lambda: x[:, ::3].fill_(1.0)):
        change()
        for top in (1, 20, 64):
            _, _, _, idx, _ = forward(x, target, top)
            assert torch.equal(idx, best(x, top))


@pytest.mark.parametrize("rows,vocab,top", [(1, 500, 3), (3, 40_000, 5), (2, 150_000, 8), (700, 3000, 0)])
def test_calls_replayed_from_a_graph(rows, vocab, top):
    x, target = logits_of(rows, vocab, torch.float32)
    x = x.contiguous()
    f32 = dict(dtype=torch.float32, device=DEV)
    out = [torch.empty(rows, **f32) for _ in range(3)]
    idx = torch.empty(rows, top, dtype=torch.int64, device=DEV) if top else None
    lps = torch.empty(rows, top, **f32) if top else None
    ws = torch.empty(cs.cs_token_workspace_bytes(rows, vocab, top), dtype=torch.uint8, device=DEV)
    one, dx = torch.ones(rows, **f32), torch.empty_like(x)

    def calls():
        cs.cs_token_logprobs(x, target, *out, idx, lps, ws)
        cs.cs_token_logprobs_grad(x, target, out[2], out[1], one, one, dx)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for turn in range(4):
        x.copy_(logits_of(rows, vocab, torch.float32, seed=10 + turn)[0])
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (*out, dx, *([idx, lps] if top else []))]
        calls()
        torch.cuda.synchronize()
        for a, b in zip(got, (*out, dx, *([idx, lps] if top else []))):
            assert torch.equal(a, b)


@pytest.mark.parametrize("vocab", [200, 3000, 40_000])
def test_a_scale_that_takes_masked_values_out_of_range(vocab):
    """logits of 1e-12 under a scale of 1e12, masks of -1e30, which are -inf once scaled"""
    x, target = logits_of(5, vocab, torch.float32)
    x.mul_(1e-12)
    x[:, ::2] = -1e30
    target[:] = 1
    check_forward(x, target, 3, 1e12)
    check_gradients(x, target, 1e12)


def test_the_most_rows_of_a_call():
    """2^24 - 1 short rows, a workgroup each in the gradient: the same bits as the few rows they repeat"""
    rows, some, vocab = (1 << 24) - 1, 4096, 3
    x, target = logits_of(some, vocab, torch.bfloat16)

    def run(x, target):
        n = x.shape[0]
        ws = torch.empty(max(cs.cs_token_workspace_bytes(n, vocab, 2), cs.cs_token_workspace_bytes(n, vocab, 0)), dtype=torch.uint8, device=DEV)
        v = [torch.empty(n, device=DEV) for _ in range(6)]
        top_idx, top_logp = torch.empty(n, 2, dtype=torch.int64, device=DEV), torch.empty(n, 2, device=DEV)
        dx, both = torch.empty_like(x), torch.empty_like(x)
        g = torch.full((n,), 0.5, device=DEV)
        cs.cs_token_logprobs(x, target, v[0], v[1], v[2], top_idx, top_logp, ws)
        cs.cs_token_logprobs_grad(x, target, v[2], v[1], g, g, dx)
        cs.cs_token_loss(x, target, g, g, v[3], v[4], v[5], both, ws)
        return v + [top_idx, top_logp, dx, both]

    few = run(x, target)
    times = rows // some + 1
    many = run(x.repeat(times, 1)[:rows].contiguous(), target.repeat(times)[:rows].contiguous())
    whole = rows // some * some
    bits = {torch.float32: torch.int32, torch.bfloat16: torch.int16, torch.int64: torch.int64}
    for a, b in zip(few, many):
        a, b = a.view(bits[a.dtype]), b.view(bits[b.dtype])
        assert bool((b[:whole].reshape(-1, *a.shape) == a).all())
        assert torch.equal(b[whole:], a[:rows - whole])

"""Cases of the operators that train a language model on answers, for timing: two losses with their gradients, and the
optimizer of its matrices.

A case is one pass of one operator, through the public entry points:

    policy        clipped policy loss with a KL estimate against a reference and an entropy bonus.  `vocab` 0: from the tokens' log
                  probabilities, with the gradients of log probability and entropy; otherwise from rows of logits, with the
                  gradient of the logits
    preference    loss of pairs of answers (logistic, hinge, square) packed after one another, with the gradient of every token's log
                  probability
    orthogonal    stacks of matrices orthogonalised by Newton-Schulz products
    muon          one step of the optimizer that does this with its momentum, over a stack of matrices

Policy loss of a token with log probability l (behaviour policy: l0, reference: l1), entropy H, advantage A and weight w:
    r = e^(l - l0),  K = e^(l1 - l) - (l1 - l) - 1,  loss = w (-min(r A, clip(r) A) + kl K - bonus H),  clip to [1 - lo, 1 + hi]
Preference loss of a pair: R = beta times the sum (or mean) of l - l1 over an answer's tokens that count, z = R_chosen - R_rejected -
margin; logistic: (1 - s) ln(1 + e^-z) + s ln(1 + e^z), hinge: max(0, 1 - z), square: ((z - 1/2) / beta)^2.  Chosen answers come first, then
the rejected ones in the same order.
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
LOW, HIGH = 0.2, 0.28                    # clipping
SMOOTH = {"logistic": 0.1, "hinge": 0.0, "square": 0.0}
COEFS = ((3.4445, -4.7750, 2.0315),) * 5
EPS = 1e-7
LR, MOMENTUM, DECAY = 0.02, 0.95, 0.01


def _policy(rows, vocab, dtype="f32", kl=0.0, bonus=0.0, masked=False, pad=0, name=None):
    case = {"kind": "policy", "rows": rows, "vocab": vocab, "dtype": dtype, "kl": kl, "bonus": bonus, "masked": masked, "pad": pad}
    return case | ({"name": name} if name else {})


def _preference(pairs, longest, loss, beta, mean=False, reference=True, name=None):
    case = {"kind": "preference", "pairs": pairs, "longest": longest, "loss": loss, "beta": beta, "mean": mean, "reference": reference}
    return case | ({"name": name} if name else {})


def _matrices(kind, count, rows, cols, dtype, g=None, name=None):
    case = {"kind": kind, "count": count, "rows": rows, "cols": cols, "dtype": dtype, "g": g or dtype}
    return case | ({"name": name} if name else {})


def listed():
    return [
        # one short answer whose log probabilities come from elsewhere: nothing but the launch and the call
        _policy(777, 0, kl=0.04, bonus=0.01, name="policy-777"),
        # a few answers, logits in 32 bits, a vocabulary that is no multiple of anything
        _policy(300, 32001, "f32", kl=0.04, name="policy-300x32001"),
        # constrained answers: most of the vocabulary masked; rows padded; entropy bonus, no reference
        _policy(2047, 50021, "f16", bonus=0.01, masked=True, pad=27, name="policy-2047x50021-f16"),
        # a training step's batch
        _policy(8192, 34000, "bf16", kl=0.04, name="policy-8192x34000-bf16"),
        # a small batch of pairs
        _preference(16, 400, "logistic", 0.1, name="preference-16x400"),
        # few pairs of very long answers, means of log probabilities without a reference
        _preference(5, 131072, "hinge", 2.0, mean=True, reference=False, name="preference-5x131072"),
        # an epoch's pairs at once
        _preference(4096, 1000, "square", 0.1, name="preference-4096x1000"),
        # a matrix of a small model: latency counts
        _matrices("orthogonal", 1, 64, 64, "f32", name="orthogonal-64x64"),
        # odd sizes
        _matrices("orthogonal", 3, 1531, 1000, "f16", name="orthogonal-3x1531x1000-f16"),
        # a large model's matrix
        _matrices("orthogonal", 1, 4096, 4096, "bf16", name="orthogonal-4096x4096-bf16"),
        # the attention matrices of a transformer of 12 layers of width 512
        _matrices("muon", 48, 512, 512, "bf16", name="muon-48x512x512-bf16"),
        # half of its feed-forward matrices, kept in 32 bits, with gradients in bf16
        _matrices("muon", 12, 2048, 512, "f32", "bf16", name="muon-12x2048x512-f32"),
    ]


def _log(rng, lo, hi):
    return int(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.999))))


def draw(rng):
    """One more case: policy losses of 1 to a million tokens, or of 1 to 16 384 rows of logits of vocabularies of 100 to 131 072;
    1 to 8192 pairs of answers of up to 131 072 tokens; 1 to 64 matrices of 16 to 4096 rows and columns; all types."""
    kind = rng.choice(["policy", "policy", "preference", "orthogonal", "muon"])
    if kind == "policy":
        more = dict(kl=rng.choice([0.0, 0.04]), bonus=rng.choice([0.0, 0.01]))
        if rng.random() < 0.3:
            return _policy(_log(rng, 1, 1_000_000), 0, **more)
        vocab = _log(rng, 100, 131072)
        if rng.random() < 0.5:
            vocab = max(128, vocab // 128 * 128)
        rows = _log(rng, 1, min(16384, max(1, 100_000_000 // vocab)))
        return _policy(rows, vocab, rng.choice(["f32", "bf16", "f16"]), masked=rng.random() < 0.3, pad=rng.choice([0, 0, 3, 40]), **more)
    if kind == "preference":
        longest = _log(rng, 1, 131072)
        pairs = _log(rng, 1, min(8192, max(1, 4_000_000 // longest)))
        loss = rng.choice(["logistic", "hinge", "square"])
        return _preference(pairs, longest, loss, rng.choice([0.1, 0.5]), rng.random() < 0.3, rng.random() < 0.7)
    while True:
        rows, cols, count = _log(rng, 16, 4096), _log(rng, 16, 4096), _log(rng, 1, 64)
        if rng.random() < 0.5:
            rows, cols = max(16, rows // 64 * 64), max(16, cols // 64 * 64)
        if count * _flops(rows, cols) <= _flops(4096, 4096) and count * rows * cols <= 40_000_000:
            break
    dtype = rng.choice(["f32", "bf16", "f16"])
    return _matrices(kind, count, rows, cols, dtype, rng.choice([dtype, "f32", "bf16"]) if kind == "muon" else dtype)


def _flops(rows, cols):
    """A and A A are symmetric: one half of each is enough"""
    n, m = sorted((rows, cols))
    return len(COEFS) * (n * n * m + n * n * n + 2 * n * n * m)


def _lengths(case):
    n = 2 * case["pairs"]
    return [0 if i % 37 == 5 else 1 + int(case["longest"] * ((i + 0.5) / n) ** 2) for i in range(n)]


# ------------------------------------------------------------------------------------------
class _State:
    pass


def _away(x, *borders):
    """values that are not next to a border, on either side of which results are different ones"""
    for b in borders:
        x = torch.where((x - b).abs() < 2e-3, b + torch.where(x < b, -2e-3, 2e-3), x)
    return x


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = _State()
    s.case = case
    f32 = dict(dtype=torch.float32, device=DEV)

    def normal(*shape):
        return torch.empty(*shape, device=DEV).normal_(generator=gen)

    def uniform(*shape):
        return torch.rand(*shape, device=DEV, generator=gen)

    if case["kind"] == "policy":
        rows, vocab = case["rows"], case["vocab"]
        if vocab:
            dtype = TYPES[case["dtype"]]
            x = 2.0 * normal(rows, vocab)
            # what a trained model gives: a few tokens stand out, and its answers are mostly among them
            few = torch.randint(0, vocab, (rows, 6), device=DEV, generator=gen)
            x.scatter_reduce_(1, few, math.log(vocab) + 1.0 + 0.7 * normal(rows, 6), "amax")
            s.target = torch.where(uniform(rows) < 0.8, few[:, 0], torch.randint(0, vocab, (rows,), device=DEV, generator=gen))
            if case["masked"]:
                closed = uniform(rows, vocab) < 0.9
                closed.scatter_(1, few, False).scatter_(1, s.target[:, None], False)
                x.masked_fill_(closed, -math.inf)
            whole = torch.zeros(rows, vocab + case["pad"], dtype=dtype, device=DEV)
            whole[:, :vocab] = x
            s.logits = whole[:, :vocab]
            logp = torch.log_softmax(s.logits.float(), 1).gather(1, s.target[:, None])[:, 0]
            s.target[uniform(rows) < 0.05] = -1          # padding: left out
            del x
        else:
            logp = s.logp = -(1.5 * normal(rows) - 1.0).exp()
            s.entropy = (normal(rows) * 0.5).exp()
        s.old = logp - _away(0.15 * normal(rows), math.log(1.0 - LOW), math.log(1.0 + HIGH))
        s.ref = logp + 0.3 * normal(rows) if case["kl"] else None
        s.advantage = normal(rows)
        s.weight = torch.where(uniform(rows) < 0.9, 1.0 / rows, 0.0)
        if case["dtype"] == "f16" and vocab:
            s.weight *= 4096.0                           # gradients in binary16 are scaled up, as a training step does it
        if own:
            from paper_1903_04488_amd import binding as B
            s.h = B.CsPolicy(LOW, HIGH, case["kl"], case["bonus"])
            s.loss, s.sums = torch.empty(rows, **f32), torch.empty(4, **f32)
            if vocab:
                s.logp, s.entropy, s.lse = (torch.empty(rows, **f32) for _ in range(3))
                s.dlogits = torch.empty(rows, vocab, dtype=dtype, device=DEV)
                need = B.cs_token_policy_workspace_bytes(rows, vocab)
            else:
                s.g_logp, s.g_entropy = torch.empty(rows, **f32), torch.empty(rows, **f32)
                need = B.cs_policy_workspace_bytes(rows)
            s.workspace = torch.empty(need, dtype=torch.uint8, device=DEV)
    elif case["kind"] == "preference":
        pairs = case["pairs"]
        # lengths of very different answers, now and then an empty one; a batch ends with padding
        lengths = _lengths(case)
        tokens = sum(lengths) + 100
        lengths = torch.tensor(lengths, device=DEV)[torch.randperm(2 * pairs, device=DEV, generator=gen)]
        s.begin = torch.zeros(2 * pairs + 1, dtype=torch.int64, device=DEV)
        s.begin[1:] = lengths.cumsum(0)
        s.logp = -(1.5 * normal(tokens) - 1.0).exp()
        s.ref = s.logp + 0.2 * normal(tokens) if case["reference"] else None
        s.counts = uniform(tokens) < 0.8                 # the questions' tokens do not count
        s.weight = torch.full((pairs,), 1.0 / pairs, device=DEV)
        s.margin = 0.0 if case["reference"] else 0.5
        s.g = torch.zeros(tokens, **f32)
        if own:
            from paper_1903_04488_amd import binding as B
            kind = {"logistic": B.CS_PREFERENCE_LOGISTIC, "hinge": B.CS_PREFERENCE_HINGE, "square": B.CS_PREFERENCE_SQUARE}[case["loss"]]
            s.h = B.CsPreference(kind, case["mean"], case["beta"], SMOOTH[case["loss"]], s.margin)
            s.loss, s.reward, s.sums = torch.empty(pairs, **f32), torch.empty(2 * pairs, **f32), torch.empty(3, **f32)
            s.workspace = torch.empty(B.cs_preference_workspace_bytes(tokens, pairs), dtype=torch.uint8, device=DEV)
    else:
        count, rows, cols, dtype = case["count"], case["rows"], case["cols"], TYPES[case["dtype"]]
        # what gradients of matrices are: noise, and some directions that are much larger
        few = max(1, min(rows, cols) // 8)
        strong = 8.0 * torch.exp(-3.0 * torch.arange(few, device=DEV) / few) / few ** 0.5
        size = 1e-3 * (0.5 * normal(count, 1, 1)).exp()

        def gradient():
            return size * (normal(count, rows, cols) + (normal(count, rows, few) * strong) @ normal(count, few, cols))

        s.g = gradient().to(TYPES[case["g"]])
        if case["kind"] == "muon":
            s.p, s.m = (0.02 * normal(count, rows, cols)).to(dtype), 5.0 * gradient()
            if own:
                from paper_1903_04488_amd.training import Muon
                s.optimizer = Muon([s.p], [s.g], lr=LR, momentum=MOMENTUM, weight_decay=DECAY, eps=EPS, coefs=COEFS, m=[s.m])
        elif own:
            from paper_1903_04488_amd.training import Orthogonalizer
            s.out = torch.empty_like(s.g)
            s.orthogonalizer = Orthogonalizer([s.g], [s.out], eps=EPS, coefs=COEFS)
    return s


# ------------------------------------------------------------------------------------------ plain forms
def _plain_policy_tokens(s, logp, entropy, weight):
    """of every token: loss, gradients of logp and entropy, and the sums; 64 bits, as log ratios are small differences"""
    kl, bonus = s.case["kl"], s.case["bonus"]
    logp, a, w = logp.double(), s.advantage.double(), weight.double()
    r = (logp - s.old.double()).exp()
    plain, clipped = r * a, r.clamp(1.0 - LOW, 1.0 + HIGH) * a
    inside = plain <= clipped
    loss, g = -torch.minimum(plain, clipped), torch.where(inside, -plain, 0.0)
    k = torch.zeros_like(loss)
    if kl:
        e = s.ref.double() - logp
        k = e.exp() - e - 1.0
        loss, g = loss + kl * k, g + kl * (1.0 - e.exp())
    if bonus:
        loss = loss - bonus * entropy.double()
    loss, g = torch.where(w != 0, w * loss, 0.0), torch.where(w != 0, w * g, 0.0)
    sums = torch.stack([loss.sum(), (w * k).sum(), (w * ~inside).sum(), w.sum()])
    return loss.float(), g.float(), (-bonus * w).float(), sums.float()


def _plain_policy(s):
    if not s.case["vocab"]:
        loss, g, h, sums = _plain_policy_tokens(s, s.logp, s.entropy, s.weight)
        return {"loss": loss, "g_logp": g, "g_entropy": h, "sums": sums}
    x = s.logits.float()
    most = x.amax(1, keepdim=True)
    d = x - most
    e = d.exp()
    total = e.sum(1, keepdim=True)
    log_total = total.log()
    entropy = log_total - torch.where(e > 0, e * d, 0.0).sum(1, keepdim=True) / total
    counts = ((s.target >= 0) & (s.target < x.shape[1]))[:, None]
    at = s.target[:, None].clamp(0, x.shape[1] - 1)
    logp = torch.where(counts, d.gather(1, at) - log_total, 0.0)
    weight = torch.where(counts[:, 0], s.weight, 0.0)
    loss, g, h, sums = _plain_policy_tokens(s, logp[:, 0], entropy[:, 0], weight)
    p = e / total
    dx = p * -g[:, None]
    if s.case["bonus"]:
        dx -= h[:, None] * torch.where(p > 0, p * (d - log_total + entropy), 0.0)
    dx.scatter_add_(1, at, g[:, None])
    return {"logp": logp[:, 0], "entropy": entropy[:, 0], "loss": loss, "sums": sums, "dlogits": dx.to(s.logits.dtype)}


def _plain_preference(s):
    """sums over answers as differences of running sums, in 64 bits"""
    pairs, beta, smooth = s.case["pairs"], s.case["beta"], SMOOTH[s.case["loss"]]
    ratio = s.logp.double() if s.ref is None else s.logp.double() - s.ref.double()

    def of_answers(x):
        running = torch.zeros(len(x) + 1, dtype=torch.float64, device=DEV)
        running[1:] = x.cumsum(0)
        return running[s.begin[1:]] - running[s.begin[:-1]]

    total = of_answers(torch.where(s.counts, ratio, 0.0))
    each = torch.full_like(total, beta)
    if s.case["mean"]:
        each = beta / of_answers(s.counts.double()).clamp(min=1.0)
    reward = total * each
    better, worse = reward[:pairs], reward[pairs:]
    z = better - worse - s.margin
    if s.case["loss"] == "logistic":
        loss = (1.0 - smooth) * torch.log1p((-z).exp()) + smooth * torch.log1p(z.exp())
        dz = smooth - 1.0 / (1.0 + z.exp())
    elif s.case["loss"] == "hinge":
        loss, dz = (1.0 - z).clamp(min=0.0), torch.where(z < 1.0, -1.0, 0.0)
    else:
        loss, dz = ((z - 0.5) / beta) ** 2, 2.0 * (z - 0.5) / beta ** 2
    dz = dz * s.weight
    coef = torch.cat([dz, -dz]) * each
    inside = torch.arange(len(s.g), device=DEV)
    answer = (torch.searchsorted(s.begin, inside, right=True) - 1).clamp(max=2 * pairs - 1)
    g = torch.where(s.counts & (inside < s.begin[-1]), coef[answer], 0.0)
    sums = torch.stack([(s.weight * loss).sum(), (s.weight * (better > worse)).sum(), (s.weight * (better - worse)).sum()])
    return {"loss": loss.float(), "reward": reward.float(), "g_logp": g.float(), "sums": sums.float()}


def _plain_orthogonal(u):
    """in 32 bits, the shorter side first"""
    tall = u.shape[1] > u.shape[2]
    x = u.transpose(1, 2).contiguous() if tall else u
    x = x / (x.square().sum((1, 2), keepdim=True).sqrt() + EPS)
    for a, b, c in COEFS:
        square = torch.matmul(x, x.transpose(1, 2).contiguous())
        x = a * x + torch.matmul(b * square + c * torch.matmul(square, square), x)
    return x.transpose(1, 2) if tall else x


def _plain_matrices(s):
    if s.case["kind"] == "orthogonal":
        return {"o": _plain_orthogonal(s.g.float()).to(s.g.dtype)}
    g = s.g.float()
    s.m = MOMENTUM * s.m + g
    o = _plain_orthogonal(g + MOMENTUM * s.m)
    shape = max(1.0, s.case["rows"] / s.case["cols"]) ** 0.5
    s.p = (s.p.float() * (1.0 - LR * DECAY) - (LR * shape) * o).to(s.p.dtype)
    return {"p": s.p, "m": s.m}


# ------------------------------------------------------------------------------------------ the framework's calls
def _own_policy(s):
    from paper_1903_04488_amd import binding as B
    if not s.case["vocab"]:
        B.cs_policy_loss(s.h, s.logp, s.entropy, s.old, s.ref, s.advantage, s.weight, s.loss, s.g_logp, s.g_entropy, s.sums, s.workspace)
        return {"loss": s.loss, "g_logp": s.g_logp, "g_entropy": s.g_entropy, "sums": s.sums}
    B.cs_token_policy_loss(s.h, s.logits, s.target, s.old, s.ref, s.advantage, s.weight, s.logp, s.entropy, s.lse, s.loss, s.sums,
                           s.dlogits, s.workspace)
    return {"logp": s.logp, "entropy": s.entropy, "loss": s.loss, "sums": s.sums, "dlogits": s.dlogits}


def _own_preference(s):
    from paper_1903_04488_amd import binding as B
    B.cs_preference_loss(s.h, s.logp, s.ref, s.counts, s.begin, s.weight, s.loss, s.reward, s.g, s.sums, s.workspace)
    return {"loss": s.loss, "reward": s.reward, "g_logp": s.g, "sums": s.sums}


def _own_matrices(s):
    if s.case["kind"] == "orthogonal":
        s.orthogonalizer.run()
        return {"o": s.out}
    s.optimizer.step()
    return {"p": s.p, "m": s.m}


def run(s):
    kind = s.case["kind"]
    if kind == "policy":
        return _own_policy(s) if own else _plain_policy(s)
    if kind == "preference":
        return _own_preference(s) if own else _plain_preference(s)
    return _own_matrices(s) if own else _plain_matrices(s)


# ------------------------------------------------------------------------------------------
def work(case):
    """Bytes: every input read once, every output written once.  Operations of products alone, the symmetric ones' half."""
    if case["kind"] == "policy":
        rows, n = case["rows"], case["rows"] * case["vocab"]
        if not n:
            return {"bytes": rows * ((24 if case["kl"] else 20) + 12), "flops": 20 * rows}
        return {"bytes": 2 * n * SIZE[case["dtype"]] + rows * ((24 if case["kl"] else 20) + 16), "flops": 12 * n}
    if case["kind"] == "preference":
        tokens = sum(_lengths(case))
        return {"bytes": tokens * (13 if case["reference"] else 9) + case["pairs"] * 32, "flops": 6 * tokens}
    count, rows, cols = case["count"], case["rows"], case["cols"]
    one = SIZE[case["dtype"]]
    each = 2 * one if case["kind"] == "orthogonal" else 2 * one + SIZE[case["g"]] + 8
    return {"bytes": count * rows * cols * each, "flops": count * _flops(rows, cols)}


# ------------------------------------------------------------------------------------------ in 64 bits
def _exact_policy_tokens(s, logp, entropy, weight):
    a, kl, bonus = s.advantage.double(), s.case["kl"], s.case["bonus"]
    ratio = torch.exp(logp - s.old)
    most = torch.where(a >= 0, 1 + HIGH, math.inf)
    least = torch.where(a >= 0, -math.inf, 1 - LOW)
    held = ratio.clamp(least, most)                      # the side on which clipping lowers the objective
    cut = held != ratio
    objective, slope = held * a, torch.where(cut, 0.0, ratio * a)
    over = torch.zeros_like(objective)
    if kl:
        e = s.ref.double() - logp
        over = torch.expm1(e) - e
        objective, slope = objective - kl * over, slope + kl * torch.expm1(e)
    objective = objective + bonus * entropy
    take = weight != 0
    loss = -(weight * objective)[take].sum()
    return (torch.where(take, -weight * objective, 0.0), torch.where(take, -weight * slope, 0.0), -bonus * weight,
            torch.stack([loss, weight.dot(over), weight[cut].sum(), weight.sum()]))


def _exact_policy(s):
    if not s.case["vocab"]:
        return dict(zip(("loss", "g_logp", "g_entropy", "sums"),
                        _exact_policy_tokens(s, s.logp.double(), s.entropy.double(), s.weight.double())))
    step = max(1, (1 << 25) // s.case["vocab"])
    pieces = [slice(i, i + step) for i in range(0, s.case["rows"], step)]
    valid = s.target >= 0
    at = s.target.clamp(min=0)
    logp, entropy = [], []
    for piece in pieces:
        lp = torch.log_softmax(s.logits[piece].double(), 1)
        logp.append(torch.where(valid[piece], lp.gather(1, at[piece, None])[:, 0], 0.0))
        entropy.append(-torch.nan_to_num(lp.exp() * lp, nan=0.0).sum(1))
    logp, entropy = torch.cat(logp), torch.cat(entropy)
    weight = torch.where(valid, s.weight, 0.0).double()
    loss, g, h, sums = _exact_policy_tokens(s, logp, entropy, weight)
    dlogits = []
    for piece in pieces:
        lp = torch.log_softmax(s.logits[piece].double(), 1)
        p = lp.exp()
        d = -g[piece, None] * p - h[piece, None] * (torch.nan_to_num(p * lp, nan=0.0) + p * entropy[piece, None])
        d[torch.arange(len(d), device=DEV), at[piece]] += g[piece]
        dlogits.append(d)
    return {"logp": logp, "entropy": entropy, "loss": loss, "sums": sums, "dlogits": torch.cat(dlogits)}


def _exact_preference(s):
    pairs, beta, loss_of = s.case["pairs"], s.case["beta"], s.case["loss"]
    lengths = s.begin.diff()
    answer = torch.repeat_interleave(torch.arange(2 * pairs, device=DEV), lengths)
    used = s.counts[:len(answer)]
    ratio = s.logp.double()
    if s.ref is not None:
        ratio = ratio - s.ref
    total = torch.zeros(2 * pairs, dtype=torch.float64, device=DEV)
    total.index_add_(0, answer[used], ratio[:len(answer)][used])
    scale = torch.full_like(total, beta)
    if s.case["mean"]:
        scale /= torch.bincount(answer[used], minlength=2 * pairs).clamp(min=1)
    reward = scale * total
    gap = reward[:pairs] - reward[pairs:]
    z = (gap - s.margin).requires_grad_()
    if loss_of == "logistic":
        soft = torch.nn.functional.logsigmoid
        loss = -(1 - SMOOTH[loss_of]) * soft(z) - SMOOTH[loss_of] * soft(-z)
    elif loss_of == "hinge":
        loss = torch.relu(1 - z)
    else:
        loss = (z / beta - 1 / (2 * beta)) ** 2
    slope = torch.autograd.grad(loss.sum(), z)[0] * s.weight
    loss = loss.detach()
    g = torch.zeros(len(s.g), dtype=torch.float64, device=DEV)
    g[:len(answer)] = torch.where(used, (torch.cat([slope, -slope]) * scale)[answer], 0.0)
    w = s.weight.double()
    return {"loss": loss, "reward": reward, "g_logp": g, "sums": torch.stack([w.dot(loss), w[gap > 0].sum(), w.dot(gap)])}


def _exact_matrices(s):
    def polynomial(u):
        """x times a polynomial of x^T x or of x x^T, whichever is smaller"""
        x = u / (torch.linalg.matrix_norm(u, keepdim=True) + EPS)
        left = x.shape[1] <= x.shape[2]
        one = torch.eye(min(x.shape[1:]), dtype=torch.float64, device=DEV)
        for a, b, c in COEFS:
            gram = x @ x.mT if left else x.mT @ x
            factor = a * one + gram @ (b * one + c * gram)
            x = factor @ x if left else x @ factor
        return x

    g = s.g.double()
    if s.case["kind"] == "orthogonal":
        return {"o": polynomial(g)}
    m = MOMENTUM * s.m.double() + g
    o = polynomial(g + MOMENTUM * m)
    shape = math.sqrt(max(1, s.case["rows"] / s.case["cols"]))
    return {"p": s.p.double() - LR * (DECAY * s.p.double() + shape * o), "m": m}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "policy":
        return _exact_policy(s)
    return _exact_preference(s) if case["kind"] == "preference" else _exact_matrices(s)

"""The calls on given tokens at the limits of what they take: the largest and smallest temperatures, infinities and NaN at tokens that are
not valid, valid tokens of little mass, gradients over the logits of rows that are summed twice, eager calls beside a graph that runs."""
import numpy as np
import pytest
import torch

from paper_2504_09135_amd import binding as ppv

from gpu_helpers import DEV, to_dev, tuning
from logprobs_oracle import Scores, check_gradient, check_values, unpack
from test_gpu_logprobs import Case, hand_made_masks, odd_values, tokens_for

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [100, 3001, 40000])
@pytest.mark.parametrize("T", [3.0e38, 1.0e38, 5.0e37, 1.0e-30, 1.0e-37])
def test_largest_and_smallest_temperatures(T, V, dtype):
    """log2(e) / T and 1 / T from fp32's subnormal numbers (which round to 2^-22 of their size at T = 3e38) to near its largest.  Where T
    is large the distribution is even, whatever the logits, and T times a log probability may be outside fp32.  The upstream gradients are
    of T's size then, so that the gradients are of ordinary size: the terms that are multiplied by 1 / T are below 2^24 units of fp32's
    subnormal numbers otherwise, and every result would pass."""
    T = float(np.float32(T))
    rng = np.random.default_rng(V)
    B = 12
    valid = hand_made_masks(B, V, rng)
    for x in (rng.normal(0, 2.5, (B, V)), rng.normal(0, 5e37, (B, V)).clip(-1.6e38, 1.6e38)):
        if T < 1.0 and abs(x).max() > 1e30:
            continue        # (log probabilities outside fp32)
        for v in (None, valid):
            c = Case(x, dtype, v, tokens_for(v, B, V, rng), T=T)
            if T > 1.0:
                c.up = {n: (u * np.float32(0.05 * T)).astype(np.float32) for n, u in c.up.items()}
            c.check_backward(c.check_forward())
            if T < 1.0 or abs(x).max() > 1e30:
                c.check_top(2)
                c.check_top(40)
            else:           # (differences of 1e-38 are none to 64-bit log probabilities: the order is that of the logits)
                ids, lps = torch.zeros((B, 40), dtype=torch.int32, device=DEV), torch.zeros((B, 40), device=DEV)
                ppv.ppv_top_logprobs(c.logits, 40, ids, lps, mask=c.mask, tokens=c.tokens, temperature=T)
                want = Scores(c.x, v, c.tokens.cpu().numpy(), 1.0).top(40)[0]
                assert np.array_equal(ids.cpu().numpy(), want)
                check_values(lps.cpu().numpy(), np.where(want < 0, -np.inf, np.take_along_axis(c.ref.log_q, want.clip(0), 1)), "top_logprobs")


# a NaN that signals, as memory that nobody has written may hold; one of the other sign
BITS = {"signalling": {"f32": 0x7F800001, "bf16": 0x7F81}, "negative": {"f32": -1, "bf16": -1}}


@pytest.mark.parametrize("value", [float("inf"), float("nan"), "signalling", "negative"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V,split", [(100, 0), (3001, 0), (40000, 0), (40000, 4), (150000, 0)])
def test_infinities_and_nan_at_tokens_that_are_not_valid(V, split, dtype, value):
    """What is not valid counts for log Z alone: the log probability, the entropy, the alternatives and the gradients of these are what
    they are without it, and log Z says that there is none.  The odd token comes first, late, and more than once."""
    rng = np.random.default_rng(V + split)
    B = 16
    x = rng.normal(0, 2.5, (B, V))
    valid = hand_made_masks(B, V, rng)
    valid[:, 5] = True
    at = np.zeros((B, V), bool)
    for b in range(B):
        for v in (0, V // 2, V - 1)[:1 + b % 3][::-1 if b % 2 else 1]:
            at[b, v] = True
        at[b, rng.integers(0, V)] = True
    at &= ~valid
    assert at.any(1).sum() >= 8
    tok = tokens_for(valid, B, V, rng)
    with tuning(ppv.PPV_TUNE_ROW_SPLIT, split):
        c = Case(x, dtype, valid, tok, T=0.8)
        assert c.buf.shape[0] == B
        if value in BITS:
            c.logits.view(torch.int32 if dtype == "f32" else torch.int16)[torch.from_numpy(at).to(DEV)] = BITS[value][dtype]
        else:
            c.logits[torch.from_numpy(at).to(DEV)] = value
        lp, lz, h, st = c.forward()
        torch.cuda.synchronize()
        check_values(lp.cpu().numpy(), c.ref.logprobs, "logprobs")
        check_values(h.cpu().numpy(), c.ref.entropy, "entropy")
        odd = at.any(1) & (tok >= 0)
        assert np.isnan(lz.cpu().numpy()[odd]).all()
        check_values(lz.cpu().numpy()[~odd], c.ref.logZ[~odd], "logZ_valid")
        for k in (3, 100):
            c.check_top(k)
        up = {n: u for n, u in c.up.items() if n != "d_logZ_valid"}
        dev = {n: to_dev(u) for n, u in up.items()}
        buf = c.gradient_buffer()
        ppv.ppv_token_logprobs_backward(c.logits, c.tokens, st, buf[:, :V], mask=c.mask, temperature=c.T, **dev)
        c.check_gradient(buf, up, "backward")
        buf = c.gradient_buffer()
        ppv.ppv_token_logprobs_grad(c.logits, c.tokens, buf[:, :V], lp, mask=c.mask, entropy=h, temperature=c.T, **dev)
        c.check_gradient(buf, up, "grad")
        check_values(lp.cpu().numpy(), c.ref.logprobs, "grad: logprobs")
        check_values(h.cpu().numpy(), c.ref.entropy, "grad: entropy")


def plain_scores(x, valid, tok):
    """log q_t and the entropy in fp32, relative to the largest valid token: differences, exponentials, sums."""
    xv = torch.where(valid, x, -torch.inf)
    m = xv.amax(1, keepdim=True)
    y = xv - m
    e = y.exp()
    s = e.sum(1)
    lp = y.gather(1, tok.long()[:, None])[:, 0] - s.log()
    return lp, s.log() - torch.where(e > 0, y * e, 0.0).sum(1) / s


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1000, 20000, 100003])
@pytest.mark.parametrize("lower", [10.0, 20.0, 27.0])
@pytest.mark.parametrize("where", ["everywhere", "first half"])
def test_broad_valid_sets_of_little_mass(where, lower, V, dtype):
    """A model that disagrees with a broad constraint, all over the row or after a part that it agrees with.  The valid tokens' exponents are rounded relative to what they lie below a reference:
    where that is the valid tokens' own, as in the plain form, the errors are the plain form's but for the order of sums and for
    references that lie up to 12 units of the exponent of 2 (8.3 of the logits) from the largest token; the plain form's exponents average
    about 6 of the logits here (2.5 squared), so twice its error is room for either side."""
    rng = np.random.default_rng(V + int(lower))
    B = 200
    x = rng.normal(0, 2.5, (B, V))
    valid = rng.random((B, V)) < 0.5
    if where == "first half":
        valid[:, V // 2:] = False
        x[:, V // 2:] += lower
    else:
        x -= lower * valid
    tok = np.array([rng.choice(np.nonzero(v)[0]) for v in valid])
    c = Case(x, dtype, valid, tok)
    lp, lz, h, st = c.forward()
    d = c.gradient_buffer()[:, :V]
    lp2, h2 = torch.zeros(B, device=DEV), torch.zeros(B, device=DEV)
    ppv.ppv_token_logprobs_grad(c.logits, c.tokens, d, lp2, mask=c.mask, entropy=h2, d_logprobs=torch.ones(B, device=DEV))
    plain = plain_scores(c.logits.float(), torch.from_numpy(valid).to(DEV), c.tokens)
    torch.cuda.synchronize()
    rms = lambda got, want: float(np.sqrt(np.mean((got.double().cpu().numpy() - want) ** 2)))  # noqa: E731
    for name, got, base, want in (("logprobs", lp, plain[0], c.ref.logprobs), ("entropy", h, plain[1], c.ref.entropy),
                                  ("grad: logprobs", lp2, plain[0], c.ref.logprobs), ("grad: entropy", h2, plain[1], c.ref.entropy)):
        ours, theirs = rms(got, want), rms(base, want)
        print(f"{name}: {ours:.2e}, the plain form's {theirs:.2e}, {ours / theirs:.2f}")
        assert ours <= 2 * theirs, (name, ours, theirs)
    check_values(lz.cpu().numpy(), c.ref.logZ, "logZ_valid")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [100, 3001, 40000, 140001])
@pytest.mark.parametrize("kind", ["far", "lowest", "late peak", "low mass", "stairs", "high"])
def test_gradient_in_place_of_rows_that_are_summed_twice(kind, V, dtype):
    """d_logits may be the logits themselves also where the sums are taken again, by every wavefront from all of the row: none of them writes
    before all have read."""
    rng = np.random.default_rng(V)
    B = 10
    x = odd_values(kind, B, V, rng)
    valid = hand_made_masks(B, V, rng)
    if kind == "low mass":
        valid[:, :V // 2] = False
    if kind == "late peak":
        valid[:, V // 2:] = False
    if kind == "stairs":
        valid[:, V // 9:] = False
    for v in (None, valid):
        c = Case(x, dtype, v, tokens_for(v, B, V, rng))
        dev = {n: to_dev(u) for n, u in c.up.items()}
        lp, h = torch.zeros(B, device=DEV), torch.zeros(B, device=DEV)
        ppv.ppv_token_logprobs_grad(c.logits, c.tokens, c.logits, lp, mask=c.mask, entropy=h, temperature=c.T, **dev)
        c.check_gradient(c.buf, c.up, kind + " in place")
        check_values(lp.cpu().numpy(), c.ref.logprobs, kind)
        check_values(h.cpu().numpy(), c.ref.entropy, kind)


@pytest.mark.parametrize("masked", [False, True])
def test_eager_calls_beside_a_graph_that_runs(masked):
    """A graph's calls and eager ones on another stream, queued together, so that they may run at the same time: split rows and calls of two
    launches meet in areas of their own.  The results of both are those of calls alone, to the bit."""
    rng = np.random.default_rng(20)
    B, V, K = 5, 200003, 7
    valid = hand_made_masks(B, V, rng) if masked else None
    cases = [Case(rng.normal(0, 2, (B, V)), "bf16", valid, tokens_for(valid, B, V, rng), seed=i) for i in range(2)]
    f = lambda *s, **kw: torch.zeros(s, device=DEV, **kw)  # noqa: E731

    class Set:
        def __init__(self, c):
            self.c, self.up = c, {n: to_dev(u) for n, u in c.up.items()}
            self.outs = [f(B), f(B), f(B), f(B, ppv.PPV_LOGPROB_STATS), f(B), f(B, K, dtype=torch.int32), f(B, K)]
            self.d = c.gradient_buffer()

        def calls(self, stream=None):
            lp, lz, h, st, lp2, ids, lps = self.outs
            c = self.c
            ppv.ppv_token_logprobs(c.logits, c.tokens, lp, mask=c.mask, logZ_valid=lz, entropy=h, stats=st, stream=stream)
            ppv.ppv_token_logprobs_grad(c.logits, c.tokens, self.d[:, :V], lp2, mask=c.mask, stream=stream, **self.up)
            ppv.ppv_top_logprobs(c.logits, K, ids, lps, mask=c.mask, stream=stream)

        def clear(self):
            for t in self.outs:
                t.fill_(9)
            self.d[:, :V] = 9

        def results(self):
            return [t.clone() for t in (*self.outs, self.d)]

    sets = [Set(c) for c in cases]
    other = torch.cuda.Stream()
    for s in sets:      # (areas are laid ready)
        s.calls()
        s.calls(other)
    torch.cuda.synchronize()
    alone = [s.results() for s in sets]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(4):
            sets[0].calls()
    for _ in range(5):
        for s in sets:
            s.clear()
        torch.cuda.synchronize()
        graph.replay()
        for _ in range(4):
            sets[1].calls(other)
        graph.replay()
        torch.cuda.synchronize()
        for s, want in zip(sets, alone):
            for a, b in zip(s.results(), want):
                assert torch.equal(a, b)
    for s in sets:
        check_values(s.outs[0].cpu().numpy(), s.c.ref.logprobs, "logprobs")
        assert np.array_equal(s.outs[5].cpu().numpy(), Scores(s.c.x, valid, None, 1.0).top(K)[0])


@pytest.mark.parametrize("V,dtype", [(9, "f32"), (70, "bf16"), (1030, "f32")])
def test_more_rows_than_a_launch_takes(V, dtype):
    """2^21 rows and some: the rows behind are another launch's, with their own tokens, masks, gradients and results."""
    B, per = (1 << 21) + 5, 4 if dtype == "f32" else 8
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    g = torch.Generator(device=DEV).manual_seed(V)
    x = torch.empty((B, (V + per - 1) // per * per), dtype=dt, device=DEV).normal_(0, 2, generator=g)[:, :V]
    mask = torch.randint(-(1 << 31), (1 << 31) - 1, (B, (V + 31) // 32), generator=g, device=DEV, dtype=torch.int32)
    if V % 32:
        mask[:, -1] &= (1 << V % 32) - 1
    tokens = torch.randint(0, V, (B,), generator=g, device=DEV).to(torch.int32)
    lp, lz, h, up = (torch.randn((B,), generator=g, device=DEV) for _ in range(4))
    lp2, ids, lps = torch.zeros(B, device=DEV), torch.zeros((B, 3), dtype=torch.int32, device=DEV), torch.zeros((B, 3), device=DEV)
    stats = torch.zeros((B, ppv.PPV_LOGPROB_STATS), device=DEV)
    rows = torch.tensor([0, 1, 4_095, (1 << 21) - 1, *range(1 << 21, B)], device=DEV)
    ref = Scores(x[rows].double().cpu().numpy(), unpack(mask[rows].cpu().numpy(), V), tokens[rows].cpu().numpy(), 1.0)
    want, size = ref.gradient(up[rows].cpu().numpy(), None, None)
    ppv.ppv_token_logprobs(x, tokens, lp, mask=mask, logZ_valid=lz, entropy=h, stats=stats)
    ppv.ppv_top_logprobs(x, 3, ids, lps, mask=mask)
    d = torch.zeros((B, x.stride(0)), dtype=dt, device=DEV)[:, :V]
    ppv.ppv_token_logprobs_backward(x, tokens, stats, d, mask=mask, d_logprobs=up)
    check_values(lp[rows].cpu().numpy(), ref.logprobs, "logprobs")
    check_values(lz[rows].cpu().numpy(), ref.logZ, "logZ_valid")
    check_values(h[rows].cpu().numpy(), ref.entropy, "entropy")
    assert np.array_equal(ids[rows].cpu().numpy(), ref.top(3)[0])
    check_values(lps[rows].cpu().numpy(), ref.top(3)[1], "top_logprobs")
    check_gradient(d[rows].float().cpu().numpy(), want, size, dtype, "backward")
    ppv.ppv_token_logprobs_grad(x, tokens, x, lp2, mask=mask, d_logprobs=up)       # in place
    check_gradient(x[rows].float().cpu().numpy(), want, size, dtype, "grad")
    check_values(lp2[rows].cpu().numpy(), ref.logprobs, "grad: logprobs")

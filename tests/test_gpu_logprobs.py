"""ppv_token_logprobs, its gradient and ppv_top_logprobs against the plain 64-bit implementation, at the sizes, masks and values where
they can go wrong."""
import threading

import numpy as np
import pytest
import torch

from paper_2504_09135_amd import binding as ppv
from paper_2504_09135_amd import workloads as W

from gpu_helpers import DEV, to_dev, tuning
from logprobs_oracle import WEIGHT, Scores, bf16, check_gradient, check_values, pack, unpack

pytestmark = pytest.mark.gpu

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
SENTINEL = 77.0


def rows_on_gpu(x, dtype, pad=0, fill=SENTINEL):
    """x [B, V] as rows that start on 16-byte boundaries, `pad` groups of 16 bytes further apart than they need be."""
    per = 4 if dtype == "f32" else 8
    B, V = x.shape
    stride = (V + per - 1) // per * per + pad * per
    buf = torch.full((B, stride), fill, dtype=TORCH[dtype], device=DEV)
    buf[:, :V] = torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(DEV).to(TORCH[dtype])
    return buf


class Case:
    def __init__(self, x, dtype, valid=None, tokens=None, T=1.0, pad=0, seed=0):
        B, self.V = x.shape
        self.dtype, self.T, self.B = dtype, T, B
        self.x = np.ascontiguousarray(x, np.float32).astype(np.float64) if dtype == "f32" else bf16(x)
        self.buf = rows_on_gpu(x, dtype, pad)
        self.logits = self.buf[:, :self.V]
        self.mask = None if valid is None else to_dev(pack(valid))
        self.tokens = None if tokens is None else to_dev(np.asarray(tokens, np.int32))
        rng = np.random.default_rng(seed)
        self.up = {n: rng.normal(0, 1, B).astype(np.float32) for n in ("d_logprobs", "d_logZ_valid", "d_entropy")}
        if tokens is None:
            del self.up["d_logprobs"]
        self.ref = Scores(self.x, valid, None if tokens is None else np.asarray(tokens), T)

    def forward(self):
        z = lambda *s: torch.full(s, 5.0, device=DEV)  # noqa: E731
        lp = None if self.tokens is None else z(self.B)
        lz, h, st = z(self.B), z(self.B), z(self.B, ppv.PPV_LOGPROB_STATS)
        ppv.ppv_token_logprobs(self.logits, self.tokens, lp, mask=self.mask, logZ_valid=lz, entropy=h, stats=st, temperature=self.T)
        return lp, lz, h, st

    def check_scores(self, lp, lz, h, what):
        torch.cuda.synchronize()
        if lp is not None:
            check_values(lp.cpu().numpy(), self.ref.logprobs, what + " logprobs")
        check_values(lz.cpu().numpy(), self.ref.logZ, what + " logZ_valid")
        check_values(h.cpu().numpy(), self.ref.entropy, what + " entropy")

    def check_forward(self):
        lp, lz, h, st = self.forward()
        self.check_scores(lp, lz, h, "forward")
        return st

    def gradient_buffer(self, pad=1):
        return rows_on_gpu(np.full((self.B, self.V), 3.0), self.dtype, pad)

    def check_gradient(self, buf, up, what):
        torch.cuda.synchronize()
        d = buf.float().cpu().numpy()
        assert (d[:, self.V:] == SENTINEL).all(), what + ": written behind the rows"
        want, size = self.ref.gradient(up.get("d_logprobs"), up.get("d_logZ_valid"), up.get("d_entropy"))
        check_gradient(d[:, :self.V], want, size, self.dtype, what)

    def check_backward(self, st, names=("d_logprobs", "d_logZ_valid", "d_entropy")):
        up = {n: self.up[n] for n in names if n in self.up}
        dev = {n: to_dev(v) for n, v in up.items()}
        buf = self.gradient_buffer()
        ppv.ppv_token_logprobs_backward(self.logits, self.tokens, st, buf[:, :self.V], mask=self.mask, temperature=self.T, **dev)
        self.check_gradient(buf, up, "backward")
        buf, z = self.gradient_buffer(2), lambda: torch.full((self.B,), 5.0, device=DEV)
        lp, lz, h = None if self.tokens is None else z(), z(), z()
        ppv.ppv_token_logprobs_grad(self.logits, self.tokens, buf[:, :self.V], lp, mask=self.mask, logZ_valid=lz, entropy=h,
                                    temperature=self.T, **dev)
        self.check_gradient(buf, up, "grad")
        self.check_scores(lp, lz, h, "grad")

    def check_top(self, k):
        z = lambda *s, **kw: torch.full(s, 5, device=DEV, **kw)  # noqa: E731
        ids, lps = z(self.B, k, dtype=torch.int32), z(self.B, k, dtype=torch.float32)
        lp, h = None if self.tokens is None else z(self.B, dtype=torch.float32), z(self.B, dtype=torch.float32)
        ppv.ppv_top_logprobs(self.logits, k, ids, lps, mask=self.mask, tokens=self.tokens, logprobs=lp, entropy=h, temperature=self.T)
        torch.cuda.synchronize()
        want_ids, want_lps = self.ref.top(k)
        assert np.array_equal(ids.cpu().numpy(), want_ids), np.argwhere(ids.cpu().numpy() != want_ids)[:5]
        check_values(lps.cpu().numpy(), want_lps, "top_logprobs")
        if lp is not None:
            check_values(lp.cpu().numpy(), self.ref.logprobs, "top: logprobs")
        check_values(h.cpu().numpy(), self.ref.entropy, "top: entropy")

    def check_all(self, ks=(1, 5, 20)):
        st = self.check_forward()
        self.check_backward(st)
        for k in ks:
            self.check_top(k)


def hand_made_masks(B, V, rng):
    """every kind of valid set, by row: none, all, one (the first, the last), few, many, a block of neighbours"""
    valid = np.zeros((B, V), bool)
    for b in range(B):
        kind = b % 8
        if kind == 1:
            valid[b] = True
        elif kind == 2:
            valid[b, 0 if b % 16 < 8 else V - 1] = True
        elif kind == 3:
            valid[b, rng.choice(V, min(V, 5), replace=False)] = True
        elif kind == 4:
            valid[b] = rng.random(V) < 0.5
        elif kind == 5:
            a = int(rng.integers(0, V))
            valid[b, a:a + max(1, V // 4)] = True
        elif kind == 6:
            valid[b, rng.choice(V, min(V, 200), replace=False)] = True
        elif kind == 7:
            valid[b] = rng.random(V) < 0.02
    return valid


def tokens_for(valid, B, V, rng):
    """valid tokens mostly; left-out rows, tokens that are not valid and tokens outside the vocabulary among them"""
    tok = rng.integers(0, V, B)
    for b in range(B):
        if valid is not None and valid[b].any() and b % 5:
            tok[b] = rng.choice(np.nonzero(valid[b])[0])
    tok[B // 2::11] = -1
    tok[B // 3::13] = V
    tok[1::17] = 0x7FFFFFF0
    tok[2::19] = -0x80000000
    return tok


SIZES = [(9, 1), (9, 2), (17, 7), (33, 8), (9, 31), (9, 33), (40, 500), (19, 1024), (8, 1025), (8, 2048), (8, 2049), (20, 4100), (16, 32000),
         (9, 50265), (17, 128256), (3, 200003), (9, 262144)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,V", SIZES)
def test_against_64_bits(B, V, dtype):
    rng = np.random.default_rng(B * 1_000_003 + V)
    x = rng.normal(0, 2.5, (B, V))
    Case(x, dtype, None, tokens_for(None, B, V, rng), pad=1).check_all((1, 20))
    valid = hand_made_masks(B, V, rng)
    Case(x, dtype, valid, tokens_for(valid, B, V, rng), T=0.7).check_all((3, 128))


@pytest.mark.parametrize("B,V,dtype", [(700, 300, "f32"), (1500, 2500, "bf16"), (600, 6000, "f32"), (300, 9000, "bf16"), (260, 20000, "bf16")])
def test_many_rows(B, V, dtype):
    rng = np.random.default_rng(V)
    x = rng.normal(0, 2.5, (B, V))
    valid = hand_made_masks(B, V, rng)
    Case(x, dtype, valid, tokens_for(valid, B, V, rng)).check_all((20,))


@pytest.mark.parametrize("V,dtype", [(40, "f32"), (364, "bf16"), (1024, "f32"), (2932, "bf16"), (5000, "bf16")])
def test_many_alternatives_of_short_rows(V, dtype):
    """A wavefront or two to a row, and nearly as many alternatives as there are maxima to bound them with, or more than tokens."""
    rng = np.random.default_rng(V)
    B = 2100
    x = rng.normal(0, 2, (B, V))
    x[::3] = np.round(x[::3])       # many equal ones
    valid = rng.random((B, V)) < rng.choice([0.02, 0.5, 1.0], (B, 1))
    for v in (None, valid):
        c = Case(x, dtype, v, rng.integers(0, V, B))
        for k in (40, 64, 65, 73, 100, 128):
            c.check_top(k)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T", [0.05, 0.6, 1.0, 1.7, 30.0])
def test_temperatures(T, dtype):
    rng = np.random.default_rng(int(T * 100))
    B, V = 16, 5000
    x = rng.normal(0, 3, (B, V))
    valid = hand_made_masks(B, V, rng)
    Case(x, dtype, valid, tokens_for(valid, B, V, rng), T=T).check_all((10,))


@pytest.mark.parametrize("waves", [0, 1, 4])
@pytest.mark.parametrize("split", [1, 2, 4, 16])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_split_rows(dtype, split, waves):
    """Rows over several workgroups, whatever the library would choose: lengths that leave a part without a tile, all masks, all k."""
    with tuning(ppv.PPV_TUNE_ROW_SPLIT, split), tuning(ppv.PPV_TUNE_WAVES_PER_ROW, waves):
        for B, V in ((9, 4100), (3, 33000), (17, 50265), (9, 200003)):
            rng = np.random.default_rng(V + split)
            x = rng.normal(0, 2.5, (B, V))
            valid = hand_made_masks(B, V, rng)
            Case(x, dtype, valid, tokens_for(valid, B, V, rng), T=0.8).check_all((1, 20, 64, 128))
            Case(x, dtype, None, tokens_for(None, B, V, rng)).check_all((5,))
        for kind in ("ties", "filtered", "late peak", "lowest"):
            x = odd_values(kind, 8, 40000, rng)
            valid = hand_made_masks(8, 40000, rng)
            Case(x, dtype, valid, tokens_for(valid, 8, 40000, rng)).check_all((3, 100))


def test_one_area_for_calls_of_every_kind():
    """The calls that split rows share a stream's scratch area, one after the other, and leave nothing in it that another takes for its own;
    graphs that hold them are replayed beside eager calls."""
    rng = np.random.default_rng(6)
    B, V = 6, 128256
    valid = hand_made_masks(B, V, rng)
    c = Case(rng.normal(0, 2, (B, V)), "bf16", valid, tokens_for(valid, B, V, rng))
    u = to_dev(rng.random(B, dtype=np.float32))
    f = lambda *s, **kw: torch.zeros(s, device=DEV, **kw)  # noqa: E731
    outs = [f(B, dtype=torch.int32), f(B), f(B), f(B), f(B), f(B, 9, dtype=torch.int32), f(B, 9), f(B)]

    def calls():
        ids, lzv, lp, lz, h, top, tops, mine = outs
        ppv.constrained_sample(c.logits, c.mask, u, ids, lzv)
        ppv.ppv_token_logprobs(c.logits, c.tokens, lp, mask=c.mask, logZ_valid=lz, entropy=h)
        ppv.ppv_top_logprobs(c.logits, 9, top, tops, mask=c.mask, tokens=c.tokens, logprobs=mine)

    with tuning(ppv.PPV_TUNE_ROW_SPLIT, 1):
        calls()
        torch.cuda.synchronize()
        alone = [t.clone() for t in outs]
    for split in (0, 4, 16, 2):
        with tuning(ppv.PPV_TUNE_ROW_SPLIT, split):
            for _ in range(3):
                for t in outs:
                    t.fill_(7)
                calls()
            graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
            torch.cuda.synchronize()
            for g in graphs:
                with torch.cuda.graph(g):
                    calls()
        first = None
        for i in range(4):
            for t in outs:
                t.fill_(7)
            torch.cuda.synchronize()
            graphs[i % 2].replay()
            torch.cuda.synchronize()
            assert torch.equal(outs[0], alone[0]) and torch.equal(outs[5], alone[5])
            check_values(outs[2].cpu().numpy(), c.ref.logprobs, "logprobs")
            check_values(outs[6].cpu().numpy(), c.ref.top(9)[1], "top_logprobs")
            first = first or [t.clone() for t in outs]
            assert all(torch.equal(a, b) for a, b in zip(outs, first))      # the same to the bit, whatever arrived last


def odd_values(kind, B, V, rng):
    x = rng.normal(0, 2, (B, V))
    if kind == "filtered":              # a caller's top-k filter: -inf nearly everywhere, all over in some rows
        keep = rng.random((B, V)) < 0.002
        keep[::5] = False
        x = np.where(keep, x, -np.inf)
    elif kind == "lowest":              # the type's lowest value as a stand-in for -inf; rows of nothing else
        low = np.float64(-3.3895313892515355e38)
        x = np.where(rng.random((B, V)) < 0.01, x, low)
        x[::5] = low
    elif kind == "high":
        x += 1e4 * np.arange(-B // 2, B - B // 2)[:, None]
    elif kind == "far":                 # numbers of both signs whose differences, as exponents of 2, are outside fp32
        x = np.where(rng.random((B, V)) < 0.5, 1.5e38, -1.5e38)
        x[1::3] *= 1e-30
        x[2::3, 5] = 1e30
    elif kind == "ties":                # a handful of values, and rows of one
        x = rng.integers(0, 3, (B, V)).astype(np.float64)
        x[::4] = 1.5
        x[1::4] = np.where(rng.random((len(x[1::4]), V)) < 0.5, 0.0, -0.0)
    elif kind == "peak":                # all mass on one token
        x[np.arange(B), rng.integers(0, V, B)] += 90.0
    elif kind == "rising":              # each token likelier than the one before
        x = np.tile(np.linspace(-20, 5, V), (B, 1))
    elif kind == "falling":
        x = np.tile(np.linspace(5, -20, V), (B, 1))
    elif kind == "late peak":           # what is valid comes first and is far below what comes later; some of it far below the rest
        x[:, V // 4:V // 2] -= 250.0
        x[:, V // 2:] += 300.0
        x[:, 3 * V // 4:] += 60.0
    elif kind == "stairs":              # a lane's tokens rise by no more than 30 at a time, by 240 in all; what is valid lies on the lowest stair, or below
        x += 30.0 * (np.arange(V) * 9 // V)
        x[:, ::3] -= 60.0 * (np.arange(V)[::3] < V // 9)
    elif kind == "low mass":            # the valid tokens far below the rest
        x[:, V // 2:] -= 300.0
    return x


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [100, 3001, 40000])
@pytest.mark.parametrize("kind", ["filtered", "lowest", "high", "far", "ties", "peak", "rising", "falling", "low mass", "late peak", "stairs"])
def test_odd_values(kind, V, dtype):
    rng = np.random.default_rng(V)
    B = 12
    x = odd_values(kind, B, V, rng)
    valid = None if kind == "far" else hand_made_masks(B, V, rng)
    if kind == "low mass":
        valid[:, :V // 2] = False
    if kind == "late peak":
        valid[:, V // 2:] = False
    if kind == "stairs":
        valid[:, V // 9:] = False
    for v in (None, valid):
        tok = tokens_for(v, B, V, rng)
        c = Case(x, dtype, v, tok)
        st = c.check_forward()
        c.check_backward(st)
        for k in (2, 40):
            c.check_top(k)


def test_no_tokens_and_single_outputs():
    """Without tokens every row is taken; each output can be asked for alone and is the same then."""
    rng = np.random.default_rng(1)
    B, V = 11, 3000
    x = rng.normal(0, 2, (B, V))
    valid = hand_made_masks(B, V, rng)
    Case(x, "bf16", valid).check_all((4,))
    Case(x, "f32").check_all((4,))
    c = Case(x, "bf16", valid, tokens_for(valid, B, V, rng))
    lp, lz, h, st = c.forward()
    for name, want in (("logprobs", lp), ("logZ_valid", lz), ("entropy", h), ("stats", st)):
        alone = torch.full_like(want, 9.0)
        ppv.ppv_token_logprobs(c.logits, c.tokens, mask=c.mask, **{name: alone})
        assert torch.equal(alone, want), name
    for names in (("d_logprobs",), ("d_logZ_valid",), ("d_entropy",), ("d_logprobs", "d_entropy"), ()):
        c.check_backward(st, names)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [40, 2500, 40001])
def test_gradient_in_place(V, dtype):
    """d_logits may be the logits themselves."""
    rng = np.random.default_rng(V)
    B = 9
    x = rng.normal(0, 2, (B, V))
    valid = hand_made_masks(B, V, rng)
    for how in ("backward", "grad"):
        c = Case(x, dtype, valid, tokens_for(valid, B, V, rng), T=1.3)
        dev = {n: to_dev(v) for n, v in c.up.items()}
        if how == "backward":
            st = c.forward()[3]
            ppv.ppv_token_logprobs_backward(c.logits, c.tokens, st, c.logits, mask=c.mask, temperature=c.T, **dev)
        else:
            lp = torch.zeros(B, device=DEV)
            ppv.ppv_token_logprobs_grad(c.logits, c.tokens, c.logits, lp, mask=c.mask, temperature=c.T, **dev)
            torch.cuda.synchronize()
            check_values(lp.cpu().numpy(), c.ref.logprobs, how)
        c.check_gradient(c.buf, c.up, how + " in place")


@pytest.mark.parametrize("split", [0, 1])
@pytest.mark.parametrize("masked", [False, True])
@pytest.mark.parametrize("V,dtype", [(66_000, "f32"), (100_003, "f32"), (140_001, "bf16"), (262_144, "bf16")])
def test_rows_that_no_workgroup_holds(V, dtype, masked, split):
    """Parts of a row that are read again for the gradient, which may lie over it."""
    rng = np.random.default_rng(V)
    B = 7
    x = rng.normal(0, 2, (B, V))
    valid = hand_made_masks(B, V, rng) if masked else None
    with tuning(ppv.PPV_TUNE_ROW_SPLIT, split):
        c = Case(x, dtype, valid, tokens_for(valid, B, V, rng), T=0.9)
        c.check_all((3,))
        dev = {n: to_dev(v) for n, v in c.up.items()}
        lp = torch.zeros(B, device=DEV)
        ppv.ppv_token_logprobs_grad(c.logits, c.tokens, c.logits, lp, mask=c.mask, temperature=c.T, **dev)
        torch.cuda.synchronize()
        check_values(lp.cpu().numpy(), c.ref.logprobs, "in place")
        c.check_gradient(c.buf, c.up, "in place")


def test_rows_that_are_left_out_are_not_read():
    """A row of NaN whose token is negative leaves zeros; NaN in one row does not reach another."""
    rng = np.random.default_rng(2)
    for V, dtype in ((300, "f32"), (9000, "bf16")):
        B = 8
        x = rng.normal(0, 2, (B, V))
        tok = rng.integers(0, V, B)
        tok[3] = -1
        c = Case(x, dtype, None, tok)
        c.buf[3, :V] = float("nan")
        st = c.check_forward()
        assert (st[3] == 0).all()
        c.check_backward(st)
        c.check_top(6)
        c.buf[5, ::7] = float("nan")
        c.buf[6, 11] = float("inf")
        lp, lz, h, st = c.forward()
        ids, lps = torch.zeros((B, 128), dtype=torch.int32, device=DEV), torch.zeros((B, 128), device=DEV)
        ppv.ppv_top_logprobs(c.logits, 128, ids, lps)
        torch.cuda.synchronize()
        rest = [0, 1, 2, 4, 7]
        check_values(lp.cpu().numpy()[rest], c.ref.logprobs[rest], "beside NaN")
        got = ids.cpu().numpy()
        assert ((got >= -1) & (got < V)).all()
        assert np.array_equal(got[rest], c.ref.top(128)[0][rest])


def test_probabilities_are_not_above_one():
    """One valid token, and all of them valid: log probabilities and log masses are 0 at most, entropies 0 at least."""
    rng = np.random.default_rng(3)
    B, V = 64, 5000
    valid = np.zeros((B, V), bool)
    tok = rng.integers(0, V, B)
    valid[np.arange(B), tok] = True
    valid[::2] = True
    c = Case(rng.normal(0, 3, (B, V)), "f32", valid, tok, T=0.9)
    lp, lz, h, _ = c.forward()
    torch.cuda.synchronize()
    assert (lp <= 0).all() and (lz <= 0).all() and (h >= 0).all()
    assert (lp[1::2] >= -1e-6).all() and (h[1::2] <= 2e-5).all() and (lz[::2] >= -2e-5).all()


def test_offsets_beyond_32_bits():
    """Rows whose logits, masks and gradients lie beyond 2^32 bytes of their buffers' starts."""
    B, V = 9_000, 262_144
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.empty((B, V), dtype=torch.bfloat16, device=DEV).normal_(0, 2, generator=g)
    mask = torch.randint(-(1 << 31), (1 << 31) - 1, (B, V // 32), generator=g, device=DEV, dtype=torch.int32)
    tokens = torch.randint(0, V, (B,), generator=g, device=DEV).to(torch.int32)
    lp, lz, h, up = (torch.randn((B,), generator=g, device=DEV) for _ in range(4))
    ids, lps = torch.zeros((B, 9), dtype=torch.int32, device=DEV), torch.zeros((B, 9), device=DEV)
    rows = torch.tensor([0, 4_095, 4_096, 8_191, 8_192, 8_999], device=DEV)
    kept, words, tk, g_up = x[rows].clone(), mask[rows].clone(), tokens[rows].clone(), up[rows].clone()
    ppv.ppv_top_logprobs(x, 9, ids, lps, mask=mask)
    ppv.ppv_token_logprobs_grad(x, tokens, x, lp, mask=mask, d_logprobs=up, logZ_valid=lz, entropy=h)      # in place
    torch.cuda.synchronize()
    ref = Scores(kept.double().cpu().numpy(), unpack(words.cpu().numpy(), V), tk.cpu().numpy(), 1.0)
    check_values(lp[rows].cpu().numpy(), ref.logprobs, "logprobs")
    check_values(lz[rows].cpu().numpy(), ref.logZ, "logZ_valid")
    check_values(h[rows].cpu().numpy(), ref.entropy, "entropy")
    want, size = ref.gradient(g_up.cpu().numpy(), None, None)
    check_gradient(x[rows].float().cpu().numpy(), want, size, "bf16", "in place")
    assert np.array_equal(ids[rows].cpu().numpy(), ref.top(9)[0])


def test_two_streams_at_once():
    """Split rows of calls that run at the same time on two streams."""
    rng = np.random.default_rng(8)
    cases = [Case(rng.normal(0, 2, (3, 128256)), "bf16", None, rng.integers(0, 128256, 3), seed=i) for i in range(2)]
    streams = [torch.cuda.Stream() for _ in cases]
    outs = [[torch.zeros(3, device=DEV), torch.zeros((3, 5), dtype=torch.int32, device=DEV), torch.zeros((3, 5), device=DEV)] for _ in cases]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, s, (lp, ids, lps) in zip(cases, streams, outs):
            ppv.ppv_token_logprobs(c.logits, c.tokens, lp, stream=s)
            ppv.ppv_top_logprobs(c.logits, 5, ids, lps, stream=s)
    torch.cuda.synchronize()
    for c, (lp, ids, lps) in zip(cases, outs):
        check_values(lp.cpu().numpy(), c.ref.logprobs, "logprobs")
        assert np.array_equal(ids.cpu().numpy(), c.ref.top(5)[0])


def test_threads_on_one_stream():
    """Calls of two launches, whose second one reads what the first one left, from several threads on one stream, beside others there."""
    rng = np.random.default_rng(12)
    B, V, N = 4, 128256, 30
    cases = [Case(rng.normal(0, 2, (B, V)), "bf16", rng.random((B, V)) < 0.3, rng.integers(0, V, B), seed=i) for i in range(3)]
    up = torch.tensor([1.0, -0.5, 2.0, 0.25], device=DEV)
    outs = [torch.zeros((N, B, V), dtype=torch.bfloat16, device=DEV) for _ in cases]
    lps = [torch.zeros((N, B), device=DEV) for _ in cases]
    ids, alternatives = torch.zeros((N, B, 20), dtype=torch.int32, device=DEV), torch.zeros((N, B, 20), device=DEV)
    torch.cuda.synchronize()
    stream, start = torch.cuda.Stream(), threading.Barrier(len(cases) + 1)

    def gradients(c, out, lp):
        start.wait()
        for i in range(N):
            ppv.ppv_token_logprobs_grad(c.logits, c.tokens, out[i], lp[i], mask=c.mask, d_logprobs=up, d_entropy=up, stream=stream)

    def tops():
        start.wait()
        for i in range(N):
            ppv.ppv_top_logprobs(cases[0].logits, 20, ids[i], alternatives[i], mask=cases[0].mask, stream=stream)
    threads = [threading.Thread(target=gradients, args=a) for a in zip(cases, outs, lps)] + [threading.Thread(target=tops)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    g = up.cpu().numpy()
    for c, out, lp in zip(cases, outs, lps):
        check_values(lp[0].cpu().numpy(), c.ref.logprobs, "logprobs")
        want, size = c.ref.gradient(g, None, g)
        check_gradient(out[0].float().cpu().numpy(), want, size, "bf16", "threads")
        assert (out == out[0]).all() and (lp == lp[0]).all()
    assert np.array_equal(ids[0].cpu().numpy(), cases[0].ref.top(20)[0]) and (ids == ids[0]).all()


def test_gradient_against_differences():
    """The gradient is what the forward call's outputs do when a logit moves: central differences in fp32 logits."""
    rng = np.random.default_rng(5)
    B, V, step = 64, 96, 0.25
    x = (np.round(rng.normal(0, 1.5, V) * 256) / 256).astype(np.float32)
    valid = np.tile(rng.random(V) < 0.6, (B, 1))
    tok = int(np.nonzero(valid[0])[0][4])
    up = {"d_logprobs": 0.7, "d_logZ_valid": -1.1, "d_entropy": 0.4}

    def value(rows, v):
        c = Case(rows, "f32", v, np.full(len(rows), tok), T=1.25)
        lp, lz, h, _ = c.forward()
        torch.cuda.synchronize()
        return sum(up[n] * t.double().cpu().numpy() for n, t in zip(up, (lp, lz, h)))

    at = rng.choice(V, B, replace=False)
    at[0] = tok
    f = {}
    for s in (-2, -1, 1, 2):
        rows = np.tile(x, (B, 1))
        rows[np.arange(B), at] += s * step
        f[s] = value(rows, valid)
    slope = (8 * (f[1] - f[-1]) - (f[2] - f[-2])) / (12 * step)
    c = Case(x[None], "f32", valid[:1], np.array([tok]), T=1.25)
    st = c.forward()[3]
    d = torch.zeros((1, V), device=DEV)
    ppv.ppv_token_logprobs_backward(c.logits, c.tokens, st, d, mask=c.mask, temperature=c.T,
                                    **{n: torch.full((1,), v, device=DEV) for n, v in up.items()})
    torch.cuda.synchronize()
    # the values are within 1e-6 of each other's truth here (96 terms), times (8 + 8 + 1 + 1) / (12 * step) = 6; and the differences are off
    # by step^4 / 30 of a fifth derivative below 1.25^-5 * 24 * 2.2 (those of a log-sum-exp and an entropy at weights below 0.2)
    bound = 6e-6 * 2.2 + step ** 4 / 30 * 0.33 * 24 * 2.2
    assert abs(slope - d.cpu().numpy()[0, at]).max() <= bound, abs(slope - d.cpu().numpy()[0, at]).max()


class Scored(torch.autograd.Function):
    """The two calls as an autograd function, as a training program wraps them."""

    @staticmethod
    def forward(ctx, logits, tokens, mask):
        B = logits.shape[0]
        lp, lz, h = (torch.empty(B, device=DEV) for _ in range(3))
        stats = torch.empty((B, ppv.PPV_LOGPROB_STATS), device=DEV)
        ppv.ppv_token_logprobs(logits, tokens, lp, mask=mask, logZ_valid=lz, entropy=h, stats=stats)
        ctx.save_for_backward(logits, tokens, mask, stats)
        return lp, lz, h

    @staticmethod
    def backward(ctx, g, z, h):
        logits, tokens, mask, stats = ctx.saved_tensors
        d = torch.empty_like(logits)
        ppv.ppv_token_logprobs_backward(logits, tokens, stats, d, mask=mask, d_logprobs=g.contiguous(), d_logZ_valid=z.contiguous(),
                                        d_entropy=h.contiguous())
        return d, None, None


def test_together_members_of_a_set():
    """As they are used: the masks of members' prefixes, the members scored under them, the scores' gradient through a linear layer, the
    alternatives at every position, and a drawn token's log probability."""
    cfg = W.scaled(W.CONFIGS["C2"], 3000, 8)
    S = W.make_constraint_set(cfg)
    V = cfg.vocab
    index = ppv.ppv_build_index(S.tokens, S.offsets, V)
    seqs = [S.seq(i) for i in range(12)]
    longest = max(len(s) for s in seqs)
    # packed positions: position j of member i asks for the valid set of its first j tokens
    pre = np.full((sum(map(len, seqs)), longest), W.PAD_TOKEN, np.int32)
    lens, tok, owner = [], [], []
    for i, s in enumerate(seqs):
        for j in range(len(s)):
            pre[len(lens), :j] = s[:j]
            lens.append(j)
            tok.append(s[j])
            owner.append(i)
    N = len(lens)
    mask = torch.zeros((N, index.n_words), dtype=torch.int32, device=DEV)
    ppv.ppv_next_token_mask(index, to_dev(pre), to_dev(np.array(lens, np.int32)), mask)
    g = torch.Generator(device=DEV).manual_seed(3)
    hidden = torch.randn((N, 24), generator=g, device=DEV)
    weight = (torch.randn((24, V), generator=g, device=DEV) * 0.5).requires_grad_()
    logits = hidden @ weight
    tokens = to_dev(np.array(tok, np.int32))
    lp, lz, h = Scored.apply(logits, tokens, mask)
    torch.cuda.synchronize()
    valid = unpack(mask.cpu().numpy(), V)
    x = logits.detach().cpu().numpy().astype(np.float64)
    ref = Scores(x, valid, np.array(tok), 1.0)
    assert np.isfinite(ref.logprobs).all()          # every token of a member is valid after its prefix
    check_values(lp.detach().cpu().numpy(), ref.logprobs, "logprobs")
    check_values(lz.detach().cpu().numpy(), ref.logZ, "logZ_valid")
    # a member's probability under the model is its probability under the constraint times its importance score
    score = torch.zeros(len(seqs), device=DEV, dtype=torch.float64).index_add_(0, to_dev(np.array(owner)), (lp + lz).detach().double())
    full = Scores(x, None, np.array(tok), 1.0).logprobs
    check_values(score.cpu().numpy(), np.bincount(owner, full, len(seqs)), "log P(member)", spread=float(longest * abs(full).max()))
    # the loss's gradient reaches the weights
    loss = -(lp + 0.3 * lz + 0.1 * h).sum() / N
    loss.backward()
    d, size = ref.gradient(np.full(N, -1 / N), np.full(N, -0.3 / N), np.full(N, -0.1 / N))
    want = hidden.cpu().double().numpy().T @ d
    room = abs(hidden.cpu().double().numpy()).T @ (WEIGHT * size + 2.0 ** -24 * abs(d)) + (N + 2) * 2.0 ** -24 * (abs(hidden.cpu().double().numpy()).T @ abs(d))
    assert (abs(weight.grad.cpu().double().numpy() - want) <= room + 1e-12).all()
    # alternatives, and the drawn token among the valid ones
    ids, lzv = torch.zeros(N, dtype=torch.int32, device=DEV), torch.zeros(N, device=DEV)
    ppv.constrained_sample(logits.detach(), mask, torch.rand(N, generator=g, device=DEV), ids, lzv)
    top, tops, mine = torch.zeros((N, 5), dtype=torch.int32, device=DEV), torch.zeros((N, 5), device=DEV), torch.zeros(N, device=DEV)
    ppv.ppv_top_logprobs(logits.detach(), 5, top, tops, mask=mask, tokens=ids, logprobs=mine)
    torch.cuda.synchronize()
    drawn = Scores(x, valid, ids.cpu().numpy(), 1.0)
    assert np.array_equal(top.cpu().numpy(), drawn.top(5)[0])
    check_values(tops.cpu().numpy(), drawn.top(5)[1], "alternatives")
    check_values(mine.cpu().numpy(), drawn.logprobs, "drawn token")
    check_values(lzv.cpu().numpy(), drawn.logZ, "constrained_sample's mass")
    index.free()


@pytest.mark.parametrize("B,V,dtype", [(3, 128256, "bf16"), (40, 9000, "f32"), (300, 700, "bf16")])
def test_captured_and_replayed(B, V, dtype):
    """All four calls in one graph, replayed on inputs that change between replays, beside eager calls of the same operators."""
    rng = np.random.default_rng(V)
    valid = hand_made_masks(B, V, rng)
    cases = [Case(rng.normal(0, 2, (B, V)), dtype, valid, tokens_for(valid, B, V, rng), seed=i) for i in range(3)]
    here = cases[0]
    up = {n: to_dev(v) for n, v in here.up.items()}
    f = lambda *s, **kw: torch.zeros(s, device=DEV, **kw)  # noqa: E731
    lp, lz, h, st = f(B), f(B), f(B), f(B, ppv.PPV_LOGPROB_STATS)
    d1, d2 = here.gradient_buffer(), here.gradient_buffer()
    lp2, ids, lps = f(B), f(B, 7, dtype=torch.int32), f(B, 7)
    logits = here.buf.clone()[:, :V]
    tokens = here.tokens.clone()

    def calls():
        ppv.ppv_token_logprobs(logits, tokens, lp, mask=here.mask, logZ_valid=lz, entropy=h, stats=st)
        ppv.ppv_token_logprobs_backward(logits, tokens, st, d1[:, :V], mask=here.mask, **up)
        ppv.ppv_token_logprobs_grad(logits, tokens, d2[:, :V], lp2, mask=here.mask, **up)
        ppv.ppv_top_logprobs(logits, 7, ids, lps, mask=here.mask)

    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    outs = (lp, lz, h, st, d1, d2, lp2, ids, lps)
    for c in (cases[1], cases[2], cases[0], cases[1]):
        logits.copy_(c.logits)
        tokens.copy_(c.tokens)
        calls()
        torch.cuda.synchronize()
        want = [t.clone() for t in outs]
        for t in (lp, lz, h, st, lp2, ids, lps):
            t.fill_(9)
        d1[:, :V] = 9
        d2[:, :V] = 9
        graph.replay()
        here.forward()          # eager work of the same kind beside it
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert torch.equal(a.nan_to_num(nan=123.0), b.nan_to_num(nan=123.0))
        check_values(lp.cpu().numpy(), c.ref.logprobs, "replayed")


def test_another_stream_than_the_current_one():
    rng = np.random.default_rng(9)
    B, V = 20, 6000
    c = Case(rng.normal(0, 2, (B, V)), "bf16", None, rng.integers(0, V, B))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    lp = torch.zeros(B, device=DEV)
    ppv.ppv_token_logprobs(c.logits, c.tokens, lp, stream=s)
    s.synchronize()
    check_values(lp.cpu().numpy(), c.ref.logprobs, "stream=")
    with torch.cuda.stream(s):
        ids, lps = torch.zeros((B, 3), dtype=torch.int32, device=DEV), torch.zeros((B, 3), device=DEV)
        ppv.ppv_top_logprobs(c.logits, 3, ids, lps)
    s.synchronize()
    assert np.array_equal(ids.cpu().numpy(), c.ref.top(3)[0])


def test_refusals_of_the_python_calls():
    """Shapes, types and alignments that do not fit are refused before anything is launched."""
    B, V = 4, 64
    x = torch.zeros((B, V), device=DEV)
    tok, f = torch.zeros(B, dtype=torch.int32, device=DEV), torch.zeros(B, device=DEV)
    st, mask = torch.zeros((B, 8), device=DEV), torch.zeros((B, 2), dtype=torch.int32, device=DEV)
    ids, lps = torch.zeros((B, 3), dtype=torch.int32, device=DEV), torch.zeros((B, 3), device=DEV)
    cases = [
        (TypeError, lambda: ppv.ppv_token_logprobs(x.half(), tok, f)),
        (TypeError, lambda: ppv.ppv_token_logprobs(x, tok.long(), f)),
        (TypeError, lambda: ppv.ppv_token_logprobs(x, tok.cpu(), f)),
        (TypeError, lambda: ppv.ppv_token_logprobs(x, tok, f.double())),
        (ValueError, lambda: ppv.ppv_token_logprobs(x.cpu(), tok, f)),
        (ValueError, lambda: ppv.ppv_token_logprobs(x.t(), tok, f)),
        (ValueError, lambda: ppv.ppv_token_logprobs(x, tok[:3], f)),
        (ValueError, lambda: ppv.ppv_token_logprobs(x, tok, f, mask=mask[:, :1])),
        (ValueError, lambda: ppv.ppv_token_logprobs(x, tok, f, stats=st[:, :6])),
        (ValueError, lambda: ppv.ppv_token_logprobs_backward(x, tok, st, x[:, :32], d_logprobs=f)),
        (ValueError, lambda: ppv.ppv_token_logprobs_backward(x, tok, st, x.bfloat16(), d_logprobs=f)),
        (ValueError, lambda: ppv.ppv_top_logprobs(x, 4, ids, lps)),
        (ValueError, lambda: ppv.ppv_top_logprobs(x, 1 << 40, ids, lps)),
    ]
    for kind, call in cases:
        with pytest.raises(kind):
            call()
    wide = torch.zeros((B + 1, 2 * V), device=DEV)
    for status, call in [
        (-1, lambda: ppv.ppv_token_logprobs(x, None, f)),
        (-1, lambda: ppv.ppv_token_logprobs(x, tok)),
        (-1, lambda: ppv.ppv_token_logprobs(x, tok, f, temperature=0.0)),
        (-1, lambda: ppv.ppv_token_logprobs(wide[:B, 1:V + 1], tok, f)),                 # rows that start off 16 bytes
        (-1, lambda: ppv.ppv_token_logprobs(torch.zeros((B, 62), device=DEV), tok, f, mask=mask)),
        (-1, lambda: ppv.ppv_token_logprobs_backward(wide[:B, :V], tok, st, wide[1:, :V], d_logprobs=f)),    # overlaps
        (-1, lambda: ppv.ppv_token_logprobs_grad(wide[:B, :V], tok, wide[:B, 4:V + 4], d_logprobs=f)),
        (-1, lambda: ppv.ppv_token_logprobs_grad(x, None, torch.zeros_like(x), d_logprobs=f)),
        (-4, lambda: ppv.ppv_top_logprobs(x, 129, ids.new_zeros((B, 129)), lps.new_zeros((B, 129)))),
        (-1, lambda: ppv.ppv_top_logprobs(x, 0, ids[:, :0].contiguous(), lps[:, :0].contiguous())),
        (-1, lambda: ppv.ppv_top_logprobs(x, 3, ids, lps, logprobs=f)),
        (-4, lambda: ppv.ppv_token_logprobs(torch.zeros((1, 262148), device=DEV), tok[:1], f[:1])),
    ]:
        with pytest.raises(ppv.PPVError) as e:
            call()
        assert e.value.status == status
    for call in (lambda z: ppv.ppv_token_logprobs(z, tok[:0], f[:0]), lambda z: ppv.ppv_top_logprobs(z, 3, ids[:0], lps[:0])):
        call(x[:0])         # no rows: nothing to do

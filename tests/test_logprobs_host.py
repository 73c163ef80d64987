"""The calls on given tokens without a GPU: arguments that are refused before anything is launched, and the plain implementation that
the GPU tests hold them to, against automatic differentiation and differences."""
import ctypes as C

import numpy as np
import pytest
import torch

from logprobs_oracle import Scores, pack, unpack

EINVAL, ERANGE = -1, -4
NEVER = C.c_void_p(4096)     # never dereferenced: the checks come first
FAR = C.c_void_p(1 << 30)


@pytest.fixture(scope="module")
def lib():
    from paper_2504_09135_amd import binding
    return binding.load_library()


def test_token_logprobs_refusals(lib):
    def call(logits=NEVER, dt=0, stride=8, mask=None, tokens=NEVER, B=1, V=8, lp=NEVER, lz=None, h=None, st=None, T=1.0):
        return lib.ppv_token_logprobs(logits, dt, stride, mask, tokens, B, V, lp, lz, h, st, T, None)
    for bad in (dict(logits=None), dict(dt=2), dict(dt=-1), dict(stride=7), dict(stride=10), dict(dt=1, stride=12), dict(B=-1), dict(V=0), dict(V=-3),
                dict(lp=None), dict(tokens=None), dict(T=0.0), dict(T=-1.0), dict(T=float("inf")), dict(T=float("nan")),
                dict(logits=C.c_void_p(4100)), dict(st=C.c_void_p(4104))):
        assert call(**bad) == EINVAL, bad
    assert call(V=262145, stride=262152) == ERANGE
    assert call(B=0) == 0 and call(B=0, logits=None) == 0
    assert call(B=0, T=0.0) == EINVAL


def test_gradient_refusals(lib):
    def backward(logits=NEVER, dt=0, stride=8, tokens=NEVER, st=NEVER, g=NEVER, B=4, V=8, d=FAR, d_stride=8, T=1.0):
        return lib.ppv_token_logprobs_backward(logits, dt, stride, None, tokens, st, g, None, None, B, V, d, d_stride, T, None)

    def grad(logits=NEVER, dt=0, stride=8, tokens=NEVER, g=NEVER, B=4, V=8, lp=NEVER, d=FAR, d_stride=8, T=1.0):
        return lib.ppv_token_logprobs_grad(logits, dt, stride, None, tokens, g, None, None, B, V, lp, None, None, d, d_stride, T, None)
    for call in (backward, grad):
        for bad in (dict(logits=None), dict(dt=7), dict(stride=4), dict(B=-1), dict(V=0), dict(d=None), dict(d_stride=7), dict(d_stride=9),
                    dict(d=C.c_void_p((1 << 30) + 4)), dict(tokens=None), dict(T=0.0),
                    dict(d=C.c_void_p(4096 + 32)), dict(d=C.c_void_p(4096 - 16)), dict(d=NEVER, d_stride=16)):   # overlaps that are not the logits
            assert call(**bad) == EINVAL, bad
        assert call(V=262145, stride=262152, d_stride=262152) == ERANGE
        assert call(B=0) == 0
    # results over the upstream gradients that other workgroups of the row may still read
    for lp in (NEVER, C.c_void_p(4096 + 12), C.c_void_p(4096 - 12)):
        assert grad(g=NEVER, lp=lp) == EINVAL
    assert backward(st=None) == EINVAL and backward(st=C.c_void_p(4100)) == EINVAL


def test_top_refusals(lib):
    def call(logits=NEVER, dt=0, stride=8, tokens=None, B=1, V=8, k=3, ids=NEVER, lps=NEVER, lp=None, T=1.0):
        return lib.ppv_top_logprobs(logits, dt, stride, None, tokens, B, V, k, ids, lps, lp, None, T, None)
    for bad in (dict(logits=None), dict(dt=3), dict(stride=6), dict(B=-2), dict(V=0), dict(k=0), dict(k=-1), dict(ids=None), dict(lps=None),
                dict(lp=NEVER), dict(T=float("nan"))):
        assert call(**bad) == EINVAL, bad
    assert call(k=129) == ERANGE and call(V=262145, stride=262152) == ERANGE
    assert call(B=0) == 0 and call(B=0, k=0) == EINVAL


def test_constants_agree_with_the_header():
    import os
    import re
    from paper_2504_09135_amd import binding
    hdr = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "ppv.h")).read()
    for name in ("PPV_LOGPROB_STATS", "PPV_TOP_MAX"):
        assert int(re.search(rf"#define {name} (\d+)", hdr).group(1)) == getattr(binding, name)


def test_plain_implementation():
    """The formulas of the oracle, against autograd in 64 bits and central differences."""
    rng = np.random.default_rng(0)
    B, V, T = 6, 23, 0.8
    x = rng.normal(0, 2, (B, V))
    valid = rng.random((B, V)) < 0.5
    valid[:, 3] = True
    valid[4] = False
    tok = np.array([3, 3, -1, 3, 3, int(np.nonzero(~valid[5])[0][0])])
    assert np.array_equal(unpack(pack(valid), V), valid)
    g, z, h = rng.normal(size=(3, B))

    def value(x):
        s = Scores(x, valid, tok, T)
        fin = lambda a: np.where(np.isfinite(a), a, 0.0)  # noqa: E731
        return (g * fin(s.logprobs) + z * fin(s.logZ) + h * s.entropy).sum()
    d = Scores(x, valid, tok, T).gradient(g, z, h)[0]
    assert (d[2] == 0).all() and (d[4] == 0).all()
    for b in range(B):
        for v in range(V):
            e = np.zeros_like(x)
            e[b, v] = 1e-5
            assert abs((value(x + e) - value(x - e)) / 2e-5 - d[b, v]) < 1e-8
    rows = [0, 1, 3]
    t = torch.tensor(x[rows], requires_grad=True)
    l = t / T
    lq = torch.log_softmax(l.masked_fill(~torch.tensor(valid[rows]), -torch.inf), 1)
    lz = torch.logsumexp(l.masked_fill(~torch.tensor(valid[rows]), -torch.inf), 1) - torch.logsumexp(l, 1)
    ent = -torch.where(torch.tensor(valid[rows]), lq.exp() * lq.clamp(min=-1e30), 0.0).sum(1)
    s = Scores(x, valid, tok, T)
    assert np.allclose(lq[:, 3].detach().numpy(), s.logprobs[rows], atol=1e-12) and np.allclose(lz.detach().numpy(), s.logZ[rows], atol=1e-12)
    assert np.allclose(ent.detach().numpy(), s.entropy[rows], atol=1e-12)
    (torch.tensor(g[rows]) * lq[:, 3] + torch.tensor(z[rows]) * lz + torch.tensor(h[rows]) * ent).sum().backward()
    assert np.allclose(t.grad.numpy(), d[rows], atol=1e-12)
    ids, lps = s.top(V + 2)
    assert (ids[4] == -1).all() and (ids[2] == -1).all()
    n = int(valid[0].sum())
    assert (np.sort(ids[0, :n]) == np.nonzero(valid[0])[0]).all() and (np.diff(lps[0, :n]) <= 0).all() and (ids[0, n:] == -1).all()

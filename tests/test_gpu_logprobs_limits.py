"""The calls on given tokens at the limits of what they take."""
import numpy as np
import pytest
import torch

from paper_2504_09135_amd import binding as ppv

from gpu_helpers import DEV, to_dev, tuning
from logprobs_oracle import Scores, check_values
from test_gpu_logprobs import Case, hand_made_masks, tokens_for

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


@pytest.mark.parametrize("value", [float("inf"), float("nan")])
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

"""The calls on given tokens at the limits of what they take."""
import numpy as np
import pytest
import torch

from paper_2504_09135_amd import binding as ppv

from gpu_helpers import DEV
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

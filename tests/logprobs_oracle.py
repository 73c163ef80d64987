"""Plain 64-bit implementation of the log probabilities of given tokens, their gradient and the most probable tokens, and the bounds
that the library's 32-bit results are held to."""
import numpy as np
import torch

HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}      # a rounding to the type, relative to the value

# An exponent y = (x - m) log2(e) / T is off by at most three roundings, 3 * 2^-24 |y|; weighted by 2^y the exponents of a row average at
# most log2(V) <= 18, so that a sum of exponentials is off by at most 18 ln 2 * 3 * 2^-24 = 2.2e-6, relative; adding up to 256 of
# them in a lane, and 64 lanes and 16 wavefronts in trees, by at most (256 + 10) * 2^-24 = 1.6e-5.
SUM = 2e-5
# What is multiplied by 1 / T (a rounded number) and added once more: four roundings of the result
VALUE = 2.0 ** -22
# A weight is off by its sum's error and its own exponent's (3 * 2^-24 |y| with |y| <= 160 where it is not 0 in fp32: 2e-5), and the
# products it enters by four roundings more
WEIGHT = SUM + 2e-5 + 4 * 2.0 ** -24


def unpack(words, V):
    """int32 [B, ceil(V / 32)] -> bool [B, V]"""
    bits = np.unpackbits(np.ascontiguousarray(words).view(np.uint8).reshape(words.shape[0], -1), axis=1, bitorder="little")
    return bits[:, :V].astype(bool)


def pack(valid):
    B, V = valid.shape
    return np.packbits(np.pad(valid, ((0, 0), (0, -V % 32))), axis=1, bitorder="little").view(np.int32).reshape(B, -1)


def log_softmax(l, valid):
    """log q over the valid tokens (-inf elsewhere, and all over a row without mass); the largest of them, the log of the sum relative to it"""
    l = np.where(valid, l, -np.inf)
    m = l.max(1, keepdims=True)
    some = np.isfinite(m)
    m = np.where(some, m, 0.0)
    with np.errstate(divide="ignore"):
        log_s = np.log(np.exp(l - m).sum(1, keepdims=True))
    return np.where(some, (l - m) - np.where(some, log_s, 0.0), -np.inf), m[:, 0], log_s[:, 0]


class Scores:
    """logits float64 [B, V] (values of the type they were given in), valid bool [B, V] or None, tokens int [B] or None"""

    def __init__(self, logits, valid, tokens, T):
        B, V = logits.shape
        self.T, self.V, self.masked = T, V, valid is not None
        self.valid = np.ones((B, V), bool) if valid is None else valid
        self.tokens = None if tokens is None else tokens.astype(np.int64)
        self.out = np.zeros(B, bool) if tokens is None else self.tokens < 0
        l = logits / T
        self.log_q, mv, zv = log_softmax(l, self.valid)
        self.log_p, m, z = log_softmax(l, np.ones((B, V), bool))
        self.q, self.p = np.exp(self.log_q), np.exp(self.log_p)
        self.mass = np.isfinite(zv)
        with np.errstate(invalid="ignore"):
            qlogq = np.where(self.q > 0, self.q * self.log_q, 0.0)
            self.entropy = np.where(self.out, 0.0, -qlogq.sum(1))
            logz = np.where(self.mass, (mv - m) + (zv - z) if self.masked else 0.0, -np.inf)
        self.logZ = np.where(self.out, 0.0, logz)
        self.hit = np.zeros((B, V), bool)
        self.logprobs = None
        if tokens is not None:
            inside = (self.tokens >= 0) & (self.tokens < V)
            rows = np.nonzero(inside)[0]
            self.hit[rows, self.tokens[rows]] = True
            lp = np.full(B, -np.inf)
            lp[rows] = self.log_q[rows, self.tokens[rows]]
            self.logprobs = np.where(self.out, 0.0, lp)

    def gradient(self, g, z, h):
        """d_logits and the sum of the sizes of its terms, for upstream gradients (None: 0).  An exponential below 2^-126 (of
        fp32's normal numbers, the smallest) is 0 to the library.  They are taken relative to the sum of the weights, or, of the valid
        tokens, to that of all where the valid ones are 2^-24 of it or more: a weight below 2^-102 may be 0, and what it would have been
        multiplied by is missing: at most 2^-102 times |g| + 2 |z| + |h| (126 ln 2 + log V + entropy), over T, which is added to the size
        over the tolerance that it is multiplied by.  (The sum that weights are relative to is 1 to within a factor of 2.)"""
        B = len(self.entropy)
        zero = np.zeros((B, 1))
        g, z, h = (zero if a is None else a.astype(np.float64)[:, None] for a in (g, z, h))
        if self.logprobs is None:
            g = zero
        else:
            g = np.where(np.isfinite(self.logprobs)[:, None], g, 0.0)
        if not self.masked:
            z = zero
        logq = np.where(self.q > 0, self.log_q, 0.0)
        H = self.entropy[:, None]
        d = g * (self.hit - self.q) + z * (self.q - self.p) - h * self.q * (logq + H)
        size = abs(g) * (self.hit + self.q) + abs(z) * (self.q + self.p) + abs(h) * self.q * (abs(logq) + H + 1.0)
        keep = (~self.out & self.mass)[:, None]
        size = size + 2.0 ** -101 / WEIGHT * (abs(g) + 2 * abs(z) + abs(h) * (126 * np.log(2) + np.log(self.V) + H))
        return np.where(keep, d, 0.0) / self.T, np.where(keep, size, 0.0) / self.T

    def top(self, k):
        """ids [B, k] and log q [B, k], most probable first, equal logits in increasing token id"""
        B = len(self.entropy)
        ids, lps = np.full((B, k), -1, np.int64), np.full((B, k), -np.inf)
        for b in range(B):
            if self.out[b]:
                continue
            c = np.nonzero(np.isfinite(self.log_q[b]))[0]
            c = c[np.argsort(-self.log_q[b, c], kind="stable")][:k]     # (equal logits have equal log q)
            ids[b, :len(c)], lps[b, :len(c)] = c, self.log_q[b, c]
        return ids, lps


def check_values(got, want, what, spread=0.0):
    """fp32 results that are a logarithm of sums plus a difference of logits over T"""
    got = got.astype(np.float64)
    fine = np.isfinite(want)
    assert np.array_equal(got[~fine], want[~fine]), (what, got[~fine], want[~fine])
    got, want = got[fine], want[fine]
    off = abs(got - want) - (SUM + VALUE * (abs(want) + spread))
    assert not off.size or off.max() <= 0, (what, off.max(), np.argmax(off), got[np.argmax(off)], want[np.argmax(off)])


def check_gradient(got, want, size, dtype, what):
    off = abs(got.astype(np.float64) - want) - (WEIGHT * size + HALF_STEP[dtype] * abs(want) * 1.001 + 1e-37)
    assert off.max() <= 0, (what, off.max(), np.unravel_index(np.argmax(off), off.shape))


def bf16(x):
    """float -> the nearest bf16, as float64"""
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).bfloat16().double().numpy()

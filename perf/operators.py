"""Log probabilities of given tokens, their gradient, and top alternatives, as cases that can be timed and compared.

A case is one call on a batch of logits rows [B, V], restricted to each row's valid set where the case has a mask:

  score     ppv_token_logprobs: log probability of the row's token, log of the valid mass, entropy
  backward  ppv_token_logprobs_backward: the gradient of these with respect to the logits, from the statistics that score leaves
  grad      ppv_token_logprobs_grad: both in one call, for training whose weights are known before the call
  top       ppv_top_logprobs: the k most probable valid tokens with their log probabilities, the given token's, the entropy

With l = logits / T, p = softmax over all tokens, q = softmax over the valid ones and t the row's token:

  logprob = log q_t,   logZ_valid = log sum_valid p,   entropy = -sum q log q
  d_l     = d_logprob (1[v = t] - q) + d_logZ_valid (q - p) - d_entropy q (log q + entropy),   d_logits = d_l / T

A row whose token is negative is left out (padding, an idle slot): zeros, and no alternatives.
"""
import math

import torch

own = False     # true: the framework's kernels; false: the plain form

DEVICE = "cuda:0"
SIGMA = 2.5             # standard deviation of the logits
LIFT = 6.0              # by which the given token's logit lies higher, as a trained model's does
STATS = 8               # words of a row's statistics
ELEMENTS = 2.5e8        # logits of a drawn case, at most; half as many where gradients are written
FEW = 64                # continuations of an ordinary prefix, at most


def new_case(op, vocab, batch, dtype, mask="none", temperature=1.0, left_out=0.0, k=0, mass=True, entropy=True):
    return {"op": op, "vocab": vocab, "batch": batch, "dtype": dtype, "mask": mask, "temperature": temperature,
            "left_out": left_out, "k": k, "mass": mass and mask != "none", "entropy": entropy}


def listed():
    return [
        # one interactive request: the drawn token's log probability, nothing but latency
        dict(new_case("score", 128_256, 1, "bf16"), name="score B=1 V=128256"),
        # item codes under their codebooks' masks, a large batch of short rows
        dict(new_case("score", 1_024, 4_096, "f32", "codes"), name="score B=4096 V=1024 f32"),
        # members scored under the constraint, the largest vocabulary and batch
        dict(new_case("score", 256_000, 1_024, "bf16", "prefix"), name="score B=1024 V=256000"),
        # the smallest training step: sixteen positions over item codes
        dict(new_case("backward", 1_024, 16, "f32", "codes"), name="backward B=16 V=1024 f32"),
        # a training batch under the constraint, all three gradients
        dict(new_case("backward", 32_000, 2_048, "bf16", "prefix"), name="backward B=2048 V=32000"),
        # policy gradient with an entropy bonus over the whole vocabulary
        dict(new_case("backward", 128_256, 1_024, "bf16"), name="backward B=1024 V=128256"),
        # a short training batch, loss and gradient at once
        dict(new_case("grad", 32_000, 64, "bf16", "prefix"), name="grad B=64 V=32000"),
        # cross entropy over many positions
        dict(new_case("grad", 32_000, 4_096, "bf16", entropy=False), name="grad B=4096 V=32000"),
        # a padded batch with an odd vocabulary, fp32 logits and a temperature
        dict(new_case("grad", 50_265, 500, "f32", "prefix", 0.7, 0.15), name="grad B=500 V=50265 f32"),
        # one request that asks for five alternatives
        dict(new_case("top", 128_256, 1, "bf16", k=5), name="top k=5 B=1 V=128256"),
        # a serving batch under broad masks, idle slots among its rows, odd vocabulary
        dict(new_case("top", 50_265, 128, "f32", "broad", 0.7, 0.1, 20), name="top k=20 B=128 V=50265 f32"),
        # a large batch's twenty alternatives over the largest vocabulary
        dict(new_case("top", 256_000, 1_024, "bf16", k=20), name="top k=20 B=1024 V=256000"),
    ]


def log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["score", "backward", "grad", "top"])
    dtype = rng.choice(["bf16", "f32"])
    vocab = log_int(rng, 300, 256_000)
    most = ELEMENTS / (2 if op in ("backward", "grad") else 1) / (2 if dtype == "f32" else 1)
    batch = log_int(rng, 1, max(1, min(8_192, int(most / vocab))))
    mask = rng.choice(["none", "none", "prefix", "broad"] + (["codes"] if vocab < 9_000 else []))
    k = log_int(rng, 1, 128) if op == "top" else 0
    temperature = 1.0 if rng.random() < 0.6 else round(rng.uniform(0.5, 2.0), 2)
    left_out = 0.0 if rng.random() < 0.6 else round(rng.uniform(0.02, 0.3), 2)
    return new_case(op, vocab, batch, dtype, mask, temperature, left_out, k, rng.random() < 0.6, rng.random() < 0.6)


# ------------------------------------------------------------------------------------------ inputs
def valid_sets(c, first, n, g):
    """bool [n, V]: the valid sets of rows first .. first + n - 1."""
    V = c["vocab"]
    rows = torch.arange(first, first + n, device=DEVICE)
    if c["mask"] == "codes":        # position l of a code has the tokens of codebook l
        per = max(1, V // 4)
        return torch.arange(V, device=DEVICE)[None, :] // per == (rows % 4)[:, None]
    if c["mask"] == "broad":        # a quarter of the vocabulary
        return torch.rand((n, V), generator=g, device=DEVICE) < 0.25
    # prefixes of members: a few continuations, and one row in eight near the root with many
    few = torch.randint(0, V, (n, FEW), generator=g, device=DEVICE)
    few = torch.where(torch.arange(FEW, device=DEVICE)[None, :] <= rows[:, None] % FEW, few, few[:, :1])
    valid = torch.zeros((n, V), dtype=torch.bool, device=DEVICE)
    valid.scatter_(1, few, True)
    root = rows[:, None] % 8 == 0
    return valid | (root & (torch.rand((n, V), generator=g, device=DEVICE) < 0.1))


def packed(valid):
    """bool [n, V] -> int32 [n, ceil(V / 32)], token v in bit v & 31 of word v >> 5."""
    n, V = valid.shape
    bits = torch.nn.functional.pad(valid, (0, -V % 32)).view(n, -1, 32).to(torch.int32)
    return (bits << torch.arange(32, device=DEVICE, dtype=torch.int32)).sum(2, dtype=torch.int32)


def prepare(case, seed):
    c = case
    B, V = c["batch"], c["vocab"]
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16
    stride = (V + 7) // 8 * 8       # rows start on 16-byte boundaries
    step = max(1, 60_000_000 // V)
    s = {"case": c, "logits": torch.empty((B, stride), dtype=dt, device=DEVICE)[:, :V], "mask": None}
    tokens = torch.randint(0, V, (B,), generator=g, device=DEVICE)
    if c["mask"] != "none":
        s["mask"] = torch.empty((B, (V + 31) // 32), dtype=torch.int32, device=DEVICE)
    for b in range(0, B, step):
        n = min(step, B - b)
        x = torch.randn((n, V), generator=g, device=DEVICE) * SIGMA
        if c["mask"] != "none":
            valid = valid_sets(c, b, n, g)
            s["mask"][b:b + n] = packed(valid)
            # the given token: the first valid one from a random place on, or the first of all
            behind = valid & (torch.arange(V, device=DEVICE)[None, :] >= tokens[b:b + n, None])
            tokens[b:b + n] = torch.where(behind.any(1), behind.int().argmax(1), valid.int().argmax(1))
        x.scatter_add_(1, tokens[b:b + n, None], torch.full((n, 1), LIFT, device=DEVICE))
        s["logits"][b:b + n] = x.to(dt)
    out = torch.rand((B,), generator=g, device=DEVICE) < c["left_out"]
    s["tokens"] = torch.where(out, -1, tokens).to(torch.int32)
    for name in ("logprobs", "logZ_valid", "entropy"):      # upstream gradients, and room for the results
        s["d_" + name] = torch.randn((B,), generator=g, device=DEVICE)
        s[name] = torch.empty((B,), device=DEVICE)
    if not c["mass"]:
        s["d_logZ_valid"] = None
    if not c["entropy"]:
        s["d_entropy"] = None
    if c["op"] == "backward":       # as the forward call has left them
        s["stats"] = torch.empty((B, STATS), device=DEVICE)
        for b in range(0, B, step):
            x, valid = rows_of(s, slice(b, b + step), torch.float64)
            s["stats"][b:b + step] = statistics(x, valid, s["tokens"][b:b + step], c["temperature"]).float()
    if c["op"] in ("backward", "grad"):
        s["d_logits"] = torch.zeros((B, stride), dtype=dt, device=DEVICE)[:, :V]
    if c["op"] == "top":
        s["top_ids"] = torch.empty((B, c["k"]), dtype=torch.int32, device=DEVICE)
        s["top_logprobs"] = torch.empty((B, c["k"]), device=DEVICE)
    return s


def rows_of(s, rows, dtype):
    x = s["logits"][rows].to(dtype)
    if s["mask"] is None:
        return x, None
    words = s["mask"][rows]
    bits = (words[:, :, None] >> torch.arange(32, device=DEVICE, dtype=torch.int32)) & 1
    return x, bits.view(x.shape[0], -1)[:, :x.shape[1]].bool()


def statistics(x, valid, tokens, T):
    """[B, STATS]: largest logit, sum of exp((l - largest) / T), the same over the valid tokens, entropy, log probability."""
    xv = x if valid is None else torch.where(valid, x, -torch.inf)
    m, mv = x.amax(1), xv.amax(1)
    z, zv = ((x - m[:, None]) / T).exp().sum(1), ((xv - mv[:, None]) / T).exp()
    sv = zv.sum(1)
    y = (xv - mv[:, None]) / T
    entropy = sv.log() - torch.where(zv > 0, y * zv, 0.0).sum(1) / sv
    logprob = (xv.gather(1, tokens.clamp(min=0).long()[:, None])[:, 0] - mv) / T - sv.log()
    zero = torch.zeros_like(m)
    got = torch.stack([m, z, mv, sv, entropy, logprob, zero, zero], 1)
    return torch.where(tokens[:, None] < 0, 0.0, got)


# ------------------------------------------------------------------------------------------ one pass
def run(state):
    return run_own(state) if own else run_plain(state)


def run_own(s):
    from paper_2504_09135_amd import binding as ppv

    c, T = s["case"], s["case"]["temperature"]
    lz = s["logZ_valid"] if c["mass"] else None
    h = s["entropy"] if c["entropy"] else None
    d = dict(d_logprobs=s["d_logprobs"], d_logZ_valid=s["d_logZ_valid"], d_entropy=s["d_entropy"])
    if c["op"] == "score":
        ppv.ppv_token_logprobs(s["logits"], s["tokens"], s["logprobs"], mask=s["mask"], logZ_valid=lz, entropy=h,
                               temperature=T)
        return {"logprobs": s["logprobs"], "logZ_valid": lz, "entropy": h}
    if c["op"] == "backward":
        ppv.ppv_token_logprobs_backward(s["logits"], s["tokens"], s["stats"], s["d_logits"], mask=s["mask"], temperature=T, **d)
        return {"d_logits": s["d_logits"]}
    if c["op"] == "grad":
        ppv.ppv_token_logprobs_grad(s["logits"], s["tokens"], s["d_logits"], s["logprobs"], mask=s["mask"], logZ_valid=lz,
                                    entropy=h, temperature=T, **d)
        return {"logprobs": s["logprobs"], "logZ_valid": lz, "entropy": h, "d_logits": s["d_logits"]}
    ppv.ppv_top_logprobs(s["logits"], c["k"], s["top_ids"], s["top_logprobs"], mask=s["mask"], tokens=s["tokens"],
                         logprobs=s["logprobs"], entropy=h, temperature=T)
    return {"logprobs": s["logprobs"], "entropy": h, "top_ids": s["top_ids"], "top_logprobs": s["top_logprobs"]}


def run_plain(s):
    c, T = s["case"], s["case"]["temperature"]
    out = s["tokens"] < 0
    x, valid = rows_of(s, slice(None), torch.float32)
    xv = x if valid is None else torch.where(valid, x, -torch.inf)
    t = s["tokens"].clamp(min=0).long()[:, None]
    if c["op"] == "backward":
        m, z, mv, sv, entropy, _ = s["stats"][:, :6].unbind(1)
        return {"d_logits": gradient(s, x, xv, t, out, m, z, mv, sv, entropy)}
    mv = xv.amax(1)
    y = (xv - mv[:, None]) / T
    e = y.exp()
    sv = e.sum(1)
    r = {"logprobs": torch.where(out, 0.0, y.gather(1, t)[:, 0] - sv.log()), "logZ_valid": None, "entropy": None}
    m = z = None
    if c["mass"]:
        m = x.amax(1)
        z = ((x - m[:, None]) / T).exp().sum(1)
        r["logZ_valid"] = torch.where(out, 0.0, (mv - m) / T + sv.log() - z.log())
    if c["entropy"]:
        entropy = sv.log() - torch.where(e > 0, y * e, 0.0).sum(1) / sv
        r["entropy"] = torch.where(out, 0.0, entropy)
    if c["op"] == "grad":
        r["d_logits"] = gradient(s, x, xv, t, out, m, z, mv, sv, entropy if c["entropy"] else None)
    if c["op"] == "top":
        del r["logZ_valid"]
        # logits as whole numbers of the same order, and below them the token, so that of equal ones the lowest comes first
        bits = (xv + 0.0).view(torch.int32).long()
        order = torch.where(bits < 0, -(bits & 0x7FFFFFFF), bits)
        key = (order << 18) | (0x3FFFF - torch.arange(x.shape[1], device=DEVICE))
        top = key.topk(min(c["k"], x.shape[1]), dim=1).values
        top = torch.nn.functional.pad(top, (0, c["k"] - top.shape[1]), value=-(1 << 62))
        ids = 0x3FFFF - (top & 0x3FFFF)
        logp = y.gather(1, ids.clamp(max=x.shape[1] - 1)) - sv.log()[:, None]
        none = out[:, None] | (top < -(0x7F800000 << 18)) | (logp == -torch.inf)
        r["top_ids"] = torch.where(none, -1, ids).to(torch.int32)
        r["top_logprobs"] = torch.where(none, -torch.inf, logp)
    return r


def gradient(s, x, xv, t, out, m, z, mv, sv, entropy):
    T = s["case"]["temperature"]
    y = (xv - mv[:, None]) / T
    q = y.exp() / sv[:, None]
    g = -s["d_logprobs"][:, None] * q
    g.scatter_add_(1, t, s["d_logprobs"][:, None])
    if s["d_logZ_valid"] is not None:
        p = ((x - m[:, None]) / T).exp() / z[:, None]
        g += s["d_logZ_valid"][:, None] * (q - p)
    if s["d_entropy"] is not None:
        log_q = y - sv.log()[:, None]
        g -= s["d_entropy"][:, None] * torch.where(q > 0, q * (log_q + entropy[:, None]), 0.0)
    return torch.where(out[:, None], 0.0, g / T).to(s["logits"].dtype)


# ------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = case
    rows = c["batch"] * (1.0 - c["left_out"])
    e = 4 if c["dtype"] == "f32" else 2
    n = rows * c["vocab"]
    writes = c["batch"] * c["vocab"] * e if c["op"] in ("backward", "grad") else 0
    mask = n / 8 if c["mask"] != "none" else 0
    small = c["batch"] * (4 * 6 + 8 * c["k"])
    ops = {"score": 5, "backward": 7, "grad": 11, "top": 6}[c["op"]]      # difference, exp, sums, comparison; the gradient's products
    return {"bytes": n * e + writes + mask + small, "flops": n * ops}


# ------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    """By log-probabilities row block by row block: log_p = l - logsumexp(l), log_q = l - logsumexp(valid l)."""
    s = prepare(case, seed)
    c, V = case, case["vocab"]
    parts = []
    step = max(1, 40_000_000 // V)
    for b in range(0, c["batch"], step):
        rows = slice(b, b + step)
        l = s["logits"][rows].double() / c["temperature"]
        tok = s["tokens"][rows].long()
        live = tok >= 0
        col = torch.arange(V, device=DEVICE)
        ok = torch.ones_like(l, dtype=torch.bool)
        if s["mask"] is not None:
            ok = (s["mask"][rows][:, col >> 5] >> (col & 31).int()) & 1 == 1
        log_q = torch.where(ok, l, -torch.inf)
        log_q = log_q - torch.logsumexp(log_q, 1, keepdim=True)
        log_p = l - torch.logsumexp(l, 1, keepdim=True)
        q = log_q.exp()
        plogp = torch.where(q > 0, q * log_q, 0.0)
        H = -plogp.sum(1)
        zero = torch.zeros_like(H)
        hit = col[None, :] == tok[:, None]
        r = {"logprobs": torch.where(live, torch.where(hit, log_q, -torch.inf).amax(1), zero)}
        if c["mass"] and c["op"] != "top":
            r["logZ_valid"] = torch.where(live, torch.logsumexp(torch.where(ok, log_p, -torch.inf), 1), zero)
        if c["entropy"]:
            r["entropy"] = torch.where(live, H, zero)
        if c["op"] in ("backward", "grad"):
            up = {n: None if s["d_" + n] is None else s["d_" + n][rows].double()[:, None] for n in ("logprobs", "logZ_valid", "entropy")}
            g = up["logprobs"] * (hit.double() - q)
            if up["logZ_valid"] is not None:
                g = g + up["logZ_valid"] * (q - log_p.exp())
            if up["entropy"] is not None:
                g = g - up["entropy"] * (plogp + q * H[:, None])
            r["d_logits"] = torch.where(live[:, None], g / c["temperature"], 0.0)
        if c["op"] == "top":
            best = log_q.topk(min(c["k"], V), dim=1).values
            best = torch.nn.functional.pad(best, (0, c["k"] - best.shape[1]), value=-math.inf)
            r["top_logprobs"] = torch.where(live[:, None], best, -torch.inf)
        parts.append(r)
    if c["op"] == "backward":
        return {"d_logits": torch.cat([r["d_logits"] for r in parts])}
    got = {name: torch.cat([r[name] for r in parts]) for name in parts[0]}
    if c["op"] == "top":
        got["top_ids"] = None
    return got

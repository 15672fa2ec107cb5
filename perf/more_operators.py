"""Measured cases of the target model's output side: the output projection in 8-bit integers, the log
probabilities of given tokens with entropy and best alternatives, and the gradient of both.

``run`` computes them with plain torch operations, or, with ``own`` set, through the library's
entry points; ``exact`` evaluates the definitions in 64 bits.

Definitions, for a row z of V logits (T the temperature, p = softmax(z / T)):
  log probability of token t    ln p_t, and 0 for an id outside [0, V) (a position without a token)
  entropy                       -sum_v p_v ln p_v
  alternatives                  the k largest logits, lower id first among equal ones, as ids and ln p
  gradient of sum_j g_j ln p_{t_j} + h * entropy, by z
and for a token's hidden state x and a weight row w_v in 8 bits with its scale u_v:
  a = max |x|, s = a / 127, r = 127 / a, q = rint(x * r), each one operation in 32 bits
  logit v = (sum_k q_k w_vk) * s * u_v + b_v
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


# ------------------------------------------------------------------------------------------ cases

def listed():
    return [
        # one token of one user, with the ten alternatives that a drafter's top-k takes too
        {"name": "logprobs_one_token", "op": "logprobs", "rows": 1, "V": 151936, "pad": 0, "dtype": "bf16", "J": 1,
         "k": 10, "T": 1.0, "masked": False, "pool": 0},
        # what 64 verified trees of 60 nodes emitted: the rows of the accepted paths out of all rows
        {"name": "logprobs_emitted", "op": "logprobs", "rows": 448, "V": 151936, "pad": 0, "dtype": "bf16", "J": 1,
         "k": 5, "T": 0.6, "masked": False, "pool": 3840},
        # candidates of every row of a batch of trees, padded rows
        {"name": "logprobs_candidates", "op": "logprobs", "rows": 3840, "V": 151936, "pad": 128, "dtype": "bf16", "J": 4,
         "k": 0, "T": 1.0, "masked": False, "pool": 0},
        # a smaller vocabulary in 32 bits, some tokens forbidden, odd sizes
        {"name": "logprobs_fp32", "op": "logprobs", "rows": 777, "V": 32001, "pad": 0, "dtype": "fp32", "J": 3, "k": 20,
         "T": 0.7, "masked": True, "pool": 0},
        # a training step of a drafter: log probabilities, entropy and the gradient of both
        {"name": "train_batch", "op": "train", "rows": 2048, "V": 151936, "pad": 0, "dtype": "bf16", "J": 1, "T": 1.0,
         "masked": False, "entropy": True},
        # few rows of a smaller vocabulary in 32 bits, several tokens a row
        {"name": "train_few_rows", "op": "train", "rows": 60, "V": 32001, "pad": 0, "dtype": "fp32", "J": 2, "T": 1.3,
         "masked": True, "entropy": False},
        # one token through the output projection
        {"name": "project_one_token", "op": "project", "tokens": 1, "V": 151936, "K": 4096, "dtype": "bf16", "out": "bf16",
         "bias": False},
        # a chain of drafts for a few users, 32-bit logits
        {"name": "project_chains", "op": "project", "tokens": 48, "V": 151936, "K": 4096, "dtype": "bf16", "out": "fp32",
         "bias": False},
        # the verification batch: 64 trees of 60 nodes
        {"name": "project_trees", "op": "project", "tokens": 3840, "V": 151936, "K": 4096, "dtype": "bf16", "out": "bf16",
         "bias": False},
        # a smaller vocabulary, nothing a multiple of anything, with a bias
        {"name": "project_odd", "op": "project", "tokens": 333, "V": 32001, "K": 5000, "dtype": "fp32", "out": "bf16",
         "bias": True},
        # scoring of a prompt: hidden states to log probabilities and entropies
        {"name": "score_prompt", "op": "score", "tokens": 500, "V": 151936, "K": 4096, "dtype": "bf16", "out": "fp32",
         "bias": False, "J": 1, "T": 1.0},
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["logprobs", "logprobs", "train", "project", "project", "score"])
    V = rng.choice([151936, 32000, _spread(rng, 500, 152000), _spread(rng, 500, 152000)])
    if op in ("logprobs", "train"):
        c = {"op": op, "rows": _spread(rng, 1, 3840 if op == "logprobs" else 2048), "V": V,
             "pad": rng.choice([0, 0, 128, rng.randrange(1, 64)]), "dtype": rng.choice(["bf16", "fp32"]),
             "J": rng.choice([1, 1, rng.randrange(1, 9)]), "T": round(rng.uniform(0.4, 2.0), 3),
             "masked": rng.random() < 0.3}
        if op == "logprobs":
            c["k"] = rng.choice([0, 1, 5, 10, rng.randrange(2, 33)])
            c["pool"] = c["rows"] * 3 + 1 if rng.random() < 0.3 else 0
        else:
            c["entropy"] = rng.random() < 0.5
        while max(c["rows"], c.get("pool", 0)) * (V + c["pad"]) * (2 if c["dtype"] == "bf16" else 4) > 1.2e9:
            c["rows"] = max(1, c["rows"] // 2)
            c["pool"] = c["rows"] * 3 + 1 if c.get("pool") else 0
        if op == "train":
            c.pop("pool", None)
        return c
    c = {"op": op, "tokens": _spread(rng, 1, 3840 if op == "project" else 1000), "V": V,
         "K": rng.choice([4096, 1024, _spread(rng, 64, 8192), _spread(rng, 64, 8192)]),
         "dtype": rng.choice(["bf16", "fp32"]), "out": "fp32" if op == "score" else rng.choice(["bf16", "fp32"]),
         "bias": rng.random() < 0.3}
    if op == "score":
        c["J"], c["T"] = rng.choice([1, 3]), round(rng.uniform(0.5, 1.5), 3)
    while c["tokens"] * c["V"] * c["K"] > 2.3e12 or c["tokens"] * c["V"] * (2 if c["out"] == "bf16" else 4) > 1.2e9:
        c["tokens"] = max(1, c["tokens"] // 2)
    return c


def work(case):
    op, V = case["op"], case["V"]
    if op in ("logprobs", "train"):
        rows, e = case["rows"], 2 if case["dtype"] == "bf16" else 4
        small = rows * 4 * (2 * case["J"] + 1 + 2 * case.get("k", 0))
        both = 2 if op == "train" else 1
        # a maximum, a scaled difference, an exponential, two sums (and the gradient's product) for each logit
        return {"bytes": both * rows * V * e + small, "flops": rows * V * (6 + 6 * (op == "train"))}
    M, K = case["tokens"], case["K"]
    b = M * K * (2 if case["dtype"] == "bf16" else 4) + V * K + 4 * V * (1 + case["bias"])
    if op == "project":
        b += M * V * (2 if case["out"] == "bf16" else 4)
    else:
        b += M * 4 * (2 * case["J"] + 1)
    return {"bytes": b, "flops": 2 * M * V * K}


# -------------------------------------------------------------------------------- making the inputs

def _gen(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1000003 + (case["V"] * 31 + case.get("rows", case.get("tokens", 0))) % 1000003)
    return g


def _logits(case, g, rows):
    """Logits as verification meets them: a normal bulk, one clear leader, often a close runner-up."""
    V, dt = case["V"], DTYPES[case["dtype"]]
    wide = torch.empty((rows, V + case["pad"]), dtype=dt, device=DEV)
    step = max(1, (1 << 28) // wide.shape[1])
    lead = torch.randint(0, V, (rows, 2), generator=g, device=DEV)
    top = torch.rand((rows, 1), generator=g, device=DEV) * 15 + 8
    near = torch.where(torch.rand((rows, 1), generator=g, device=DEV) < 0.3,
                       0.85 + 0.15 * torch.rand((rows, 1), generator=g, device=DEV), 0.4)
    for r0 in range(0, rows, step):
        n = min(step, rows - r0)
        wide[r0:r0 + n] = (torch.randn((n, wide.shape[1]), generator=g, device=DEV) * 3).to(dt)
    z = wide[:, :V]
    z.scatter_(1, lead[:, 1:], (top * near).to(dt))
    z.scatter_(1, lead[:, :1], top.to(dt))
    if case["masked"]:
        off = torch.rand((V,), generator=g, device=DEV) < 0.4
        off[lead.flatten()] = False
        z.masked_fill_(off, float("-inf"))
        for j in range(2):
            z.scatter_(1, lead[:, 1 - j:2 - j], (top * (near if j == 0 else 1)).to(dt))
    return z, lead


def _tokens(g, lead, J, V, z=None):
    """The leader, the runner-up or any token; a tenth of the places behind the first hold none."""
    rows = lead.shape[0]
    u = torch.rand((rows, J), generator=g, device=DEV)
    t = torch.randint(0, V, (rows, J), generator=g, device=DEV)
    if z is not None:                # a forbidden token is never the one that a text holds
        t = torch.where(torch.isinf(z.gather(1, t)), lead[:, :1], t)
    t = torch.where(u < 0.5, lead[:, :1], torch.where(u < 0.7, lead[:, 1:], t))
    t[:, 1:] = torch.where(torch.rand((rows, J - 1), generator=g, device=DEV) < 0.1, -1, t[:, 1:])
    return t.to(torch.int32).contiguous()


def _weights(V, K, g):
    """A weight matrix quantised once, row by row: codes [V, K] in rows of a multiple of 16 bytes, scales."""
    wide = torch.zeros((V, -(-K // 16) * 16), dtype=torch.int8, device=DEV)
    scale = torch.empty((V,), dtype=torch.float32, device=DEV)
    step = max(1, (1 << 28) // K)
    for v0 in range(0, V, step):
        w = torch.randn((min(step, V - v0), K), generator=g, device=DEV) * 0.02
        s = w.abs().amax(1) / 127
        wide[v0:v0 + step, :K] = (w / s[:, None]).round().to(torch.int8)
        scale[v0:v0 + step] = s
    return wide[:, :K], scale


def prepare(case, seed):
    g = _gen(case, seed)
    s = {"case": case}
    V, op = case["V"], case["op"]
    if op in ("logprobs", "train"):
        rows, J = case["rows"], case["J"]
        s["logits"], lead = _logits(case, g, case.get("pool") or rows)
        s["rows"] = None
        if case.get("pool"):
            ids = torch.randperm(case["pool"], generator=g, device=DEV)[:rows]
            s["rows"] = torch.where(torch.rand((rows,), generator=g, device=DEV) < 0.25, -1, ids).to(torch.int32)
            lead = lead[ids]
            s["tok"] = _tokens(g, lead, J, V, s["logits"][ids] if case["masked"] else None)
        else:
            s["tok"] = _tokens(g, lead, J, V, s["logits"] if case["masked"] else None)
    else:
        rows, J, dt = case["tokens"], case.get("J", 0), DTYPES[case["dtype"]]
        loud = 1 + 15 * (torch.rand((case["K"],), generator=g, device=DEV) > 0.995).float()
        s["x"] = (torch.randn((rows, case["K"]), generator=g, device=DEV) * loud).to(dt)
        s["w"], s["ws"] = _weights(V, case["K"], g)
        s["bias"] = torch.randn((V,), generator=g, device=DEV) if case["bias"] else None
        s["logits"] = torch.empty((rows, V), dtype=DTYPES[case["out"]], device=DEV)
        if own:
            from paper_2601_15498_b200 import scores
            s["work"] = scores.project_workspace(rows, V, case["K"], DEV)
        if op == "score":
            s["tok"] = torch.randint(0, V, (rows, J), generator=g, device=DEV).to(torch.int32)
    if op == "train":
        s["g"] = torch.randn((rows, J), generator=g, device=DEV) / rows
        s["h"] = torch.randn((rows,), generator=g, device=DEV) * 0.01 / rows if case["entropy"] else None
        s["grad"] = torch.empty((rows, V), dtype=s["logits"].dtype, device=DEV)
    return s


# ------------------------------------------------------------------------------------- one pass

def run(s):
    case = s["case"]
    if own:
        return _run_own(s, case)
    if case["op"] in ("project", "score"):
        logits = _plain_project(s, case)
        if case["op"] == "project":
            return logits
        got = _plain_logprobs(logits, s["tok"], case["T"], 0)
        return {"logprob": got["logprob"], "entropy": got["entropy"]}
    z = s["logits"]
    if case["op"] == "logprobs":
        if s["rows"] is not None:
            z = z[s["rows"].long().clamp(min=0)]
        got = _plain_logprobs(z, s["tok"], case["T"], case["k"])
        got.pop("logp")
        if s["rows"] is not None:
            none = (s["rows"] < 0)[:, None]
            got["logprob"] = got["logprob"].masked_fill(none, 0.0)
            got["entropy"] = got["entropy"].masked_fill(none[:, 0], 0.0)
            if case["k"]:
                got["top_logprob"] = got["top_logprob"].masked_fill(none, float("-inf"))
                got["top_id"] = got["top_id"].masked_fill(none, -1)
        return got
    got = _plain_logprobs(z, s["tok"], case["T"], 0)
    p = got["logp"].exp()
    ok = (s["tok"] >= 0) & (s["tok"] < case["V"])
    g = torch.where(ok, s["g"], 0.0)
    grad = p * -g.sum(1, keepdim=True)
    if s["h"] is not None:
        grad -= s["h"][:, None] * torch.where(p > 0, p * (got["logp"] + got["entropy"][:, None]), 0.0)
    grad.scatter_add_(1, s["tok"].long().clamp(0, case["V"] - 1), g)
    return {"logprob": got["logprob"], "entropy": got["entropy"], "grad": (grad / case["T"]).to(z.dtype)}


def _plain_project(s, case):
    x = s["x"].float()
    a = x.abs().amax(1, keepdim=True)
    q = torch.round(x * (127 / a))
    y = (q @ s["w"].float().T) * (a / 127) * s["ws"]
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(DTYPES[case["out"]])


def _plain_logprobs(z, tok, T, k):
    V = z.shape[1]
    x = z.float() / T
    m = x.amax(1, keepdim=True)
    logp = x - m
    logp = logp - logp.exp().sum(1, keepdim=True).log()
    p = logp.exp()
    out = {"logp": logp, "entropy": -torch.where(p > 0, p * logp, 0.0).sum(1)}
    t = tok.long()
    out["logprob"] = torch.where((t >= 0) & (t < V), logp.gather(1, t.clamp(0, V - 1)), 0.0)
    if k:
        # distinct whole keys in the order of the rule: the value's bits, then the ids falling
        b = (z.float() + 0.0).view(torch.int32).long()
        key = (torch.where(b < 0, -(b & 0x7fffffff), b) << 20) + (V - torch.arange(V, device=z.device))
        top = key.topk(k, 1).indices
        out["top_id"], out["top_logprob"] = top.to(torch.int32), logp.gather(1, top)
    return out


def _run_own(s, case):
    from paper_2601_15498_b200 import scores
    if case["op"] in ("project", "score"):
        q, qs = scores.quantize_rows(s["x"])
        logits = scores.project_int8(q, qs, s["w"], s["ws"], bias=s["bias"], out=s["logits"], workspace=s["work"])
        if case["op"] == "project":
            return logits
        got = scores.token_logprobs(logits, s["tok"], temperature=case["T"])
        return {"logprob": got["logprob"], "entropy": got["entropy"]}
    if case["op"] == "logprobs":
        got = scores.token_logprobs(s["logits"], s["tok"], temperature=case["T"], k=case["k"], rows=s["rows"])
        names = ("logprob", "entropy") + (("top_id", "top_logprob") if case["k"] else ())
        return {n: got[n] for n in names}
    got = scores.token_logprobs(s["logits"], s["tok"], temperature=case["T"])
    grad = scores.token_logprobs_backward(s["logits"], s["tok"], got, s["g"], grad_entropy=s["h"],
                                          temperature=case["T"], out=s["grad"])
    return {"logprob": got["logprob"], "entropy": got["entropy"], "grad": grad}


# --------------------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("project", "score"):
        x = s["x"].float()                       # the codes are defined by operations in 32 bits
        a = x.abs().amax(1)
        q = torch.round(x * (127 / a)[:, None]).double()
        y = torch.matmul(q, s["w"].double().t())
        y *= (a / 127).double()[:, None]
        y *= s["ws"].double()[None]
        if s["bias"] is not None:
            y += s["bias"].double()[None]
        if case["op"] == "project":
            return y
        parts = [_exact_rows(y[i:i + 256], s["tok"][i:i + 256], case["T"]) for i in range(0, y.shape[0], 256)]
        return {n: torch.cat([p[n] for p in parts]) for n in ("logprob", "entropy")}
    V, k = case["V"], case.get("k", 0)
    parts = []
    for r0 in range(0, case["rows"], 256):
        rows = slice(r0, min(r0 + 256, case["rows"]))
        pick = s["rows"][rows].long() if s["rows"] is not None else None
        z = s["logits"][rows] if pick is None else s["logits"][pick.clamp(min=0)]
        z, tok = z.double(), s["tok"][rows]
        e = _exact_rows(z, tok, case["T"])
        lse = e.pop("lse")
        if k:
            best = z.sort(dim=1, descending=True, stable=True)
            e["top_id"] = best.indices[:, :k].to(torch.int32)
            e["top_logprob"] = best.values[:, :k] / case["T"] - lse
        if pick is not None:
            gone = pick < 0
            e["logprob"][gone], e["entropy"][gone] = 0, 0
            if k:
                e["top_id"][gone], e["top_logprob"][gone] = -1, float("-inf")
        if case["op"] == "train":
            # by the chain rule through z / T: each token pulls on its own logit and pushes on all
            p = torch.softmax(z / case["T"], 1)
            grad = torch.zeros_like(p)
            g = s["g"][rows].double()
            for j in range(case["J"]):
                on = ((tok[:, j] >= 0) & (tok[:, j] < V)).nonzero()[:, 0]
                grad[on] -= g[on, j, None] * p[on]
                grad[on, tok[on, j].long()] += g[on, j]
            if s["h"] is not None:
                surprise = torch.where(p > 0, -p.clamp(min=1e-320).log(), 0.0)
                grad += s["h"][rows].double()[:, None] * p * (surprise - e["entropy"][:, None])
            e["grad"] = grad / case["T"]
        parts.append(e)
    return {n: torch.cat([p[n] for p in parts]) for n in parts[0]}


def _exact_rows(z, tok, T):
    V = z.shape[1]
    y = z / T
    lse = torch.logsumexp(y, 1, keepdim=True)
    p = (y - lse).exp()
    inside = (tok >= 0) & (tok < V)
    at = torch.where(inside, tok, 0).long()
    lp = torch.where(inside, y.gather(1, at) - lse, 0.0)
    return {"lse": lse, "logprob": lp, "entropy": -torch.special.xlogy(p, p).sum(1)}

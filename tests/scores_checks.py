"""Plain 64-bit forms of token log probabilities, entropy, alternatives and their gradient, and how far
fp32 arithmetic may be from them.

The kernels sum 2^x with x = (z - m) c, c = log2(e) / T.  In units of 2^-24 (half a step of fp32):
  x            4 |x|: the difference, c and the product round once each, c once more on its way to fp32
  2^x          4: the exponential unit's stated error is below 2^-22
  s            2^x and x of its terms, weighted by the terms themselves (sum 2^x |x| / s <= log2 V <= 18), at most
               128 additions in one chain (batches of a thread, pairs, lanes, warps, blocks), and an
               exponential each time the running maximum moves, at most once a batch: 4 * 80
so s is off by at most (4 + 4 * 18 + 128 + 320) units = 524, and ln s by that and its own rounding.
"""
import math

import torch

UNIT = 2.0 ** -24
SUM = 524


def reference(z, tok=None, T=1.0, k=0):
    """fp64 form of one call: z [rows, V] any dtype, tok [rows, J] or None."""
    z = z.double()
    z = torch.where(torch.isnan(z), float("-inf"), z)
    V = z.shape[1]
    m = z.amax(1, keepdim=True)
    ok = torch.isfinite(m)
    y = torch.where(ok, (z - m) / T, float("-inf"))
    s = y.exp().sum(1, keepdim=True)
    logp = torch.where(ok, y - s.log(), float("nan"))
    p = logp.exp()
    out = {"m": m, "s": torch.where(ok, s, float("nan")), "logp": logp, "p": p, "ok": ok[:, 0], "y": y,
           "entropy": torch.where(ok[:, 0], -torch.where(p > 0, p * logp, 0.0).sum(1), float("nan"))}
    if tok is not None:
        t = tok.to(z.device).long()
        inside = (t >= 0) & (t < V)
        out["logprob"] = torch.where(inside, logp.gather(1, t.clamp(0, V - 1)), 0.0)
    if k:
        best = z.sort(dim=1, descending=True, stable=True).indices[:, :k]
        out["top_id"], out["top_logprob"] = best, logp.gather(1, best)
    return out


def reference_grad(ref, tok, g, h, T):
    t = tok.to(ref["logp"].device).long()
    V = ref["logp"].shape[1]
    inside = (t >= 0) & (t < V)
    g = torch.where(inside, g.double(), 0.0)
    p, logp = ref["p"], ref["logp"]
    size = p * g.abs().sum(1, keepdim=True)
    grad = -p * g.sum(1, keepdim=True)
    if h is not None:
        term = torch.where(p > 0, p * (logp + ref["entropy"][:, None]), 0.0)
        grad = grad - h.double()[:, None] * term
        size = size + h.double().abs()[:, None] * torch.where(p > 0, p * (logp.abs() + ref["entropy"][:, None] + 1), 0.0)
    grad = grad.scatter_add(1, t.clamp(0, V - 1), g)
    size = size.scatter_add(1, t.clamp(0, V - 1), g.abs())
    bad = ~ref["ok"][:, None]
    return torch.where(bad, 0.0, grad / T), torch.where(bad, 0.0, size / T)


def same_kind(got, want):
    """Infinities and NaN in the same places; what passes fp32's largest number is infinite there."""
    got, want = got.double(), want.float().double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    inf = torch.isinf(want)
    assert torch.equal(torch.isinf(got), inf) and torch.equal(got[inf], want[inf])
    return torch.isfinite(want)


def within(got, want, tol, what):
    f = same_kind(got, want)
    d = (got.double() - want).abs()
    tol = tol.expand_as(want) if torch.is_tensor(tol) else torch.full_like(want, tol)
    over = (d > tol) & f
    assert not over.any(), (what, d[over][:4].tolist(), tol[over][:4].tolist(), want[over][:4].tolist())


def check_forward(z, got, tok=None, T=1.0, k=0):
    """got (a call's dict) against the fp64 form of rows z."""
    ref = reference(z, tok, T, k)
    ln_s = torch.where(ref["ok"], ref["s"][:, 0].log(), 0.0)
    own = UNIT * (SUM + 4 * ln_s)                                       # ln s: its error, its rounding
    f = lambda lp: own[:, None] + UNIT * 6 * (torch.nan_to_num(lp.abs(), posinf=0) + ln_s[:, None])  # noqa: E731
    assert torch.equal(got["stats"][:, 0].double(), ref["m"][:, 0])
    within(got["stats"][:, 1], ref["s"][:, 0], UNIT * (SUM + 4) * torch.nan_to_num(ref["s"][:, 0]), "s")
    # u / s = -sum p |x| ln2 has the relative errors of s twice, once more weighted by |x|
    within(got["entropy"], ref["entropy"], own + UNIT * (2 * SUM + 4 * 18) * (ln_s + 1), "entropy")
    if tok is not None:
        lp = got["logprob"].view(z.shape[0], -1)
        within(lp, ref["logprob"], f(ref["logprob"]), "logprob")
    if k:
        assert torch.equal(got["top_id"].long(), ref["top_id"])
        within(got["top_logprob"], ref["top_logprob"], f(ref["top_logprob"]), "top_logprob")
    return ref


def check_grad(z, grad, ref, tok, g, h, T):
    want, size = reference_grad(ref, tok, g, h, T)
    # 2^x and 1 / s, the line a + b x (each part of it rounded a few times), the sum of the g and the last
    # addition; a 2^x below 2^-126 is 0, which loses at most 2^-126 |a + b x|
    x = torch.nan_to_num(ref["y"].abs() * math.log2(math.e), posinf=0.0)
    tol = UNIT * (2 * SUM + 8 * x + 64 + tok.shape[1]) * size + 2.0 ** -125
    line = g.double().abs().sum(1, keepdim=True)
    if h is not None:
        line = line + h.double().abs()[:, None] * (x + torch.nan_to_num(ref["entropy"] + ref["s"][:, 0].log())[:, None])
    tol = tol + 2.0 ** -126 * line / T
    if grad.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * want.abs() + 2.0 ** -133
    within(grad, want, tol, "grad")

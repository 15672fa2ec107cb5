"""Token log probabilities, entropy, alternatives and their gradient on the device, against plain forms in
64 bits (scores_checks.py derives the tolerances)."""
import numpy as np
import pytest
import torch

import hookctl as hooks
import scores_checks as sc
from paper_2601_15498_b200 import mars, scores, synth
from tests.test_gpu_parity import special_rows

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, FP32 = torch.bfloat16, torch.float32


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def rows_of(R, V, dtype, seed, spread=3.0, pad=0, shift=0):
    """[R, V] logits inside a buffer with guard values around every row."""
    wide = torch.full((R, V + pad + shift), 3e38, dtype=dtype, device=DEV)
    z = wide[:, shift:shift + V]
    z.copy_((torch.randn((R, V), generator=gen(seed), device=DEV) * spread).to(dtype))
    return z


def tokens(R, J, V, seed):
    t = torch.randint(0, V, (R, J), generator=gen(seed), device=DEV).to(torch.int32)
    if J > 1:
        t[:, 1] = t[:, 0]                                   # the same token twice
    if J > 2:
        t[::2, 2] = -1
        t[1::2, 2] = V
    return t


@pytest.mark.parametrize("R,V,J,k,T", [(1, 151936, 1, 10, 1.0), (60, 151936, 4, 5, 0.7), (700, 32001, 1, 0, 1.3),
                                       (5, 1, 3, 1, 1.0), (3, 2, 1, 2, 0.5), (9, 33, 2, 32, 2.0), (40, 257, 8, 7, 1.0),
                                       (2, 70001, 300, 20, 1.0), (1300, 4099, 2, 3, 0.9), (4, 500003, 1, 32, 1.0)])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_forward_and_gradient(R, V, J, k, T, dtype):
    z, tok = rows_of(R, V, dtype, R + V, pad=3 if V % 2 else 0, shift=V % 5), tokens(R, J, V, J)
    got = scores.token_logprobs(z, tok, temperature=T, k=k)
    ref = sc.check_forward(z, got, tok, T, k)
    if R * V > 3e7:
        return
    g = torch.randn((R, J), generator=gen(7), device=DEV)
    h = torch.randn((R,), generator=gen(8), device=DEV)
    for ge in (None, h):
        grad = scores.token_logprobs_backward(z, tok, got, g, ge, temperature=T)
        sc.check_grad(z, grad, ref, tok, g, ge, T)


@pytest.mark.parametrize("S", [2, 4, 8])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_rows_split_over_clusters(S, dtype):
    hooks.set("HOOK_FORCE_SPLIT", S)
    for R, V, k in ((3, 1, 1), (6, 17, 5), (5, 1000, 32), (9, 40007, 10), (700, 2049, 3)):
        z, tok = rows_of(R, V, dtype, S * V, pad=1), tokens(R, 2, V, 3)
        z[0] = torch.linspace(-8, 8, V, device=DEV).to(dtype)              # ascending: the queue overflows
        z[R // 2] = 0.5                                                   # ties everywhere
        sc.check_forward(z, scores.token_logprobs(z, tok, k=k), tok, 1.0, k)
        sc.check_forward(z, scores.token_logprobs(z, tok), tok, 1.0, 0)


def masked_rows(V, dtype):
    low = torch.finfo(dtype).min
    z = rows_of(12, V, dtype, 5)
    z[0] = float("-inf")                                                  # the mask leaves nothing
    z[1] = low                                                            # the same with the type's lowest value
    z[2, V // 3:] = low
    z[3, ::2] = float("-inf")
    z[4, 1::2] = low; z[4, ::2] = float("-inf")                           # both, and nothing else
    z[5, V // 2] = float("inf")
    z[6] = float("nan")
    z[7, ::3] = float("nan"); z[7, 1::3] = float("-inf")
    z[8] = float("-inf"); z[8, V - 1] = -2.5
    z[9] = 0.0; z[9, ::2] = -0.0
    z[10] *= 1e30; z[10, 0] = float("-inf")
    z[11] = -torch.finfo(dtype).max; z[11, V // 2] = torch.finfo(dtype).max
    return z


@pytest.mark.parametrize("V", [3, 40, 4099, 151936])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_masked_rows(V, dtype):
    z, tok = masked_rows(V, dtype), tokens(12, 4, V, 1)
    k = min(V, 10)
    for T in (1.0, 0.25):
        got = scores.token_logprobs(z, tok, temperature=T, k=k)
        ref = sc.check_forward(z, got, tok, T, k)
        g = torch.randn((12, 4), generator=gen(2), device=DEV)
        h = torch.randn((12,), generator=gen(3), device=DEV)
        grad = scores.token_logprobs_backward(z, tok, got, g, h, temperature=T)
        sc.check_grad(z, grad, ref, tok, g, h, T)
        assert (grad[[0, 5, 6]] == 0).all() and torch.isfinite(grad).all()


@pytest.mark.parametrize("T", [1e-30, 1e-4, 1e4, 1e30, 3e38])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_extreme_temperatures_and_sizes_of_logits(T, dtype):
    V = 2500
    for scale in (1e-30, 1.0, 1e8, 1e36):
        z, tok = rows_of(6, V, dtype, 4, spread=scale), tokens(6, 3, V, 1)
        z[0, ::2] = float("-inf")
        got = scores.token_logprobs(z, tok, temperature=T, k=4)
        ref = sc.reference(z, tok, T, 4)
        sc.within(got["logprob"], ref["logprob"], sc.UNIT * (sc.SUM + 6 * torch.nan_to_num(ref["logprob"].abs(), posinf=0) + 100), "logprob")
        assert torch.equal(got["top_id"].long(), ref["top_id"]) and torch.isfinite(got["entropy"]).all()
        sc.within(got["entropy"], ref["entropy"], sc.UNIT * 10 * (2 * sc.SUM + 72), "entropy")
        if T >= 1e-4:
            g = torch.randn((6, 3), generator=gen(2), device=DEV)
            grad = scores.token_logprobs_backward(z, tok, got, g, g[:, 0].contiguous(), temperature=T)
            sc.check_grad(z, grad, sc.reference(z, tok, T), tok, g, g[:, 0], T)


@pytest.mark.parametrize("T", [2.0, 4.0, 1e3, 1e37, 1e38, 3e38])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_logits_further_apart_than_the_largest_number(T, dtype):
    """Logits of both signs at the end of the range: their difference passes it, divided by T it need not."""
    big = torch.finfo(dtype).max
    for V in (2, 37, 4099, 151936):
        z, tok = rows_of(5, V, dtype, 6), tokens(5, 4, V, 2)
        z[0] = -big; z[0, V // 2] = big
        z[1] = big; z[1, ::2] = -big
        z[2] = torch.linspace(-1, 1, V, device=DEV) * big
        z[3] = torch.linspace(1, -1, V, device=DEV) * big; z[3, V // 3] = float("-inf")
        z[4, 0] = big; z[4, -1] = -big
        tok[:, 0], tok[:, 3] = 0, V // 2
        k = min(V, 9)
        got = scores.token_logprobs(z, tok, temperature=T, k=k)
        ref = sc.check_forward(z, got, tok, T, k)
        assert torch.isfinite(got["logprob"][:3, [0, 3]]).all()             # twice the largest number over T >= 2
        g = torch.randn((5, 4), generator=gen(2), device=DEV)
        h = torch.randn((5,), generator=gen(3), device=DEV)
        sc.check_grad(z, scores.token_logprobs_backward(z, tok, got, g, h, temperature=T), ref, tok, g, h, T)


@pytest.mark.parametrize("T", [1e34, 1e38, 3e38])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_gradient_where_temperature_times_sum_overflows(T, dtype):
    z, tok = rows_of(5, 40007, dtype, 4, spread=T / 8), tokens(5, 3, 40007, 1)
    z.clamp_(-0.4 * 3e38, 0.4 * 3e38)
    got = scores.token_logprobs(z, tok, temperature=T)
    ref = sc.check_forward(z, got, tok, T)
    g = torch.randn((5, 3), generator=gen(2), device=DEV) * 1e14
    h = torch.randn((5,), generator=gen(3), device=DEV) * 1e14
    for ge in (None, h):
        grad = scores.token_logprobs_backward(z, tok, got, g, ge, temperature=T)
        sc.check_grad(z, grad, ref, tok, g, ge, T)
        assert (grad != 0).all()


@pytest.mark.parametrize("T", [1e-34, 1e-36, 4e-38])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_gradient_whose_factors_end_the_range(T, dtype):
    """g / T passes fp32's largest number; what is multiplied by a probability of 0 is 0 all the same, a nearly certain
    token's gradient finite."""
    z, tok = rows_of(4, 1001, dtype, 4, spread=2 * T), tokens(4, 3, 1001, 1)
    z[1] = 0.0                                                         # uniform: every part is g / (1001 T)
    z[2, ::2] = float("-inf")
    z[3] = -1.0; z[3, 5] = 1.0; tok[3] = 5                             # certain
    got = scores.token_logprobs(z, tok, temperature=T)
    ref = sc.check_forward(z, got, tok, T)
    g, h = torch.randn((4, 3), generator=gen(2), device=DEV) * 40, torch.randn((4,), generator=gen(3), device=DEV) * 40
    for ge in (None, h):
        grad = scores.token_logprobs_backward(z, tok, got, g, ge, temperature=T)
        assert not torch.isnan(grad).any() and (grad[3] == 0).all() and (grad[2, ::2] == 0).all()
        sc.check_grad(z, grad, ref, tok, g, ge, T)


def test_alternatives_follow_the_order_of_topk_rows():
    for V, dtype in ((4099, BF16), (4099, FP32), (37, FP32)):
        z = special_rows(V, dtype)
        for k in (1, min(9, V), min(32, V)):
            val, idx = mars.topk_rows(z, k)
            got = scores.token_logprobs(z, k=k)
            assert torch.equal(got["top_id"], idx)
            sc.check_forward(z, got, None, 1.0, k)


@pytest.mark.parametrize("k", [0, 6])
def test_picked_rows(k):
    z = rows_of(50, 3001, BF16, 9)
    ids = torch.tensor([49, 0, 7, 7, -1, 3, 50, 7, -2 ** 31, 2 ** 31 - 1, 12], dtype=torch.int32, device=DEV)
    tok = tokens(11, 2, 3001, 4)
    out = {n: torch.full((13,) + s, -777, dtype=d, device=DEV) for n, s, d in (
        ("logprob", (2,), FP32), ("entropy", (), FP32), ("stats", (2,), FP32), ("top_id", (6,), torch.int32), ("top_logprob", (6,), FP32))}
    inner = {n: t[1:12] for n, t in out.items()}
    got = scores.token_logprobs(z, tok, k=k, rows=ids, out=inner)
    live = ((ids >= 0) & (ids < 50)).nonzero()[:, 0]
    part = {n: t[live] for n, t in got.items()}
    sc.check_forward(z[ids[live].long()], part, tok[live], 1.0, k)
    gone = ((ids < 0) | (ids >= 50)).nonzero()[:, 0]
    assert (got["logprob"][gone] == 0).all() and (got["entropy"][gone] == 0).all()
    assert (got["stats"][gone, 0] == float("-inf")).all() and (got["stats"][gone, 1] == 0).all()
    if k:
        assert (got["top_id"][gone] == -1).all() and (got["top_logprob"][gone] == float("-inf")).all()
    for n, t in out.items():
        assert (t[0] == -777).all() and (t[12] == -777).all(), n
        if n.startswith("top") and not k:
            assert (t == -777).all()
    hooks.set("HOOK_FORCE_SPLIT", 4)
    again = scores.token_logprobs(z, tok, k=k, rows=ids)
    sc.check_forward(z[ids[live].long()], {n: t[live] for n, t in again.items()}, tok[live], 1.0, k)
    assert (again["entropy"][gone] == 0).all()


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_gradient_in_place_beside_and_across_alignments(dtype):
    R, V, J = 7, 4099, 5
    z = rows_of(R, V, dtype, 3, pad=5, shift=2)
    tok = tokens(R, J, V, 6)
    tok[:, 3] = tok[:, 4]
    g, h = torch.randn((R, J), generator=gen(1), device=DEV), torch.randn((R,), generator=gen(2), device=DEV)
    got = scores.token_logprobs(z, tok)
    base = scores.token_logprobs_backward(z, tok, got, g, h)
    sc.check_grad(z, base, sc.reference(z, tok), tok, g, h, 1.0)
    for shift in range(0, 9):
        wide = torch.full((R + 1, V + 20), -777.0, dtype=dtype, device=DEV)
        scores.token_logprobs_backward(z, tok, got, g, h, out=wide[:R, shift:])
        assert torch.equal(wide[:R, shift:shift + V], base)
        assert (wide[:R, :shift] == -777).all() and (wide[:R, shift + V:] == -777).all() and (wide[R] == -777).all()
    keep = z.clone()
    between = z.as_strided((R - 1, z.stride(0) - V), z.stride(), z.storage_offset() + V)     # what lies between the rows
    behind = between.clone()
    scores.token_logprobs_backward(z, tok, got, g, h, out=z)
    assert torch.equal(z, base) and torch.equal(between, behind) and not torch.equal(z, keep)


def test_gradient_against_differences():
    """Central differences of the fp64 value, and of the device's own forward: with a step of 2^-5 their
    error is the third derivative's, at most (2^-5)^2 / 6 of sums of probabilities times g, and twice the forward's error
    over the step."""
    R, V, J, T = 3, 23, 4, 0.8
    z = rows_of(R, V, FP32, 11, spread=1.5)
    tok = tokens(R, J, V, 2)
    g, h = torch.randn((R, J), generator=gen(4), device=DEV), torch.randn((R,), generator=gen(5), device=DEV)
    got = scores.token_logprobs(z, tok, temperature=T)
    grad = scores.token_logprobs_backward(z, tok, got, g, h, temperature=T)

    def value(x):
        f = scores.token_logprobs(x, tok, temperature=T)
        return ((f["logprob"] * g).sum(1) + f["entropy"] * h).double()
    step = 2.0 ** -5
    size = (g.abs().sum(1) + 12 * h.abs()).double()
    for v in range(V):
        hi, lo = z.clone(), z.clone()
        hi[:, v] += step
        lo[:, v] -= step
        d = (value(hi) - value(lo)) / (hi[:, v] - lo[:, v]).double()
        tol = size * (step ** 2 / 6 / T ** 3 * 2 + 2 * 8 * sc.UNIT * 64 / step)
        assert ((d - grad[:, v].double()).abs() <= tol).all()


@pytest.mark.parametrize("entropy", [False, True])
def test_autograd(entropy):
    R, V, J = 6, 1001, 3
    z = rows_of(R, V, FP32, 21).contiguous().requires_grad_()
    tok, w = tokens(R, J, V, 1), torch.randn((R, J), generator=gen(1), device=DEV)
    lp, H = scores.logprobs(z, tok, 1.25)
    (((lp * w).sum() if not entropy else (lp * w).sum() - 0.3 * H.sum())).backward()
    ref = sc.reference(z.detach(), tok, 1.25)
    h = torch.full((R,), -0.3, device=DEV) if entropy else torch.zeros((R,), device=DEV)
    sc.check_grad(z.detach(), z.grad, ref, tok, w, h, 1.25)
    one = scores.logprobs(z, tok[:, 0])[0]                                # [rows] tokens, broadcast gradient
    z.grad = None
    one.mean().backward()
    sc.check_grad(z.detach(), z.grad, sc.reference(z.detach(), tok[:, :1]), tok[:, :1].contiguous(), torch.full((R, 1), 1 / R, device=DEV), None, 1.0)


def test_same_bits_again_and_on_another_stream_and_in_a_graph():
    z, tok = rows_of(300, 32001, BF16, 2), tokens(300, 3, 32001, 8)
    g, h = torch.randn((300, 3), generator=gen(3), device=DEV), torch.randn((300,), generator=gen(4), device=DEV)

    def both(out=None, gout=None):
        f = scores.token_logprobs(z, tok, k=8, out=out)
        return f, scores.token_logprobs_backward(z, tok, f, g, h, out=gout)
    base, bgrad = both()
    torch.cuda.synchronize()
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    many = []
    for i in range(6):
        with torch.cuda.stream(side[i % 2]):
            many.append(both())
    torch.cuda.synchronize()
    for f, gr in many:
        assert all(torch.equal(f[n], base[n]) for n in base) and torch.equal(gr, bgrad)
    out = {n: torch.empty_like(t) for n, t in base.items()}
    gout = torch.empty_like(bgrad)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both(out, gout)
    z.copy_(z.flip(0)); tok.copy_(tok.flip(0)); g.copy_(g.flip(0)); h.copy_(h.flip(0))
    base, bgrad = both()
    for _ in range(2):
        for t in list(out.values()) + [gout]:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[n], base[n]) for n in base) and torch.equal(gout, bgrad)


def test_far_rows_of_a_large_buffer():
    """Row offsets beyond 32 bits: 9 rows 2^28 elements apart."""
    wide = torch.empty((8 * (1 << 28) + 4099,), dtype=BF16, device=DEV)
    z = wide.as_strided((9, 4099), (1 << 28, 1))
    z.copy_((torch.randn((9, 4099), generator=gen(1), device=DEV) * 3).to(BF16))
    tok = tokens(9, 2, 4099, 3)
    got = scores.token_logprobs(z, tok, k=4)
    ref = sc.check_forward(z, got, tok, 1.0, 4)
    g = torch.randn((9, 2), generator=gen(1), device=DEV)
    sc.check_grad(z.clone(), scores.token_logprobs_backward(z, tok, got, g, out=z), ref, tok, g, None, 1.0)


def test_emitted_tokens_of_a_verified_batch():
    """Verification, then what it emitted, as a server reports it."""
    w = synth.tree_workload("emitted", 5, 33, 5, 3, 32000, BF16, DEV, 31, 0.9, 3.0, 12.0, 20.0, 0.5)
    out = mars.verify_tree(w.logits, w.tok, w.parent, w.theta)
    got = scores.emitted_logprobs(w.logits, out, k=2)
    ref = sc.reference(w.logits)
    n, tok, path = (out[x].cpu().numpy() for x in ("out_len", "out_tokens", "path_nodes"))
    assert n.max() > 1
    for b in range(5):
        for i in range(tok.shape[1]):
            lp = float(got["logprob"][b, i])
            if i >= n[b]:
                assert lp == 0 and (got["top_id"][b, i] == -1).all()
                continue
            row = b * 33 + path[b, i]
            assert abs(lp - float(ref["logp"][row, tok[b, i]])) <= 1e-4
            assert int(got["top_id"][b, i, 0]) == int(w.logits[row].float().argmax()) or \
                w.logits[row, got["top_id"][b, i, 0]] == w.logits[row].max()
            if tok[b, i] == got["top_id"][b, i, 0]:
                assert lp == float(got["top_logprob"][b, i, 0])
    drawn = mars.verify_tree_stochastic(w.logits, w.tok, w.parent, synth.make_uniforms(5, 33, 1), w.theta, 0.8)
    again = scores.emitted_logprobs(w.logits, drawn, temperature=0.8)
    assert torch.isfinite(again["logprob"]).all() and (again["logprob"] <= 0).all()


def test_emitted_tokens_of_verified_chains():
    w = synth.cfg2(DEV, B=6)
    B, K = w.draft.shape[0], w.draft.shape[1] + 1
    out = mars.verify_chain(w.logits, w.draft, w.theta)
    got = scores.emitted_logprobs(w.logits, out, chain=True)
    ref = sc.reference(w.logits)["logp"].view(B, K, -1)
    tok, n = out["out_tokens"].long(), out["out_len"]
    live = torch.arange(K, device=DEV)[None] < n[:, None]
    want = torch.where(live, ref.gather(2, tok.clamp(min=0)[:, :, None])[:, :, 0], 0.0)
    assert (got["logprob"].double() - want).abs().max() <= 1e-4 and int(n.max()) > 1
    assert (got["stats"][:, :, 1][~live] == 0).all()


def test_numbers_of_other_kinds_as_arguments():
    z, tok = rows_of(3, 500, FP32, 1), tokens(3, 2, 500, 1)
    a = scores.token_logprobs(z, tok, temperature=np.float32(2), k=np.int64(3))
    b = scores.token_logprobs(z, tok.cpu().long().numpy(), temperature=torch.tensor(2.0), k=3)
    assert all(torch.equal(a[n], b[n]) for n in a)
    c = scores.token_logprobs(z[:, :400], tok % 400, V=300)
    sc.check_forward(z[:, :300], c, tok % 400, 1.0, 0)
    one = scores.token_logprobs(z[:1], tok[:1, :0])
    assert one["logprob"].shape == (1, 0) and torch.isfinite(one["entropy"]).all()


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_gradient_of_the_entropy_alone(dtype):
    z = rows_of(5, 3001, dtype, 2).contiguous().requires_grad_()
    none = torch.empty((5, 0), dtype=torch.int32, device=DEV)
    lp, H = scores.logprobs(z, none, 0.8)
    assert lp.shape == (5, 0)
    w = torch.randn((5,), generator=gen(1), device=DEV)
    (H * w).sum().backward()
    tok = torch.full((5, 1), -1, dtype=torch.int32, device=DEV)
    sc.check_grad(z.detach(), z.grad, sc.reference(z.detach(), tok, 0.8), tok, torch.zeros((5, 1), device=DEV), w, 0.8)
    assert (z.grad != 0).any(1).all()


def test_captured_training_step():
    """Forward and backward of the autograd form in one graph, replayed over other logits, tokens and weights."""
    z, tok = rows_of(30, 5001, BF16, 2).contiguous().requires_grad_(), tokens(30, 2, 5001, 1)
    w, c = torch.randn((30, 2), generator=gen(1), device=DEV), torch.randn((30,), generator=gen(2), device=DEV)

    def step():
        lp, H = scores.logprobs(z, tok, 0.9)
        return torch.autograd.grad((lp * w).sum() + (H * c).sum(), z)[0]
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        grad = step()
    for i in range(3):
        with torch.no_grad():
            z.copy_(rows_of(30, 5001, BF16, 30 + i))
        tok.copy_(tokens(30, 2, 5001, 40 + i))
        w.copy_(torch.randn((30, 2), generator=gen(50 + i), device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        sc.check_grad(z.detach(), grad, sc.reference(z.detach(), tok, 0.9), tok, w, c, 0.9)
        assert torch.equal(grad, step())


def test_weights_of_another_shape_are_refused():
    z, tok = rows_of(4, 100, FP32, 1), tokens(4, 2, 100, 1)
    f, f1 = scores.token_logprobs(z, tok), scores.token_logprobs(z, tok[:, 0])
    g, h = torch.randn((4, 2), generator=gen(1), device=DEV), torch.randn((4,), generator=gen(2), device=DEV)
    for bad in ((g.T, None), (g[:, 0], None), (g.view(2, 4), h), (g, h[:3]), (g[:, :1], h)):
        with pytest.raises(mars.MarsError):
            scores.token_logprobs_backward(z, tok, f, *bad)
    with pytest.raises(mars.MarsError):
        scores.token_logprobs_backward(z, tok[:, 0], f1, g[:, :1].T)
    assert torch.equal(scores.token_logprobs_backward(z, tok, f, g.flatten(), h[:, None]), scores.token_logprobs_backward(z, tok, f, g, h))
    one = scores.token_logprobs_backward(z, tok[:, 0], f1, g[:, 0])
    for t, w in ((tok[:, 0], g[:, :1]), (tok[:, :1], g[:, 0]), (tok[:, :1], g[:, :1])):
        assert torch.equal(scores.token_logprobs_backward(z, t, f1, w), one)


def test_ids_beyond_32_bits_are_outside():
    z = rows_of(6, 500, FP32, 1)
    tok = torch.tensor([[3, 2 ** 32 + 3], [2 ** 32, 7], [-2 ** 32, 2 ** 40 + 1]] * 2, device=DEV)
    ids = torch.tensor([0, 1, 2 ** 32, 2, 2 ** 33 + 1, -2 ** 32], device=DEV)
    got = scores.token_logprobs(z, tok, rows=ids)
    ref = sc.reference(z)["logp"]
    want = torch.zeros((6, 2), dtype=torch.float64, device=DEV)
    want[0, 0], want[1, 1], want[3, 0] = ref[0, 3], ref[1, 7], ref[2, 3]
    assert ((got["logprob"].double() - want).abs() <= sc.UNIT * (sc.SUM + 100)).all() and ((got["logprob"] == 0) == (want == 0)).all()
    assert (got["entropy"][[2, 4, 5]] == 0).all() and (got["entropy"][[0, 1, 3]] > 0).all()
    grad = scores.token_logprobs_backward(z, tok, scores.token_logprobs(z, tok), torch.ones((6, 2), device=DEV))
    assert (grad[2] == 0).all() and (grad[5] == 0).all() and (grad[0] != 0).any()


def test_refusals_of_the_binding():
    z = torch.zeros((4, 100), device=DEV)
    tok = torch.zeros((4, 2), dtype=torch.int32, device=DEV)
    f = scores.token_logprobs(z, tok)
    for bad in (lambda: scores.token_logprobs(z.half(), tok), lambda: scores.token_logprobs(z.T, tok[:1]),
                lambda: scores.token_logprobs(z, tok[:3]), lambda: scores.token_logprobs(z, tok, k=33),
                lambda: scores.token_logprobs(z, tok, k=101), lambda: scores.token_logprobs(z, tok, temperature=0.0),
                lambda: scores.token_logprobs(z, tok, temperature=float("nan")), lambda: scores.token_logprobs(z.cpu(), tok),
                lambda: scores.token_logprobs(z, torch.zeros((4, 1025), dtype=torch.int32, device=DEV)),
                lambda: scores.token_logprobs(z, tok, V=101), lambda: scores.token_logprobs(z[:1], tok[:1], V=101),
                lambda: scores.token_logprobs(z[:, :50], tok, V=60), lambda: scores.token_logprobs(z[:1].expand(4, 100), tok),
                lambda: scores.token_logprobs_backward(z[:, :50], tok, f, torch.zeros((4, 2), device=DEV), V=51),
                lambda: scores.token_logprobs(z, tok, out={"logprob": torch.empty((4, 3), device=DEV)}),
                lambda: scores.token_logprobs_backward(z, tok, f, torch.zeros((4, 3), device=DEV)),
                lambda: scores.token_logprobs_backward(z, tok, {"stats": f["stats"]}, torch.zeros((4, 2), device=DEV), torch.zeros(4, device=DEV)),
                lambda: scores.token_logprobs_backward(z, tok, f, torch.zeros((4, 2), device=DEV), out=torch.empty((4, 99), device=DEV)),
                lambda: scores.token_logprobs_backward(z, tok, f, torch.zeros((4, 2), device=DEV), out=z.bfloat16())):
        with pytest.raises(mars.MarsError):
            bad()

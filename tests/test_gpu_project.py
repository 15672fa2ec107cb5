"""The 8-bit output projection on the device.  Codes, sums and every rounding of the call are defined, so all
comparisons are bit for bit."""
import ctypes

import numpy as np
import pytest
import torch

import hookctl as hooks
import scores_checks as sc
from paper_2601_15498_b200 import kv_cache, mars, scores

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, FP16, FP32 = torch.bfloat16, torch.float16, torch.float32


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def codes(R, K, seed, shift=0, full=False):
    """[R, K] codes in rows of a multiple of 16 bytes between guard values, scales of both signs of exponent."""
    wide = torch.full((R + 2, -(-K // 16) * 16 + 16 * shift), 99, dtype=torch.int8, device=DEV)
    q = wide[1:R + 1, :K]
    q.copy_(torch.randint(-127, 128, (R, K), generator=gen(seed), device=DEV) if not full else
            torch.full((R, K), 127, device=DEV) * (1 - 2 * (torch.arange(R, device=DEV) % 2))[:, None])
    return q, torch.exp2(torch.randn((R,), generator=gen(seed + 1), device=DEV) * 3) * 1e-3


def plain(q, s, w, u, bias, dtype):
    y = (q.double() @ w.double().T).float() * s[:, None]
    # a product of two fp32 numbers is exact in 64 bits: with the bias, one rounding in all
    y = (y.double() * u[None] + (0.0 if bias is None else bias.double()[None])).float()
    return y.to(dtype)


@pytest.mark.parametrize("M,V,K", [(1, 1, 1), (1, 300, 64), (2, 256, 128), (3, 257, 129), (31, 1000, 1000), (33, 640, 4096),
                                   (100, 77, 31), (255, 513, 200), (256, 4096, 512), (257, 700, 384), (333, 3001, 5000),
                                   (513, 2049, 130), (700, 256, 16), (1, 151936, 256), (64, 20000, 2048), (1025, 130, 8192)])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_product(M, V, K, dtype):
    (q, s), (w, u) = codes(M, K, M + K, shift=1), codes(V, K, V + 7, shift=M % 2)
    bias = torch.randn((V,), generator=gen(3), device=DEV) if M % 2 else None
    wide = torch.full((M + 1, V + 5), -777.0, dtype=dtype, device=DEV)
    out = wide[:M, 2:2 + V] if V % 2 else wide[:M, :V]
    got = scores.project_int8(q, s, w, u, bias=bias, out=out)
    assert got is out and torch.equal(out, plain(q, s, w, u, bias, dtype))
    at = 2 if V % 2 else 0
    assert (wide[M] == -777).all() and (wide[:, :at] == -777).all() and (wide[:, at + V:] == -777).all()


@pytest.mark.parametrize("M,V,K", [(33, 640, 4096), (256, 4096, 512), (700, 256, 16), (64, 20000, 2048), (40, 900, 6000),
                                   (1025, 130, 8192), (300, 25000, 512), (17, 2, 100), (272, 1000, 129), (1, 151936, 256)])
@pytest.mark.parametrize("pad", [0, 2, 5])
@pytest.mark.parametrize("biased", [False, True])
def test_pairs_of_logits_in_one_word(M, V, K, pad, biased):
    """bf16 logits of even V, row stride and 4-byte alignment are written two at a time: whole and partial groups of tokens,
    several groups and tiles, whole and cut tiles; a padding of 5 takes the other way to the same bits."""
    (q, s), (w, u) = codes(M, K, M + K), codes(V, K, V + 7)
    bias = torch.randn((V,), generator=gen(3), device=DEV) if biased else None
    want = plain(q, s, w, u, bias, BF16)
    wide = torch.full((M + 2, V + pad), -777.0, dtype=BF16, device=DEV)
    for at in (0,) if not pad else (0, pad - 1, pad):
        wide.fill_(-777.0)
        out = wide[1:M + 1, at:at + V]
        scores.project_int8(q, s, w, u, bias=bias, out=out)
        assert torch.equal(out, want)
        assert (wide[[0, -1]] == -777).all() and (wide[:, :at] == -777).all() and (wide[:, at + V:] == -777).all()


@pytest.mark.parametrize("V", [1, 15, 33, 255, 257, 1001, 4111])
@pytest.mark.parametrize("M,K", [(256, 128), (130, 4000), (33, 20000)])
def test_warps_with_lanes_beyond_the_last_weight_row(M, V, K):
    """Several groups of tokens per warp, whole and cut tiles, a last weight tile of any width: lanes that have no
    weight row are back for the next group's load."""
    (q, s), (w, u) = codes(M, K, 1), codes(V, K, 2)
    work = scores.project_workspace(M, V, K, DEV)
    for dtype in (BF16, FP32):
        want = plain(q, s, w, u, None, dtype)
        for _ in range(3):
            assert torch.equal(scores.project_int8(q, s, w, u, dtype=dtype, workspace=work), want)


def test_largest_sums_are_exact():
    """127 * 127 * 2^17 stays below 2^31, and a float that is halfway goes to the even one."""
    K = 1 << 17
    (q, s), (w, u) = codes(3, K, 1, full=True), codes(300, K, 2, full=True)
    q[2] = torch.randint(-127, 128, (K,), generator=gen(5), device=DEV).to(torch.int8)
    got = scores.project_int8(q, s, w, u, dtype=FP32)
    assert torch.equal(got, plain(q, s, w, u, None, FP32))
    assert float(got[0, 0] / (s[0] * u[0])) == pytest.approx(127 * 127 * K, rel=2 ** -21)


def test_workspace_serves_calls_of_one_size_after_another():
    """A workspace zeroed once: split tiles (few weight rows, long K) leave it as they found it."""
    M, V, K = 40, 900, 6000
    (w, u) = codes(V, K, 3)
    work = scores.project_workspace(M, V, K, DEV)
    for i in range(5):
        q, s = codes(M, K, 10 + i)
        assert torch.equal(scores.project_int8(q, s, w, u, dtype=FP32, workspace=work), plain(q, s, w, u, None, FP32))
        assert int(work[:4].view(torch.int32)) == 0
    small = codes(7, 640, 4)
    (w2, u2) = codes(5000, 640, 5)
    assert torch.equal(scores.project_int8(*small, w2, u2, workspace=work), plain(*small, w2, u2, None, BF16))


def test_streams_and_graph():
    M, V, K = 70, 5003, 1500
    (q, s), (w, u) = codes(M, K, 1), codes(V, K, 2)
    want = plain(q, s, w, u, None, BF16)
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    works = [scores.project_workspace(M, V, K, DEV) for _ in side]
    torch.cuda.synchronize()
    many = []
    for i in range(8):
        with torch.cuda.stream(side[i % 2]):
            many.append(scores.project_int8(q, s, w, u, workspace=works[i % 2]))
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for x in many)
    x = torch.randn((M, K), generator=gen(3), device=DEV).to(BF16)
    out = torch.empty((M, V), dtype=BF16, device=DEV)
    pair = scores.quantize_rows(x)
    graphs = []
    for _ in range(2):                                 # two graphs, one workspace
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            scores.project_int8(*scores.quantize_rows(x, out=pair), w, u, out=out, workspace=works[0])
        graphs.append(graph)
    for i in range(4):
        x.copy_(torch.randn((M, K), generator=gen(30 + i), device=DEV).to(BF16))
        out.zero_()
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        assert torch.equal(out, plain(*scores.quantize_rows(x), w, u, None, BF16))


@pytest.mark.parametrize("between", ["quantize_rows", "token_logprobs", "topk_rows", "project_int8", "verify_tree", "append"])
@pytest.mark.parametrize("use_graph", [False, True])
def test_logits_of_the_call_before_last_are_complete(between, use_graph):
    """MARS_LOGITS_READY vouches that the operation right before the call does not produce its logits.  The projection
    two calls before may: whatever stands between them, the verification sees all of its logits."""
    B, N, V, K = 24, 8, 30000, 640
    (w, u), (small, su) = codes(V, K, 1), codes(300, 64, 2)
    xs = [codes(B * N, K, 10 + i) for i in range(2)]
    want = [plain(*x, w, u, None, BF16) for x in xs]
    tok = want[0].argmax(1).view(B, N).int()
    parent = torch.arange(-1, N - 1, device=DEV, dtype=torch.int32)
    rounds, flags = 12, mars.COUNTERS_ZERO | mars.LOGITS_READY
    ws = torch.zeros(mars.workspace_bytes(B, N, V, mars.BF16), dtype=torch.uint8, device=DEV)
    ws2 = torch.zeros_like(ws)
    ref = [{k: t.clone() for k, t in mars.verify_tree(z, tok, parent, 0.9, debug=True).items() if k != "_keepalive"} for z in want]
    outs = [mars.alloc_outputs(B, N, N - 1, DEV, debug=True) for _ in range(rounds)]
    spare = mars.alloc_outputs(B, N, N - 1, DEV)
    logits = torch.zeros((B * N, V), dtype=BF16, device=DEV)
    work, work2 = scores.project_workspace(B * N, V, K, DEV), scores.project_workspace(1, 300, 64, DEV)
    row = torch.randn((1, 64), generator=gen(3), device=DEV)
    pair, few = scores.quantize_rows(row), torch.randn((1, 5000), generator=gen(4), device=DEV)
    lp = scores.token_logprobs(few)
    topk = (torch.empty((1, 4), device=DEV), torch.empty((1, 4), dtype=torch.int32, device=DEV))
    work_k = torch.empty(int(mars.lib().mars_topk_workspace_bytes(1, 5000, mars.FP32, 4)), dtype=torch.uint8, device=DEV)
    cache = kv_cache.KVCache.empty(1, 2, 1, 64, 16, 1, 2, DEV)
    kv_cache.resize(cache, torch.tensor([8], dtype=torch.int32, device=DEV))
    kv = torch.randn((1, 1, 1, 64), generator=gen(5), device=DEV).to(BF16)
    other = {"quantize_rows": lambda: scores.quantize_rows(row, out=pair), "token_logprobs": lambda: scores.token_logprobs(few, out=lp),
             "topk_rows": lambda: mars.topk_rows(few, 4, out=topk, workspace=work_k),
             "project_int8": lambda: scores.project_int8(*pair, small, su, workspace=work2),
             "verify_tree": lambda: mars.verify_tree(want[1], tok, parent, 0.9, flags=mars.COUNTERS_ZERO, workspace=ws2, out=spare),
             "append": lambda: kv_cache.append(cache, 0, kv, kv)}[between]
    mars.verify_tree(want[0], tok, parent, 0.9, workspace=ws)
    torch.cuda.synchronize()

    def run_all():
        for i in range(rounds):
            scores.project_int8(*xs[i % 2], w, u, out=logits, workspace=work)
            other()
            mars.verify_tree(logits, tok, parent, 0.9, flags=flags, workspace=ws, out=outs[i])
    if use_graph:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run_all()
        graph.replay()
        graph.replay()
    else:
        run_all()
    torch.cuda.synchronize()
    for i in range(rounds):
        for k, t in ref[i % 2].items():
            assert torch.equal(outs[i][k], t), (i, k)


@pytest.mark.parametrize("M,V,K", [(1, 151936, 256), (40, 32000, 1024), (333, 5001, 300)])
@pytest.mark.parametrize("use_graph", [False, True])
def test_calls_read_what_their_predecessor_writes(M, V, K, use_graph):
    """Projection, log probabilities, a gradient in the logits' place and the log probabilities of that, over and over with
    nothing in between: bit for bit what the calls give one at a time."""
    (w, u) = codes(V, K, 1)
    xs = [codes(M, K, 10 + i) for i in range(3)]
    tok = torch.randint(0, V, (M, 2), generator=gen(2), device=DEV).to(torch.int32)
    g = torch.randn((M, 2), generator=gen(3), device=DEV)
    work, logits = scores.project_workspace(M, V, K, DEV), torch.zeros((M, V), dtype=BF16, device=DEV)

    def step(x):
        scores.project_int8(*x, w, u, out=logits, workspace=work)
        first = scores.token_logprobs(logits, tok, k=3)
        yield first
        scores.token_logprobs_backward(logits, tok, first, g, out=logits)
        yield scores.token_logprobs(logits, tok)
    want = []
    for x in xs:
        one = []
        for got in step(x):
            torch.cuda.synchronize()
            one.append({n: t.clone() for n, t in got.items()})
        want.append(one)
    assert not torch.equal(want[0][0]["logprob"], want[1][0]["logprob"])

    def run_all():
        return [list(step(xs[i % 3])) for i in range(12)]
    if use_graph:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            many = run_all()
        graph.replay()
        graph.replay()
    else:
        many = run_all()
    torch.cuda.synchronize()
    for i, pair in enumerate(many):
        for got, ref in zip(pair, want[i % 3]):
            for n in ref:
                assert torch.equal(torch.nan_to_num(got[n]), torch.nan_to_num(ref[n])), (i, n)


def quantised(x):
    x = x.float()
    a = x.abs().amax(1)
    a = torch.where(torch.isnan(x).any(1), float("nan"), a)
    bad, zero = ~torch.isfinite(a), a < 2.0 ** -119
    r = torch.where(bad | zero, 0.0, a.reciprocal() * 127)
    q = torch.where(bad[:, None], 0.0, torch.round(x * r[:, None]))
    return q.to(torch.int8), torch.where(bad, float("nan"), torch.where(zero, 0.0, a / torch.full_like(a, 127)))     # (a number as divisor would become a product)


@pytest.mark.parametrize("R,K", [(1, 1), (3, 7), (5, 100), (2, 4096), (9, 5000), (1, 8191), (2, 20001), (4, 70000), (600, 64)])
@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
def test_quantise(R, K, dtype):
    for shift in (0, 1, 8):
        wide = (torch.randn((R, K + 24), generator=gen(K), device=DEV) * torch.exp2(torch.randint(-9, 6, (R, 1), generator=gen(1), device=DEV).float())).to(dtype)
        x = wide[:, shift:shift + K]
        want = quantised(x)
        buf = torch.full((R + 1, -(-K // 16) * 16 + 16), 99, dtype=torch.int8, device=DEV)
        q, s = scores.quantize_rows(x, out=(buf[:R, :K], torch.empty((R,), device=DEV)))
        assert torch.equal(q, want[0]) and torch.equal(s, want[1])
        assert (buf[R] == 99).all() and (buf[:, K:] == 99).all()
        # a code is off by half a step at most, and by what x r and the scale round: 2^-24 of 127 each, thrice
        assert ((q.double() * s.double()[:, None] - x.double()).abs() <= s.double()[:, None] * (0.5 + 3 * 127 * 2.0 ** -24)).all()
        assert (q.abs().amax(1) == 127).all()


@pytest.mark.parametrize("dtype", [BF16, FP16, FP32])
def test_quantise_special_rows(dtype):
    x = torch.randn((8, 333), generator=gen(1), device=DEV).to(dtype)
    x[0] = 0.0
    x[1, 100] = float("nan")
    x[2, 332] = float("inf")
    x[3, 0] = float("-inf"); x[3, 1] = float("nan")
    x[4] = torch.finfo(dtype).max
    x[5] = torch.finfo(dtype).tiny
    x[6] = -0.0
    x[7] = 0.0; x[7, 7] = -1.0
    q, s = scores.quantize_rows(x)
    want = quantised(x)
    assert torch.equal(q, want[0]) and torch.equal(torch.nan_to_num(s, nan=-1.0), torch.nan_to_num(want[1], nan=-1.0))
    assert torch.isnan(s[1:4]).all() and (s[[0, 6]] == 0).all() and q[7, 7] == -127
    w, u = codes(40, 333, 2)
    y = scores.project_int8(q, s, w, u, dtype=FP32)
    # (row 4: the sum times the scale, a step of the definition, passes fp32's largest number: 127 * 2^15 * 2^121)
    assert torch.isnan(y[1:4]).all() and (y[0] == 0).all() and torch.isfinite(y[[0, 5, 6, 7]]).all()
    assert torch.equal(y[[0, 4, 5, 6, 7]], plain(q, s, w, u, None, FP32)[[0, 4, 5, 6, 7]])


def test_hidden_states_to_verified_tokens_and_their_log_probabilities():
    """The run of a decode step: quantise, project, verify, report; and the gradient of what was reported."""
    B, N, V, K = 3, 12, 5000, 512
    hidden = torch.randn((B * N, K), generator=gen(1), device=DEV).to(BF16)
    w = torch.randn((V, K), generator=gen(2), device=DEV).to(BF16) * 0.1
    wq, ws = scores.quantize_rows(w)
    logits = scores.project_int8(*scores.quantize_rows(hidden), wq, ws, dtype=FP32)
    # a row of codes is off by half a step of 1/127 of its largest: products of K such pairs
    step = hidden.float().abs().amax(1)[:, None] * w.float().abs().amax(1)[None] / 127
    far = step * (w.float().abs().sum(1) / w.float().abs().amax(1) + (hidden.float().abs().sum(1) / hidden.float().abs().amax(1))[:, None] + K / 127) * 0.51
    assert ((logits - hidden.float() @ w.float().T).abs() <= far).all()
    tok = logits.argmax(1).view(B, N)
    parent = torch.arange(-1, N - 1, device=DEV).expand(B, N)
    tok = torch.cat([tok[:, :1], tok[:, :-1]], 1)                   # every draft is the best token of its parent's row
    out = mars.verify_tree(logits, tok, parent, theta=0.9)
    assert (out["accept_len"] == N - 1).all()
    got = scores.emitted_logprobs(logits, out, k=3)
    ref = sc.reference(logits)
    want = ref["logp"].gather(1, logits.argmax(1)[:, None]).view(B, N)
    assert (got["logprob"].double() - want).abs().max() <= sc.UNIT * (sc.SUM + 200)
    assert torch.equal(got["top_id"][:, :, 0].long(), logits.argmax(1).view(B, N))
    z = logits.clone().requires_grad_()
    lp, _ = scores.logprobs(z, logits.argmax(1))
    lp.sum().backward()
    sc.check_grad(logits, z.grad, ref, logits.argmax(1)[:, None].int(), torch.ones((B * N, 1), device=DEV), None, 1.0)


@pytest.mark.parametrize("M,V,K", [(40, 900, 6000), (300, 25000, 512)])
def test_pairs_that_give_up_leave_nan_and_a_status(M, V, K):
    """What a wait that runs out leaves behind (through the test hook): logits that were not computed are NaN, the
    others right, the status says so, and zeroed counters make the workspace serve again."""
    (q, s), (w, u) = codes(M, K, 1), codes(V, K, 2)
    want = plain(q, s, w, u, None, FP32)
    work = scores.project_workspace(M, V, K, DEV)
    lost = []
    try:
        for first in (1, 2, 40, 75):
            mars.test_hook(mars.HOOK_PROJECT_GIVE_UP, first)
            got = scores.project_int8(q, s, w, u, dtype=FP32, workspace=work)
            torch.cuda.synchronize()
            gone = torch.isnan(got)
            assert torch.equal(got[~gone], want[~gone])
            lost.append(int(gone.sum()))
            # a call that runs fewer pairs than `first` - 1 loses nothing and reports nothing
            assert int(work[:4].view(torch.int32)) == (3 if lost[-1] else 0)
            work[:scores.PROJECT_COUNTER_BYTES].zero_()
    finally:
        mars.test_hook(mars.HOOK_PROJECT_GIVE_UP, 0)
    assert lost[0] == M * V and lost == sorted(lost, reverse=True) and lost[3] == 0 and lost[1] > 0
    assert torch.equal(scores.project_int8(q, s, w, u, dtype=FP32, workspace=work), want)
    assert int(work[:4].view(torch.int32)) == 0


@pytest.mark.parametrize("M,V,K", [(40, 900, 6000), (300, 25000, 512), (1, 20000, 4096), (256, 4096, 4096)])
def test_workspace_serves_calls_after_one_whose_pairs_gave_up(M, V, K):
    """The counters come back to zero whichever pairs give up, so a call that follows has every logit right without any
    clearing, and a status of its own."""
    (q, s), (w, u) = codes(M, K, 1), codes(V, K, 2)
    (q2, s2) = codes(M, K, 3)
    want, want2 = plain(q, s, w, u, None, FP32), plain(q2, s2, w, u, None, FP32)
    work = scores.project_workspace(M, V, K, DEV)
    counters = work[256:scores.PROJECT_COUNTER_BYTES].view(torch.int32)
    for first in (1, 2, 3, 17, 40, 60, 74, 75):
        try:
            mars.test_hook(mars.HOOK_PROJECT_GIVE_UP, first)
            got = scores.project_int8(q, s, w, u, dtype=FP32, workspace=work)
            torch.cuda.synchronize()
        finally:
            mars.test_hook(mars.HOOK_PROJECT_GIVE_UP, 0)
        gone = torch.isnan(got)
        assert torch.equal(got[~gone], want[~gone]), first
        assert int(work[:4].view(torch.int32)) == (3 if gone.any() else 0)
        assert not counters.any(), first
        got = scores.project_int8(q2, s2, w, u, dtype=FP32, workspace=work)
        assert torch.equal(got, want2), first
        assert int(work[:4].view(torch.int32)) == 0


def test_one_row_of_codes_out_of_a_matrix_of_any_stride():
    """A single row's stride is no distance between rows: 1 token, 1 weight row, 1 quantised row."""
    (q, s), (w, u) = codes(1, 100, 1), codes(40, 100, 2)
    odd = torch.zeros((3, 201), dtype=torch.int8, device=DEV)
    odd[0, :100] = q[0]
    assert torch.equal(scores.project_int8(odd[:1, :100], s, w, u), plain(q, s, w, u, None, BF16))
    assert torch.equal(scores.project_int8(w, u, odd[:1, :100], s, dtype=FP32), plain(w, u, q, s, None, FP32))
    x = torch.randn((1, 100), generator=gen(3), device=DEV)
    want = scores.quantize_rows(x)
    odd.fill_(99)
    got = scores.quantize_rows(x, out=(odd[:1, :100], torch.empty((1,), device=DEV)))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and (odd[1:] == 99).all() and (odd[0, 100:] == 99).all()


def test_a_failed_call_leaves_no_error_behind():
    """A stream operation that the runtime refuses (on the legacy stream, while a stream that waits for it is captured) is
    that call's error and no later one's."""
    with open("/proc/self/maps") as f:
        rt = ctypes.CDLL(next(line.split()[-1] for line in f if "libcudart" in line))
    (q, s), (w, u) = codes(4, 64, 1), codes(10, 64, 2)
    want = scores.project_int8(q, s, w, u)
    out, work = torch.empty_like(want), scores.project_workspace(4, 10, 64, DEV)
    z = torch.randn((3, 100), generator=gen(1), device=DEV)
    val, idx = mars.topk_rows(z, 2)
    torch.cuda.synchronize()
    stream, graph = ctypes.c_void_p(), ctypes.c_void_p()
    assert rt.cudaStreamCreate(ctypes.byref(stream)) == 0
    assert rt.cudaStreamBeginCapture(stream, 0) == 0
    try:
        code = mars.lib().mars_project_int8(q.data_ptr(), q.stride(0), s.data_ptr(), w.data_ptr(), w.stride(0), u.data_ptr(), None, 4, 10,
                                            64, out.data_ptr(), 10, mars.BF16, 0, work.data_ptr(), work.nbytes, None)
    finally:
        rt.cudaStreamEndCapture(stream, ctypes.byref(graph))
        rt.cudaStreamDestroy(stream)
        rt.cudaGetLastError()
    assert code == 4                                                         # MARS_ERR_CUDA
    again = mars.topk_rows(z, 2)
    assert torch.equal(again[0], val) and torch.equal(again[1], idx)
    assert torch.equal(scores.project_int8(q, s, w, u), want)


def test_refusals_of_the_binding():
    (q, s), (w, u) = codes(4, 64, 1), codes(10, 64, 2)
    good = scores.project_workspace(4, 10, 64, DEV)
    for bad in (lambda: scores.project_int8(q, s[:3], w, u), lambda: scores.project_int8(q.float(), s, w, u),
                lambda: scores.project_int8(q, s.double(), w, u), lambda: scores.project_int8(q[:, :32], s, w, u),
                lambda: scores.project_int8(q, s, w, u, dtype=FP16), lambda: scores.project_int8(q, s, w, u, bias=torch.zeros(9, device=DEV)),
                lambda: scores.project_int8(q, s, w, u, out=torch.empty((4, 9), device=DEV)),
                lambda: scores.project_int8(q, s, w, u, workspace=good[:100]),
                lambda: scores.project_int8(q, s, w, u, workspace=good[1:]),
                lambda: scores.project_int8(q[:, 1:17], s, w[:, :16], u), lambda: scores.project_int8(q.cpu(), s.cpu(), w, u),
                lambda: scores.quantize_rows(q), lambda: scores.quantize_rows(s), lambda: scores.quantize_rows(torch.zeros((2, 64))),
                lambda: scores.quantize_rows(torch.zeros((2, 20), device=DEV), out=(torch.empty((2, 20), dtype=torch.int8, device=DEV), torch.empty(2, device=DEV))),
                lambda: scores.project_workspace(0, 10, 64, DEV)):
        with pytest.raises(mars.MarsError):
            bad()

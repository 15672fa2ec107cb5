"""The paged 4-bit KV cache on the device against the plain model: tables and stored bytes exactly,
attention within bounds that count its roundings."""
import numpy as np
import pytest
import torch

import hookctl as hooks
from oracle import kv_oracle as ko
from paper_2601_15498_b200 import kv_cache as kv, mars, synth

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NP = {torch.bfloat16: np.float32, torch.float16: np.float32, torch.float32: np.float32}


def i32(x):
    return torch.as_tensor(np.asarray(x, np.int32), device=DEV)


def host(t):
    return t.float().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


class Pair:
    """A device cache and its model, driven side by side."""

    def __init__(self, layers=1, pages=64, heads=2, d=128, page=16, seqs=4, width=12, seed=0, scales="pow2"):
        self.rng = np.random.default_rng(seed)
        g = np.exp2(self.rng.integers(-3, 3, (layers, 2, heads))) if scales == "pow2" \
            else self.rng.uniform(0.05, 3.0, (layers, 2, heads))
        self.c = kv.KVCache.empty(layers, pages, heads, d, page, seqs, width, DEV, scales=g.astype(np.float32))
        # what nobody wrote is garbage, NaN scales among it
        self.c.pages.copy_(torch.as_tensor(self.rng.integers(0, 256, self.c.pages.shape, dtype=np.uint8)))
        self.m = ko.Model(layers, pages, heads, d, page, seqs, width, g)

    def resize(self, extra, check=True):
        st = torch.full((self.c.seqs,), -7, dtype=torch.int32, device=DEV)
        kv.resize(self.c, i32(extra), status=st)
        want = self.m.resize(extra)
        if check:
            self.tables()
            assert np.array_equal(host(st), want)
        return want

    def tables(self):
        torch.cuda.synchronize()
        c, m = self.c, self.m
        for name, a, b in (("table", c.block_table, m.table), ("len", c.seq_len, m.len), ("held", c.seq_pages, m.held),
                           ("refs", c.page_refs, m.refs), ("free", c.free_bits, m.free_bits())):
            assert np.array_equal(host(a), b), name

    def rand(self, B, N, dtype, loud=True):
        x = self.rng.standard_normal((B, N, self.m.H, self.m.d))
        if loud:
            x *= np.exp2(self.rng.integers(-6, 7, (B, N, 1, 1)))
        return torch.as_tensor(x, device=DEV).to(dtype)

    def append(self, B, N, dtype=torch.bfloat16, count=None, k=None, v=None):
        for layer in range(self.m.L):
            k1 = self.rand(B, N, dtype) if k is None else k
            v1 = self.rand(B, N, dtype) if v is None else v
            st = torch.full((B,), -7, dtype=torch.int32, device=DEV)
            kv.append(self.c, layer, k1, v1, count=None if count is None else i32(count), status=st)
            assert np.array_equal(host(st), self.m.append(layer, host(k1), host(v1), count))

    def grow(self, lens):
        """Committed tokens: room, rows, lengths."""
        ex = [-2] * self.m.S
        ex[:len(lens)] = lens
        assert (self.resize(ex, check=False)[:len(lens)] == 0).all()
        self.append(len(lens), max(max(lens), 1), count=lens)
        path = [n - 1 for n in lens]
        kv.commit(self.c, None, i32(path))
        self.m.len[:len(lens)], st = self.m.commit(None, path)
        assert (st == 0).all()

    def stored(self):
        """Bytes of every written slot agree; the model keeps zeros where nothing was written."""
        got = host(self.c.pages)
        d, nb = self.m.d, self.m.page // 16
        a = got.reshape(*got.shape[:3], nb, 18 * d)
        b = self.m.pool().reshape(a.shape)
        for b_ in range(self.m.S):
            upto = self.m.len[b_]
            for pos in range(upto):
                p, s = self.m.at(b_, pos)
                for lo, w in ((0, d // 2), (8 * d, d // 2), (16 * d, d // 16), (17 * d, d // 16)):
                    x = a[:, p, :, s // 16, lo + (s % 16) * w:lo + (s % 16 + 1) * w]
                    y = b[:, p, :, s // 16, lo + (s % 16) * w:lo + (s % 16 + 1) * w]
                    assert np.array_equal(x, y), (b_, pos, lo)


def trees(rng, B, N, absent=0.0):
    p = np.full((B, N), -1, np.int32)
    for i in range(1, N):
        p[:, i] = (rng.uniform(0, 1, B) ** 1.5 * i).astype(np.int32)
        p[rng.uniform(0, 1, B) < absent, i] = -1
    return p


def check_attention(pr, q, parent=None, count=None, scale=None, layer=0, out=None, workspace=None):
    B, N, Hq, d = q.shape
    out = torch.full((B, N, Hq, d), 7.25, dtype=q.dtype, device=DEV) if out is None else out
    before = host(out).copy()
    st = torch.full((B,), -7, dtype=torch.int32, device=DEV)
    kv.tree_attention(q, pr.c, layer, None if parent is None else i32(parent), count=None if count is None else i32(count),
                      scale=scale, out=out, status=st, workspace=workspace)
    torch.cuda.synchronize()
    want, live, status, mag, tot, amp = ko.attention(pr.m, layer, host(q).astype(np.float64), parent, count, scale)
    assert np.array_equal(host(st), status)
    got = host(out).astype(np.float64)
    assert np.array_equal(got[~live], before[~live].astype(np.float64))       # rows without a result stay
    # Roundings, relative to the probability-weighted |V| (mag):
    #   P to fp16: 2^-11 each while it is a normal number; P is 2^7 or more at the row's largest score, so a
    #   smaller one is off by at most 2^-25, that is 2^-32 of the largest probability, hence of 1: 2^-32 of
    #   the plain sum of |V| (tot).  A score is a sum of d products with fp32 accumulation, off by at most
    #   d * 2^-23 of sum |q||k| (amp, times log2 e in the kernel's units, back by ln 2), four more roundings
    #   (scale, maximum, exponential) at 2^-23 of its size; a shift of a score moves a probability by that
    #   fraction, and the sum below it too: twice.  q to fp16 after scaling: below 2^-25 of the row's largest
    #   element, covered by one more 2^-23 of amp per element.  Sums over keys: keys * 2^-23.
    # then half a step of the output type.
    keys = int(pr.m.len.max()) + N
    rel = 2.0 ** -11 + 2 * (2 * d + 8) * 2.0 ** -23 * amp[..., None] + 2 * (keys + 64) * 2.0 ** -23
    half = torch.finfo(q.dtype).eps / 2
    tol = mag * rel + tot * 2.0 ** -32
    tol = tol + half * (np.abs(want) + tol) + 2.0 ** -24
    err = np.abs(got - want)
    bad = (err > tol) & live[..., None, None]
    assert not bad.any(), (np.argwhere(bad)[:3], err[bad][:3], tol[bad][:3], want[bad][:3])
    assert not np.isnan(got[live]).any()
    return out


# ------------------------------------------------------------------------------------- append, gather

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_append_stores_what_the_model_stores(d, page):
    pr = Pair(layers=2, pages=40, heads=3, d=d, page=page, seqs=3, width=9, seed=d + page)
    pr.grow([35, 0, 17])
    pr.stored()
    pr.resize([20, 3, 0])
    pr.append(3, 20, torch.float16, count=[20, 3, 40])       # the last one has no room
    pr.m.len[:] = [35 + 20, 3, 17]
    pr.stored()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("scales", ["pow2", "any"])
def test_append_types_scales_and_special_values(dtype, scales):
    pr = Pair(heads=2, d=64, page=32, seqs=2, width=4, seed=5, scales=scales)
    pr.resize([64, 64])
    k, v = pr.rand(2, 64, dtype), pr.rand(2, 64, dtype)
    k[0, 0, 0, :5] = torch.tensor([float("nan"), float("inf"), -float("inf"), -0.0, 0.0], device=DEV).to(dtype)
    k[0, 1] = 0
    v[0, 2] = torch.finfo(dtype).max
    v[1, 3] = torch.finfo(dtype).smallest_normal
    v[1, 4, :, :16] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0] * 2, device=DEV).to(dtype)   # borders
    pr.append(2, 64, dtype, k=k, v=v)
    pr.m.len[:] = 64
    pr.stored()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_append_keeps_the_sign_of_zeros(dtype):
    """-0 / (s * g) is -0 and has the code 8; under a scale of 0 all codes are 0."""
    pr = Pair(d=64, page=16, seqs=2, width=4, seed=90)
    pr.resize([9, 9])
    k, v = pr.rand(2, 9, dtype), pr.rand(2, 9, dtype)
    k[..., ::3] = -0.0
    v[..., 1::2] = 0.0
    v[:, 4] = -0.0
    pr.append(2, 9, k=k, v=v)
    pr.m.len[:2] = 9
    pr.stored()


def test_append_of_strided_slices_and_gather_back():
    pr = Pair(heads=2, d=128, page=64, seqs=3, width=4, seed=6)
    pr.resize([30, 30, 30])
    qkv = torch.randn((3, 30, 4 + 2 + 2, 128), device=DEV).to(torch.bfloat16)
    k, v = qkv[:, :, 4:6], qkv[:, :, 6:]
    pr.append(3, 30, k=k, v=v)
    pr.m.len[:] = 30
    pr.stored()
    for dtype in (torch.float32, torch.bfloat16, torch.float16):
        ko_, vo_ = kv.gather(pr.c, 0, 1, i32([3, 0, 90]), i32([27, 11, 9]), rows=27, dtype=dtype)
        for b, (s, n) in enumerate(((3, 27), (0, 11), (90, 0))):
            want = pr.m.rows(0, b, s, n) if n else [np.zeros((0, 2, 128))] * 2
            for got, w in zip((ko_, vo_), want):
                w = torch.as_tensor(w).float().to(dtype).float().numpy()      # 6 bits times a power of two: exact
                assert np.array_equal(host(got)[0, b, :n], w)
                assert (host(got)[0, b, n:] == 0).all()


def test_fp32_rows_of_one_token_and_odd_counts():
    pr = Pair(layers=3, pages=10, heads=1, d=64, page=16, seqs=5, width=3, seed=8)
    pr.resize([1, 2, 16, 17, 0])
    pr.append(5, 17, torch.float32, count=[1, 2, 16, 17, -4])
    pr.m.len[:] = [1, 2, 16, 17, 0]
    pr.stored()


# ------------------------------------------------------------------------------------- tables

def test_resize_grows_trims_releases_and_runs_out():
    pr = Pair(pages=70, heads=1, d=64, page=16, seqs=40, width=6, seed=9)
    rng = np.random.default_rng(10)
    seen = set()
    for step in range(12):
        ex = rng.integers(-2, 60, 40)
        ex[rng.integers(0, 40, 4)] = 2000                     # wider than the table
        seen |= set(pr.resize(ex).tolist())
        ln = [int(rng.integers(0, h * 16 + 1)) for h in pr.m.held]
        pr.m.len[:] = ln
        pr.c.seq_len.copy_(i32(ln))
        if step % 3 == 2:
            pr.resize([-1] * 20 + [0] * 20)
    assert seen == {0, ko.NO_ROOM, ko.OUT_OF_PAGES}
    pr.resize([-1] * 40)
    assert (pr.m.refs == 0).all()


@pytest.mark.parametrize("pages,seqs", [(1, 1), (31, 3), (33, 2), (40000, 1500), (140001, 8192)])
def test_resize_of_small_and_large_pools(pages, seqs):
    pr = Pair(pages=pages, heads=1, d=64, page=16, seqs=seqs, width=40, seed=pages)
    rng = np.random.default_rng(seqs)
    for _ in range(2):
        pr.resize(rng.integers(-2, 500, seqs))
    pr.resize(np.where(rng.uniform(0, 1, seqs) < 0.5, -1, 0))


def test_fork_shares_pages_and_copies_the_ragged_one():
    pr = Pair(layers=2, pages=60, heads=2, d=128, page=32, seqs=10, width=6, seed=11)
    pr.grow([70, 64, 5, 0, 33])
    src = [0, 0, 1, 2, 3, 9, 4, 4, 0, -1, 2, 5]
    dst = [5, 6, 7, 8, 9, 3, 4, 8, 1, 2, 77, 9]     # empty source, self, taken twice, not empty, out of range
    st = kv.fork(pr.c, i32(src), i32(dst))
    want = pr.m.fork(src, dst)
    assert np.array_equal(host(st), want)
    assert want.tolist() == [0, 0, 0, 0, 0, 0, 9, 9, 9, 9, 9, 9]
    pr.tables()
    pr.stored()
    # both go on by themselves
    pr.resize([40] * 9 + [-2])
    pr.append(9, 40)
    pr.m.len[:9] += 40
    pr.c.seq_len.copy_(i32(pr.m.len))
    pr.stored()
    pr.resize([-1, -1, -2, -2, -2, -2, -2, 0, 0, 0])
    pr.tables()
    pr.stored()


def test_fork_out_of_pages():
    pr = Pair(pages=8, heads=1, d=64, page=16, seqs=9, width=4, seed=12)
    pr.grow([20, 16, 40])                                     # 2 + 1 + 3 of 8 pages
    src, dst = [0, 1, 2, 0, 1], [3, 4, 5, 6, 7]
    st = kv.fork(pr.c, i32(src), i32(dst))
    want = pr.m.fork(src, dst)
    assert np.array_equal(host(st), want) and want.tolist() == [0, 0, 0, 7, 0]
    pr.tables()
    pr.stored()


# ------------------------------------------------------------------------------------- commit

@pytest.mark.parametrize("d,page", [(64, 16), (128, 64)])
@pytest.mark.parametrize("in_place", [True, False])
def test_commit_moves_the_path(d, page, in_place):
    pr = Pair(layers=3, pages=64, heads=2, d=d, page=page, seqs=7, width=10, seed=13)
    pr.grow([11, 30, 0, 16, 5, 7, 9])
    pr.resize([50] * 7)
    pr.append(7, 50)
    path = np.full((7, 30), -1, np.int32)
    acc = np.zeros(7, np.int32)
    for b, nodes in enumerate(([0, 1, 2, 3], [0, 7, 9, 30, 31, 49], [0], list(range(0, 50, 2)), [0, 3, 3], [0, 4, 90],
                               [])):
        path[b, :len(nodes)] = nodes
        acc[b] = len(nodes) - 1
    path[3, 25:] = 7
    new = None if in_place else torch.full((7,), -5, dtype=torch.int32, device=DEV)
    st = torch.full((7,), -7, dtype=torch.int32, device=DEV)
    got = kv.commit(pr.c, i32(path), i32(acc), new_len=new, status=st)
    want, status = pr.m.commit(path, acc)
    assert np.array_equal(host(st), status) and status.tolist() == [0, 0, 0, 0, 8, 8, 0]
    assert np.array_equal(host(got), want)
    assert np.array_equal(host(pr.c.seq_len), want if in_place else pr.m.len)
    pr.m.len[:] = want
    pr.stored()


def test_commit_of_long_paths_and_bad_lengths():
    pr = Pair(layers=1, pages=200, heads=1, d=128, page=16, seqs=5, width=40, seed=14)
    pr.grow([3, 3, 3, 3, 3])
    pr.resize([200] * 5)
    pr.append(5, 200)
    path = np.tile(np.arange(0, 200, 3, dtype=np.int32), (5, 1))       # 67 nodes, several batches of a warp
    acc = np.array([66, 67, -2, 40, -1], np.int32)
    st = torch.zeros((5,), dtype=torch.int32, device=DEV)
    kv.commit(pr.c, i32(path), i32(acc), status=st)
    want, status = pr.m.commit(path, acc)
    assert np.array_equal(host(st), status) and status.tolist() == [0, 8, 8, 0, 0]
    pr.m.len[:] = want
    pr.tables()
    pr.stored()


# ------------------------------------------------------------------------------------- attention

@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads,group", [(2, 1), (1, 4), (2, 5), (1, 16), (1, 24)])
def test_attention_of_single_tokens(dtype, d, heads, group):
    lens = [0, 1, 15, 16, 17, 63, 64, 65, 200, 331]
    pr = Pair(pages=120, heads=heads, d=d, page=16, seqs=10, width=22, seed=group + d)
    pr.grow(lens)
    pr.resize([1] * 10)
    pr.append(10, 1, dtype)
    q = torch.randn((10, 1, heads * group, d), device=DEV).to(dtype)
    check_attention(pr, q)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d,page", [(64, 32), (128, 64)])
@pytest.mark.parametrize("N", [2, 6, 33, 60, 65])
def test_attention_of_trees(dtype, d, page, N):
    rng = np.random.default_rng(N)
    lens = [0, 1, 100, 64, 130]
    pr = Pair(pages=60, heads=2, d=d, page=page, seqs=5, width=10, seed=N)
    pr.grow(lens)
    pr.resize([N] * 5)
    pr.append(5, N, dtype)
    q = torch.randn((5, N, 4, d), device=DEV).to(dtype)
    check_attention(pr, q, parent=trees(rng, 5, N))
    count = np.array([N, N // 2, 0, 1, N + 9], np.int32)
    check_attention(pr, q, parent=trees(rng, 5, N, absent=0.15), count=count)
    check_attention(pr, q, parent=trees(rng, 1, N)[0], count=count)


@pytest.mark.parametrize("d,group", [(64, 1), (128, 3), (128, 8), (64, 32)])
@pytest.mark.parametrize("N", [3, 8, 77, 150])
def test_attention_of_chains(d, group, N):
    lens = [0, 50, 7, 129]
    pr = Pair(pages=140, heads=1, d=d, page=16, seqs=4, width=20, seed=N + d)
    pr.grow(lens)
    pr.resize([N] * 4)
    pr.append(4, N)
    q = torch.randn((4, N, group, d), device=DEV).to(torch.float16)
    check_attention(pr, q)
    check_attention(pr, q, count=[N, N - 1, 1, 0], scale=0.31)


def test_attention_of_a_large_tree():
    N = 1024
    pr = Pair(pages=80, heads=1, d=64, page=32, seqs=2, width=40, seed=3)
    pr.grow([33, 2])
    pr.resize([N, N])
    pr.append(2, N)
    q = torch.randn((2, N, 2, 64), device=DEV).to(torch.bfloat16)
    check_attention(pr, q, parent=trees(np.random.default_rng(4), 2, N), count=[N, 700])


def test_attention_statuses_and_untouched_rows():
    pr = Pair(pages=60, heads=2, d=64, page=16, seqs=6, width=8, seed=21)
    pr.grow([20, 30, 40, 5, 6, 0])
    pr.resize([6, 2, 6, 6, 6, 6])                 # sequence 1 has room for 34 tokens, not 36... its page holds 32
    pr.append(6, 6)
    parent = trees(np.random.default_rng(1), 6, 6)
    parent[2, 3] = 4                              # no tree
    parent[3, 0] = 0
    parent[4, 5] = -2
    pr.m.len[5] = -3                              # nonsense length
    pr.c.seq_len.copy_(i32(pr.m.len))
    q = torch.randn((6, 6, 4, 64), device=DEV).to(torch.bfloat16)
    check_attention(pr, q, parent=parent, count=[6, 6, 6, 6, 6, 6])


def test_attention_large_scores_and_special_rows_of_q():
    pr = Pair(pages=40, heads=1, d=128, page=16, seqs=3, width=12, seed=22)
    pr.grow([90, 17, 3])
    pr.resize([4] * 3)
    pr.append(3, 4)
    q = torch.randn((3, 4, 2, 128), device=DEV)
    q[0, 0] *= 1e-30                              # scores of nothing: the mean of V
    q[0, 1] = 0
    q[1, 2] *= 3e-3
    q[2, 0, :, ::2] *= 1e-4
    check_attention(pr, q.to(torch.bfloat16))
    # scores of thousands (one-hot rows): the bound on a probability grows with them, the row stays finite
    big = (q * 500).to(torch.bfloat16)
    out = kv.tree_attention(big, pr.c, 0)
    assert torch.isfinite(out).all()
    nan = q.to(torch.bfloat16)
    nan[0, 0, 0, 3] = float("nan")
    out = kv.tree_attention(nan, pr.c, 0)
    assert out[0, 0, 0].isnan().all() and torch.isfinite(out[0, 0, 1]).all() and torch.isfinite(out[1:]).all()


def test_attention_of_strided_q_and_out_in_a_second_layer():
    pr = Pair(layers=2, pages=40, heads=2, d=128, page=16, seqs=3, width=12, seed=23)
    pr.grow([90, 17, 3])
    pr.resize([5] * 3)
    pr.append(3, 5)
    qkv = torch.randn((3, 5, 4 + 2 + 2, 128), device=DEV).to(torch.bfloat16)
    wide = torch.full((3, 5, 6, 128), 7.25, dtype=torch.bfloat16, device=DEV)
    check_attention(pr, qkv[:, :, :4], layer=1, out=wide[:, :, 1:5])
    assert (wide[:, :, 0] == 7.25).all() and (wide[:, :, 5] == 7.25).all()


def test_page_ids_outside_the_pool_are_not_followed():
    """A damaged table entry (no call writes one) is read as NaN for its sequence alone."""
    pr = Pair(pages=40, heads=2, d=64, page=16, seqs=3, width=12, seed=24)
    pr.grow([90, 50, 20])
    pr.resize([2] * 3)
    pr.append(3, 2)
    q = torch.randn((3, 2, 4, 64), device=DEV).to(torch.bfloat16)
    good = kv.tree_attention(q, pr.c, 0)
    for bad in (-1, 40, 1 << 30, -(1 << 31)):
        pr.c.block_table[1, 1] = bad
        out = kv.tree_attention(q, pr.c, 0)
        assert out[1].isnan().all() and torch.equal(out[0], good[0]) and torch.equal(out[2], good[2])


def test_attention_repeats_itself_and_splits_evenly():
    """One long sequence over the whole grid, ragged neighbours, one workspace for many calls."""
    pr = Pair(pages=700, heads=2, d=64, page=128, seqs=4, width=400, seed=25)
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    lens = [40000, 130, 0, 9000]
    pr.resize([n + 3 for n in lens])
    k = torch.randn((4, 40003, 2, 64), generator=g, device=DEV).to(torch.bfloat16)
    v = torch.randn((4, 40003, 2, 64), generator=g, device=DEV).to(torch.bfloat16)
    kv.append(pr.c, 0, k, v, count=i32([n + 3 for n in lens]))
    pr.c.seq_len.copy_(i32(lens))
    q = torch.randn((4, 3, 8, 64), generator=g, device=DEV).to(torch.bfloat16)
    ws = kv.attention_workspace(q, pr.c)
    out = [kv.tree_attention(q, pr.c, 0, workspace=ws).clone() for _ in range(3)] + [kv.tree_attention(q, pr.c, 0)]
    for o in out[1:]:
        assert torch.equal(o, out[0])
    kd, vd = kv.gather(pr.c, 0, 1, None, i32([n + 3 for n in lens]), rows=40003, dtype=torch.float32)
    for b, n in enumerate(lens):
        for i in range(3):
            kk, vv = kd[0, b, :n + i + 1].double(), vd[0, b, :n + i + 1].double()
            z = torch.einsum("thd,hgd->hgt", kk, q[b, i].double().view(2, 4, 64)) / 8
            w = torch.softmax(z, -1)
            o = torch.einsum("hgt,thd->hgd", w, vv).reshape(8, 64)
            mag = torch.einsum("hgt,thd->hgd", w, vv.abs()).reshape(8, 64)
            tol = mag * (2.0 ** -11 + 2.0 ** -13 + 40000 * 2.0 ** -24) + 2.0 ** -8 * o.abs()
            assert ((out[0][b, i].double() - o).abs() <= tol).all()


# ------------------------------------------------------------------------------------- together

def test_one_decode_cycle_of_the_library():
    """Room, append, attention, LM head with verification, commit, trim: twice, as a program runs them."""
    B, N, H, G, d, V = 3, 12, 2, 4, 64, 2000
    pr = Pair(layers=2, pages=60, heads=H, d=d, page=16, seqs=B, width=12, seed=31)
    pr.grow([40, 9, 77])
    g = torch.Generator(device=DEV)
    g.manual_seed(7)
    wo = (torch.randn((V, H * G * d), generator=g, device=DEV) * 0.2).to(torch.bfloat16)
    ws = None
    for cycle in range(2):
        pr.resize([N] * B)
        parent = trees(np.random.default_rng(cycle), B, N)
        k, v = pr.rand(B, N, torch.bfloat16, loud=False), pr.rand(B, N, torch.bfloat16, loud=False)
        pr.append(B, N, k=k, v=v)
        q = torch.randn((B, N, H * G, d), generator=g, device=DEV).to(torch.bfloat16)
        ws = kv.attention_workspace(q, pr.c) if ws is None else ws
        o = torch.full(q.shape, 7.25, dtype=q.dtype, device=DEV)
        check_attention(pr, q, parent=parent, layer=1, out=o, workspace=ws)
        hidden = o.view(B * N, H * G * d)
        top = torch.topk(hidden.float() @ wo.float().T, 2).indices.cpu().numpy().reshape(B, N, 2)
        tok = np.zeros((B, N), np.int32)
        for i in range(1, N):
            tok[:, i] = top[np.arange(B), parent[:, i], 0]
        out = mars.lmhead_verify(hidden, wo, None, tok, parent, 0.9)
        path, acc = host(out["path_nodes"]), host(out["accept_len"])
        assert (acc > 0).any()
        kv.commit(pr.c, out["path_nodes"], out["accept_len"])
        pr.m.len[:], st = pr.m.commit(path, acc)
        assert (st == 0).all()
        pr.resize([0] * B)
        pr.stored()


def test_cycle_in_a_captured_graph():
    """append, attention and commit captured once and replayed on new contents."""
    B, N, H, d = 2, 6, 2, 128
    pr = Pair(pages=40, heads=H, d=d, page=16, seqs=B, width=12, seed=33)
    pr.grow([21, 50])
    pr.resize([40] * B)
    parent = trees(np.random.default_rng(5), B, N)
    k, v, q = (torch.zeros((B, N, h, d), dtype=torch.bfloat16, device=DEV) for h in (H, H, 2 * H))
    par, path, acc = i32(parent), i32(np.zeros((B, 4))), i32([0] * B)
    o = torch.zeros((B, N, 2 * H, d), dtype=torch.bfloat16, device=DEV)
    ws = kv.attention_workspace(q, pr.c)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        kv.append(pr.c, 0, k, v)
        kv.tree_attention(q, pr.c, 0, par, out=o, workspace=ws)
        kv.commit(pr.c, path, acc)
    for step in range(3):
        k.copy_(pr.rand(B, N, torch.bfloat16, loud=False))
        v.copy_(pr.rand(B, N, torch.bfloat16, loud=False))
        q.copy_(torch.randn(q.shape, device=DEV))
        path.copy_(i32([[0, 2, 5, -1], [0, 1, 3, 4]]))
        acc.copy_(i32([2, 3]))
        graph.replay()
        torch.cuda.synchronize()
        pr.m.append(0, host(k), host(v))
        want, live, _, mag, _, _ = ko.attention(pr.m, 0, host(q).astype(np.float64), parent)
        assert (np.abs(host(o) - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -10 * mag + 1e-6).all()
        pr.m.len[:], _ = pr.m.commit(host(path), host(acc))
        pr.tables()
        pr.stored()


# ------------------------------------------------------------------------------------- edges of the split

@pytest.mark.parametrize("N,group", [(1, 8), (1, 9), (4, 4), (1, 17), (8, 4), (11, 3), (1, 64), (1, 130), (32, 4), (43, 3)])
def test_attention_at_the_borders_of_the_row_tiles(N, group):
    """8, 9, 16, 17, 32, 33, 64, 128, 129 and 130 query rows per KV head: every kernel and its neighbour."""
    pr = Pair(pages=60, heads=1, d=128, page=32, seqs=3, width=16, seed=N * group)
    pr.grow([200, 31, 0])
    pr.resize([N] * 3)
    pr.append(3, N)
    q = torch.randn((3, N, group, 128), device=DEV).to(torch.bfloat16)
    check_attention(pr, q)
    check_attention(pr, q, parent=trees(np.random.default_rng(N), 3, N), count=[N, N, max(N // 2, 1)])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("N,group", [(17, 1), (6, 4), (24, 1), (5, 5), (3, 8)])
def test_attention_of_tiles_of_24_rows_and_beside_them(N, group, d):
    pr = Pair(pages=60, heads=2, d=d, page=16, seqs=3, width=20, seed=N * group)
    pr.grow([257, 15, 0])
    pr.resize([N] * 3)
    pr.append(3, N)
    q = torch.randn((3, N, 2 * group, d), device=DEV).to(torch.float16)
    check_attention(pr, q)
    check_attention(pr, q, parent=trees(np.random.default_rng(N), 3, N, absent=0.1), count=[N, N, max(N // 2, 1)])


def test_attention_of_a_tree_above_the_mask_store_with_few_rows_each():
    """Trees that only the kernel for few rows takes, in tiles of 32 rows that begin inside a node's heads."""
    pr = Pair(pages=60, heads=1, d=64, page=32, seqs=2, width=16, seed=131)
    pr.grow([100, 1])
    pr.resize([150] * 2)
    pr.append(2, 150)
    q = torch.randn((2, 150, 3, 64), device=DEV).to(torch.bfloat16)
    check_attention(pr, q, parent=trees(np.random.default_rng(5), 2, 150, absent=0.03))


def test_attention_of_a_prompt_of_many_tiles():
    """More than 32 tiles of query rows in an item list: every lane of a warp holds more than one."""
    pr = Pair(pages=60, heads=1, d=64, page=64, seqs=2, width=50, seed=132)
    pr.grow([33, 0])
    pr.resize([2300, 17])
    pr.append(2, 2300, count=[2300, 17])
    q = torch.randn((2, 2300, 4, 64), device=DEV).to(torch.bfloat16)
    check_attention(pr, q, count=[2300, 17])


def test_pools_beyond_32_bit_offsets():
    """The same calls in a small pool and in one of 5.5 GB whose only free pages are its last ones: the same
    rows, lengths and results, pages shifted."""
    L, H, d, page, few = 2, 4, 128, 16, 40
    many = 300000
    caches = []
    for n in (few, many):
        c = kv.KVCache.empty(L, n, H, d, page, 6, 16, DEV)
        if n == many:
            c.free_bits.zero_()
            c.free_bits[-1] = -1                     # 32 pages, and 8 before them
            c.free_bits[-2] = -(1 << 24)
        caches.append(c)
    assert caches[1].pages.nbytes > 1 << 32 and many % 32 == 0
    rng = np.random.default_rng(7)
    k, v = (torch.as_tensor(rng.standard_normal((3, 70, H, d)), device=DEV).to(torch.bfloat16) for _ in range(2))
    q = torch.as_tensor(rng.standard_normal((3, 70, 2 * H, d)), device=DEV).to(torch.bfloat16)
    par = i32(trees(rng, 3, 30))
    got = []
    for c in caches:
        r = []
        kv.resize(c, i32([100, 70, 75, -2, -2, -2]))
        for layer in range(L):
            kv.append(c, layer, k, v, count=i32([70, 35, 64]))
        kv.commit(c, None, i32([69, 34, 63]))
        kv.resize(c, i32([30, 30, 30, -2, -2, -2]))
        for layer in range(L):
            kv.append(c, layer, v[:, :30].contiguous(), k[:, :30].contiguous())
            r.append(kv.tree_attention(q[:, :30].contiguous(), c, layer, par))
            r.append(kv.tree_attention(q[:, :3].contiguous(), c, layer))
            r.append(kv.tree_attention(q[:, :1], c, layer))
        kv.commit(c, i32([[0, 2, 5, 9]] * 3), i32([3, 2, 0]))
        r.append(kv.fork(c, i32([0, 1]), i32([3, 5])))
        r += kv.gather(c, 0, L, None, c.seq_len.clone(), rows=80)
        kv.resize(c, i32([0, -1, 0, 16, -2, 0]))
        r += [c.seq_len.clone(), c.seq_pages.clone(), c.block_table - (c.num_pages - few) * (c.block_table >= 0),
              c.page_refs[c.num_pages - few:].clone()]
        got.append(r)
    for a, b in zip(*got):
        assert torch.equal(a, b)
    assert int(got[0][-3].sum()) > 0 and bool((caches[1].block_table.max() > many - few).item())


@pytest.mark.parametrize("N", [128, 129])
def test_attention_of_trees_at_the_border_of_the_mask_store(N):
    pr = Pair(pages=40, heads=1, d=128, page=64, seqs=2, width=8, seed=N)
    pr.grow([100, 1])
    pr.resize([N] * 2)
    pr.append(2, N)
    q = torch.randn((2, N, 2, 128), device=DEV).to(torch.float16)
    check_attention(pr, q, parent=trees(np.random.default_rng(N), 2, N, absent=0.05))


@pytest.mark.parametrize("B,N", [(300, 1), (1000, 1), (1000, 40)])
def test_attention_of_many_sequences_most_of_them_idle(B, N):
    """More sequences than threads that split the work, and blocks whose share spans many idle ones."""
    rng = np.random.default_rng(B)
    pr = Pair(pages=2 * B * (1 + N // 32), heads=1, d=64, page=16, seqs=B, width=5, seed=B)
    lens = [int(x) for x in rng.integers(0, 20, B)]
    pr.resize([n + N for n in lens], check=False)
    k = pr.rand(B, 20 + N, torch.bfloat16, loud=False)
    pr.append(B, 20 + N, count=[n + N for n in lens], k=k, v=k.flip(-1).contiguous())
    pr.m.len[:] = lens
    pr.c.seq_len.copy_(i32(lens))
    count = np.where(rng.uniform(0, 1, B) < 0.04, N, 0).astype(np.int32)
    q = torch.randn((B, N, 2, 64), device=DEV).to(torch.bfloat16)
    check_attention(pr, q, count=count)
    if N == 1:
        check_attention(pr, q)


@pytest.mark.parametrize("d,N,group", [(128, 7, 4), (64, 9, 1), (128, 60, 4), (64, 100, 2), (64, 130, 1)])
def test_attention_of_trees_padded_with_nodes_that_were_never_appended(d, N, group):
    """Behind a sequence's nodes the parents are -1 and the slots hold what they held, here NaN scales
    in every byte; inside it too, and with parents that are no tree only the root's row is there."""
    pr = Pair(pages=60, heads=2, d=d, page=32, seqs=3, width=16, seed=d + N)
    pr.c.pages.fill_(0x7f)
    pr.grow([70, 0, 33])
    pr.resize([N] * 3)
    real = [N // 2, 1, N]
    pr.append(3, N, count=real)
    parent = trees(np.random.default_rng(N), 3, N)
    for b in range(3):
        parent[b, real[b]:] = -1
    q = torch.randn((3, N, 2 * group, d), device=DEV).to(torch.bfloat16)
    check_attention(pr, q, parent=parent)
    parent[1, 1:] = N + 3
    check_attention(pr, q, parent=parent)


@pytest.mark.parametrize("N,group", [(80, 4), (33, 1)])
def test_attention_of_many_ragged_chains(N, group):
    """More sequences than warps share the split of chains of several tiles."""
    B = 70
    rng = np.random.default_rng(N)
    pr = Pair(pages=B * 11, heads=1, d=64, page=16, seqs=B, width=11, seed=N)
    lens = [int(x) for x in rng.integers(0, 90, B)]
    pr.grow(lens)
    pr.resize([N] * B)
    count = rng.integers(0, N + 1, B).astype(np.int32)
    pr.append(B, N, count=count)
    q = torch.randn((B, N, group, 64), device=DEV).to(torch.float16)
    check_attention(pr, q, count=count)
    check_attention(pr, q[:30].contiguous(), count=count[:30])


def test_attention_of_an_idle_batch_writes_nothing():
    pr = Pair(pages=10, heads=2, d=64, page=16, seqs=3, width=4, seed=40)
    pr.grow([20, 3, 0])
    for N in (1, 40):
        q = torch.randn((3, N, 4, 64), device=DEV).to(torch.bfloat16)
        check_attention(pr, q, count=[0, -5, 0])


def test_two_streams_with_workspaces_of_their_own():
    """Calls of both kernels in flight at once, on streams that nothing orders."""
    prs, qs, ws, out, streams = [], [], [], [], []
    for s in range(2):
        pr = Pair(pages=200, heads=2, d=128, page=64, seqs=4, width=60, seed=50 + s)
        pr.grow([500, 20, 130, 64])
        pr.resize([33] * 4)
        pr.append(4, 33)
        q = torch.randn((4, 33 if s else 2, 8, 128), device=DEV).to(torch.bfloat16)
        prs.append(pr), qs.append(q), ws.append(kv.attention_workspace(q, pr.c)), out.append(torch.zeros_like(q))
        streams.append(torch.cuda.Stream())
    torch.cuda.synchronize()
    for _ in range(20):
        for s in range(2):
            with torch.cuda.stream(streams[s]):
                kv.tree_attention(qs[s], prs[s].c, 0, out=out[s], workspace=ws[s])
    torch.cuda.synchronize()
    for s in range(2):
        assert torch.equal(out[s], check_attention(prs[s], qs[s]))


def test_one_workspace_for_calls_of_different_sizes():
    """The largest call's workspace serves the smaller ones, in any order."""
    pr = Pair(pages=200, heads=2, d=64, page=32, seqs=3, width=60, seed=60)
    pr.grow([900, 20, 130])
    pr.resize([64] * 3)
    pr.append(3, 64)
    qs = [torch.randn((3, N, 8, 64), device=DEV).to(torch.bfloat16) for N in (64, 1, 3, 64, 5, 1)]
    ws = kv.attention_workspace(qs[0], pr.c)
    need = max(kv.attention_workspace_bytes(3, q.shape[1], 8, 2, 64) for q in qs)
    ws = torch.zeros((need,), dtype=torch.uint8, device=DEV)
    for q in qs:
        check_attention(pr, q, workspace=ws)


def test_append_rows_off_the_32_byte_grid_and_wide_heads():
    """16-byte aligned rows that are not 32-byte aligned; more values in a row than a block has threads."""
    pr = Pair(heads=20, d=128, page=16, seqs=2, width=4, pages=12, seed=70)
    pr.resize([10, 10])
    flat = torch.randn((2 * 10 * 41 * 128 + 8,), device=DEV).to(torch.bfloat16)
    both = flat[8:].view(2, 10, 41, 128)
    assert both.data_ptr() % 32 == 16
    k, v = both[:, :, :20], both[:, :, 20:40]
    pr.append(2, 10, k=k, v=v)
    pr.m.len[:] = 10
    pr.stored()
    out = (torch.zeros((2 * 10 * 20 * 128 + 8,), dtype=torch.bfloat16, device=DEV)[8:].view(1, 2, 10, 20, 128),
           torch.zeros((1, 2, 10, 20, 128), dtype=torch.bfloat16, device=DEV))
    kv.gather(pr.c, 0, 1, i32([0, 0]), i32([10, 10]), out=out)
    for got, want in zip(out, pr.m.rows(0, 1, 0, 10)):
        assert np.array_equal(host(got)[0, 1], torch.as_tensor(want).float().to(torch.bfloat16).float().numpy())


def test_quotients_on_every_border():
    """x / (s * g) exactly between two codes, for every scale of a sixteen and many g: to the even code."""
    rng = np.random.default_rng(80)
    g = rng.uniform(0.01, 50.0, (1, 2, 64)).astype(np.float32)
    g[0, 0, :32] = np.exp2(rng.integers(-8, 8, 32))
    c = kv.KVCache.empty(1, 40, 64, 64, 16, 2, 20, DEV, scales=g)
    m = ko.Model(1, 40, 64, 64, 16, 2, 20, g)
    kv.resize(c, i32([300, 300]))
    m.resize([300, 300])
    mids = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])
    s = ko.E4M3[rng.integers(1, 127, (2, 300, 64, 4, 1))]
    x = np.tile(mids, 2) * s * np.where(rng.uniform(0, 1, (2, 300, 64, 4, 16)) < 0.5, -1, 1)
    x = (x * g[0, 0][None, None, :, None, None]).reshape(2, 300, 64, 64)
    x = np.nextafter(x.astype(np.float32), np.where(rng.uniform(0, 1, x.shape) < 0.3, np.float32(np.inf), x.astype(np.float32)))
    k = torch.as_tensor(x, device=DEV)
    kv.append(c, 0, k, k)
    m.append(0, x, x)
    for b in range(2):
        for pos in range(0, 300, 7):
            p, slot = m.at(b, pos)
            raw = host(c.pages)[0, p].reshape(64, 1, 18 * 64)[:, 0]
            code = raw[:, slot * 32:(slot + 1) * 32]
            assert np.array_equal(code & 15, m.code[0, p, slot, :, 0, 0::2]) and np.array_equal(code >> 4, m.code[0, p, slot, :, 0, 1::2])
            assert np.array_equal(raw[:, 16 * 64 + slot * 4:16 * 64 + slot * 4 + 4], m.scale[0, p, slot, :, 0])


# ------------------------------------------------------------------------------------- waits that give up

GIVE_UP = [("trees", 128, 60, 4), ("trees", 64, 33, 1), ("chain", 128, 100, 1), ("chain", 64, 90, 8)]


def give_up_case(kind, d, N, group, seed=95):
    """A batch for the kernel for many query rows: (pair, q, parent, count, call) with call(hook, workspace) ->
    (out, status).  Sequence 3 has no work."""
    rng = np.random.default_rng(seed)
    pr = Pair(pages=260, heads=3, d=d, page=64, seqs=5, width=60, seed=seed)
    pr.grow([1500, 40, 2100, 5, 900])
    pr.resize([N] * 5)
    pr.append(5, N)
    q = torch.randn((5, N, 3 * group, d), device=DEV).to(torch.bfloat16)
    parent = trees(rng, 5, N, absent=0.05) if kind == "trees" else None
    count = [N, N - 1, N, 0, N // 2]

    def call(hook, workspace):
        hooks.set("HOOK_ATTENTION_GIVE_UP", hook)
        out = torch.full(q.shape, 7.25, dtype=q.dtype, device=DEV)
        st = torch.full((5,), -7, dtype=torch.int32, device=DEV)
        kv.tree_attention(q, pr.c, 0, None if parent is None else i32(parent), count=i32(count), out=out, status=st,
                          workspace=workspace)
        torch.cuda.synchronize()
        hooks.clear("HOOK_ATTENTION_GIVE_UP")
        return out, host(st)
    return pr, q, parent, count, call


@pytest.mark.parametrize("kind,d,N,group", GIVE_UP)
def test_waits_that_give_up_are_reported(kind, d, N, group):
    """The kernel returns, every sequence with work says so, and with the workspace zeroed the next call is as ever."""
    pr, q, parent, count, call = give_up_case(kind, d, N, group)
    ws = kv.attention_workspace(q, pr.c)
    good = check_attention(pr, q, parent=parent, count=count, workspace=ws)
    out, st = call(1, ws)
    assert st.tolist() == [3, 3, 3, 0, 3] and torch.equal(out[3], good[3])
    ws.zero_()
    out, st = call(0, ws)
    assert torch.equal(out, good) and (st == 0).all()


@pytest.mark.parametrize("kind,d,N,group", GIVE_UP)
def test_rows_and_workspace_after_waits_that_gave_up(kind, d, N, group):
    """What a block that gave up owes is NaN, everything else as ever, and the workspace serves the next call."""
    pr, q, parent, count, call = give_up_case(kind, d, N, group)
    ws = kv.attention_workspace(q, pr.c)
    good, _ = call(0, ws)
    untouched = (good == 7.25).all(-1)
    missing = 0
    for first in (1, 2, 9, 20, 30, 12):
        out, st = call(first, ws)
        same, none = (out == good).all(-1), out.isnan().all(-1)
        assert bool((same | none).all()) and bool(same[untouched].all())
        missing += int(none.sum())
        out, st = call(0, ws)
        assert torch.equal(out, good) and (st == 0).all(), first
    assert missing


@pytest.mark.parametrize("d,group", [(128, 4), (64, 8)])
def test_a_sequence_with_a_block_that_gave_up_never_says_ok(d, group):
    """The block that reports on a sequence comes to it late, long after another block's waits for it ran out."""
    N, lens = 60, [60000, 60000]
    pr = Pair(pages=2000, heads=2, d=d, page=128, seqs=2, width=480, seed=96)
    pr.resize([n + N for n in lens])
    k = torch.randn((2, 60000 + N, 2, d), device=DEV).to(torch.bfloat16)
    kv.append(pr.c, 0, k, k.flip(1))
    pr.c.seq_len.copy_(i32(lens))
    q = torch.randn((2, N, 2 * group, d), device=DEV).to(torch.bfloat16)
    parent = i32(trees(np.random.default_rng(3), 2, N))
    ws = kv.attention_workspace(q, pr.c)
    st = torch.full((2,), -7, dtype=torch.int32, device=DEV)
    good = kv.tree_attention(q, pr.c, 0, parent, status=st, workspace=ws)
    assert (host(st) == 0).all()
    told = set()
    for first in [1, 20, 40, 60, 70, 74, 75, 76, 80, 90, 100, 110, 120, 130, 140, 146, 147, 148]:
        for _ in range(3):
            out = torch.full(q.shape, 7.25, dtype=q.dtype, device=DEV)
            st.fill_(-7)
            hooks.set("HOOK_ATTENTION_GIVE_UP", first)
            kv.tree_attention(q, pr.c, 0, parent, out=out, status=st, workspace=ws)
            torch.cuda.synchronize()
            hooks.clear("HOOK_ATTENTION_GIVE_UP")
            for b in range(2):
                s = int(st[b])
                told.add((b, s))
                assert s in (0, 3) and (s == 3) == bool(out[b].isnan().any()), (first, b, s)
                assert torch.equal(out[b][~out[b].isnan()], good[b][~out[b].isnan()])
    assert told == {(0, 0), (0, 3), (1, 3)}


@pytest.mark.parametrize("N", [3, 40])
def test_rows_without_a_result_are_zero_in_an_output_of_the_calls_own(N):
    """Short counts, absent nodes, no room, no tree: nothing of what the memory held before shows."""
    pr = Pair(pages=60, heads=2, d=64, page=16, seqs=4, width=8, seed=97)
    pr.grow([20, 16, 40, 5])
    pr.resize([N, 0, N, N])
    pr.append(4, N)
    q = torch.randn((4, N, 4, 64), device=DEV).to(torch.bfloat16)
    parent = trees(np.random.default_rng(1), 4, N)
    parent[2, 1] = 2                              # no tree
    parent[3, N - 1] = -1                         # absent
    count = [N - 1, N, N, N]
    par, cnt = i32(parent), i32(count)
    held = [torch.full(q.shape, 9.0, dtype=q.dtype, device=DEV) for _ in range(50)]
    places = {x.data_ptr() for x in held}
    del held                                      # memory that held nines
    out = kv.tree_attention(q, pr.c, 0, par, count=cnt)
    assert out.data_ptr() in places
    want = check_attention(pr, q, parent=parent, count=count, out=torch.zeros_like(q))
    assert torch.equal(out, want) and bool((out[1] == 0).all()) and bool((out[0, N - 1] == 0).all())


# ------------------------------------------------------------------------------------- rounding on the way out

def round_once(x, dtype):
    """64-bit values to the nearest of a type, ties to even, beyond its range to infinity."""
    bits, low, top = {torch.bfloat16: (8, -126, 3.3895313892515355e38), torch.float16: (11, -14, 65504.0),
                      torch.float32: (24, -126, 3.4028234663852886e38)}[dtype]
    e = np.maximum(np.frexp(x)[1] - 1, low)
    step = np.exp2(e - (bits - 1.0))
    y = np.rint(x / step) * step
    return np.where(np.abs(y) > top, np.copysign(np.inf, y), y)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_gather_rounds_once(dtype):
    """Every code under every scale byte, under head scales for which a product rounded to fp32 and then again is
    another number, and under the smallest and largest ones."""
    rng = np.random.default_rng(100)
    f = np.unique(np.outer(ko.E2M1, ko.E4M3))
    hard = []
    while len(hard) < 12 and dtype != torch.float32:
        g = (rng.uniform(1.0, 2.0, 20000) * np.exp2(rng.integers(-9, 9, 20000))).astype(np.float32)
        x = f[None, :] * g[:, None].astype(np.float64)
        hard += g[(round_once(round_once(x, torch.float32), dtype) != round_once(x, dtype)).any(1)].tolist()
    g = rng.uniform(1.0, 2.0, 240).astype(np.float32)
    g = np.concatenate([np.float32(hard), (g[:200] * np.float32(2.0 ** -100)) * np.exp2(rng.integers(-40, 0, 200)).astype(np.float32),
                        g[200:240] * np.float32(2.0 ** 118), np.exp2(rng.integers(-149, 128, 40)).astype(np.float32),
                        np.float32([1.401298464324817e-45, 1.1754942106924411e-38, 1.1754943508222875e-38, 3.4028234663852886e38])])
    g = np.maximum(g, np.float32(1.401298464324817e-45))
    check_gather(g, dtype)


def check_gather(g, dtype):
    """Every code under every scale byte and the head scales g, against the nearest value of the type."""
    H = len(g)
    c = kv.KVCache.empty(1, 2, H, 64, 16, 1, 2, DEV, scales=np.stack([g, g[::-1]])[None])
    kv.resize(c, i32([32]))
    page = np.zeros((2, 1152), np.uint8)           # token t, group j: scale byte 4 t + j; codes 0 .. 15 in each
    for t in range(32):
        p, s = divmod(t, 16)
        for side in range(2):
            at = 512 * side + s * 32
            page[p, at:at + 32] = np.tile(np.arange(0, 16, 2) | (np.arange(1, 16, 2) << 4), 4)
            page[p, 1024 + 64 * side + s * 4:1024 + 64 * side + s * 4 + 4] = np.minimum(np.arange(4 * t, 4 * t + 4), 126)
    c.pages.copy_(torch.as_tensor(page)[None, :, None, :].expand(1, 2, H, 1152))
    k, v = kv.gather(c, 0, 1, i32([0]), i32([32]), rows=32, dtype=dtype)
    codes = np.tile(np.arange(16), 4)[None]
    mag = ko.values(np.repeat(codes, 32, 0), np.minimum(np.arange(128).reshape(32, 4), 126), 1.0)
    for got, gs in ((k, g), (v, g[::-1])):
        true = mag[:, None, :] * gs[None, :, None].astype(np.float64)
        got, want = got[0, 0].double().cpu().numpy(), round_once(true, dtype)
        # bf16 below its normal numbers goes through fp32: off by half a step, 2^-134, and half an fp32 step more
        low = (np.abs(true) < 2.0 ** -126) & (dtype == torch.bfloat16)
        assert np.array_equal(got[~low], want[~low]) and (np.abs(got - true)[low] <= 2.0 ** -134 + 2.0 ** -149).all()


def test_gather_rounds_once_under_subnormal_scales():
    """Products of short subnormal scales that lie exactly between two bf16 values go to the even one."""
    rng = np.random.default_rng(106)
    n = np.concatenate([(1 << 13) + 32 + 64 * np.arange(100), 32 * rng.integers(1, 1 << 18, 100), rng.integers(1, 1 << 23, 100)])
    check_gather((n * 2.0 ** -149).astype(np.float32), torch.bfloat16)


# ------------------------------------------------------------------------------------- extreme rows of q

def check_huge(pr, q, parent=None):
    """Rows whose best score is ahead of the next by more than both can be off are that key's V; all rows lie
    between V's smallest and largest value.  A score is a sum of d products with fp32 accumulation, off by at most
    d * 2^-23 of sum |q||k|, and four more roundings at 2^-23 of its size; a lead of 60 beyond that leaves
    e^-60 of each other key.  P of the best key is 2^7 and rounds to fp16 by 2^-11 at most."""
    B, N, Hq, d = q.shape
    st = torch.full((B,), -7, dtype=torch.int32, device=DEV)
    out = torch.full(q.shape, 7.25, dtype=q.dtype, device=DEV)
    kv.tree_attention(q, pr.c, 0, None if parent is None else i32(parent), out=out, status=st)
    assert (host(st) == 0).all()
    got, qq = host(out).astype(np.float64), q.double().cpu().numpy()
    half, ahead = torch.finfo(q.dtype).eps / 2, 0
    for b in range(B):
        ln = int(pr.m.len[b])
        see, _, _ = ko.ancestors(None if parent is None else parent[b], N)
        k, v = pr.m.rows(0, b, 0, ln + N)
        for i in range(N):
            use = np.concatenate([np.arange(ln), ln + np.flatnonzero(see[i])])
            for h in range(Hq):
                kk, vv = k[use, h * pr.m.H // Hq], v[use, h * pr.m.H // Hq]
                z = kk @ qq[b, i, h] * d ** -0.5
                off = (d + 4) * 2.0 ** -23 * (np.abs(kk) @ np.abs(qq[b, i, h])).max() * d ** -0.5
                top = int(z.argmax())
                x, lo, hi = got[b, i, h], vv.min(0), vv.max(0)
                slack = (2.0 ** -10 + half) * np.maximum(np.abs(lo), np.abs(hi))
                assert ((x >= lo - slack) & (x <= hi + slack)).all(), (b, i, h, z[top])
                if np.delete(z, top).max(initial=-np.inf) < z[top] - 2 * off - 60:
                    ahead += 1
                    rest = len(use) * np.exp(-60.0) * np.abs(vv).max(0)     # where the best key's V is 0
                    assert (np.abs(x - vv[top]) <= (2.0 ** -10 + half) * np.abs(vv[top]) + rest).all(), (b, i, h, z[top])
    return ahead


@pytest.mark.parametrize("N", [2, 60])
@pytest.mark.parametrize("dtype,qmag,kscale", [(torch.float16, 500.0, 1.0), (torch.float16, 1.2e4, 2.0 ** 6), (torch.float16, 1.2e4, 2.0 ** 14),
                                               (torch.bfloat16, 1e12, 2.0 ** 4), (torch.bfloat16, 1e30, 2.0 ** 10),
                                               (torch.bfloat16, 1e37, 2.0 ** 30), (torch.bfloat16, 1e30, 2.0 ** -90)])
def test_attention_of_huge_scores(N, dtype, qmag, kscale):
    pr = Pair(pages=80, heads=1, d=128, page=16, seqs=3, width=20, seed=101)
    g = np.array([[[kscale], [1.0]]], np.float32)
    pr.c.scales.copy_(torch.as_tensor(g))
    pr.m.scales = g
    pr.resize([203 + N, 17 + N, N])
    k, v = ((pr.rand(3, 203 + N, torch.float32, loud=False) * s).contiguous() for s in (kscale, 1.0))
    pr.append(3, 203 + N, torch.float32, count=[203 + N, 17 + N, N], k=k, v=v)
    pr.m.len[:] = [203, 17, 0]
    pr.c.seq_len.copy_(i32(pr.m.len))
    q = (torch.randn((3, N, 4, 128), device=DEV) * qmag).to(dtype)
    assert bool(torch.isfinite(q).all())
    assert check_huge(pr, q) > 6 * N
    assert check_huge(pr, q, parent=trees(np.random.default_rng(N), 3, N)) > 6 * N


@pytest.mark.parametrize("N", [2, 60])
@pytest.mark.parametrize("kscale", [2.0 ** -120, 2.0 ** -70, 1.0])
def test_attention_of_the_largest_finite_q(N, kscale):
    """Rows of bf16 q whose largest element is 2^127 or more, over small and ordinary K."""
    pr = Pair(pages=80, heads=1, d=64, page=16, seqs=3, width=20, seed=102)
    g = np.array([[[kscale], [1.0]]], np.float32)
    pr.c.scales.copy_(torch.as_tensor(g))
    pr.m.scales = g
    pr.resize([203 + N, 17 + N, N])
    k, v = ((pr.rand(3, 203 + N, torch.float32, loud=False) * s).contiguous() for s in (kscale, 1.0))
    pr.append(3, 203 + N, torch.float32, count=[203 + N, 17 + N, N], k=k, v=v)
    pr.m.len[:] = [203, 17, 0]
    pr.c.seq_len.copy_(i32(pr.m.len))
    q = (torch.randn((3, N, 4, 64), device=DEV) * 2.0 ** 124).to(torch.bfloat16)
    q[..., 3] = torch.finfo(torch.bfloat16).max
    q[:, 1, 2] = 2.0 ** 127
    q[:, 0, 1] = -torch.finfo(torch.bfloat16).max
    assert bool(torch.isfinite(q).all())
    if kscale < 2.0 ** -100:
        check_attention(pr, q)
    else:
        assert check_huge(pr, q) > 6 * N


# ------------------------------------------------------------------------------------- damaged tables and special rows, tiles

@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind", ["trees", "chain"])
def test_page_ids_outside_the_pool_are_not_followed_by_tiles(kind, d):
    """As above for many query rows; the damaged entry also behind the 32 key tiles that are located at once."""
    N, B, H = 60, 12, 12
    rng = np.random.default_rng(d)
    pr = Pair(pages=B * 50, heads=H, d=d, page=128, seqs=B, width=50, seed=103)
    lens = [6000, 5800] + [6100] * (B - 3) + [20]
    pr.resize([n + N for n in lens])
    k = torch.randn((B, 6160, H, d), device=DEV).to(torch.bfloat16)
    kv.append(pr.c, 0, k, k.flip(1).contiguous(), count=i32([n + N for n in lens]))
    pr.c.seq_len.copy_(i32(lens))
    q = torch.randn((B, N, 4 * H, d), device=DEV).to(torch.bfloat16)
    parent = i32(trees(rng, B, N)) if kind == "trees" else None
    ws = kv.attention_workspace(q, pr.c)
    good = kv.tree_attention(q, pr.c, 0, parent, workspace=ws)
    assert torch.isfinite(good).all()
    table = pr.c.block_table.clone()
    for b, entry in ((1, 0), (1, 31), (1, 40), (1, 45), (11, 0)):
        for bad in (-1, B * 50, 1 << 30, -(1 << 31)):
            pr.c.block_table[b, entry] = bad
            st = torch.full((B,), -7, dtype=torch.int32, device=DEV)
            out = kv.tree_attention(q, pr.c, 0, parent, status=st, workspace=ws)
            assert out[b].isnan().all() and (host(st) == 0).all()
            out[b] = good[b]
            assert torch.equal(out, good)
            pr.c.block_table.copy_(table)


@pytest.mark.parametrize("kind", ["trees", "chain"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_special_rows_of_q_in_tiles(kind, dtype):
    """Rows of nothing, of one element, with a NaN or an infinity: NaN where the formula has it, for their row alone."""
    N = 60
    pr = Pair(pages=120, heads=2, d=128, page=16, seqs=3, width=40, seed=104)
    pr.grow([390, 17, 0])
    pr.resize([N] * 3)
    pr.append(3, N)
    q = torch.randn((3, N, 8, 128), device=DEV)
    q[0, 0] = 0
    q[0, 1] *= 1e-30
    q[1, 2] *= 3e-3
    q[2, 3, :, ::2] *= 1e-4
    q[0, 4] *= 40
    q[1, 5:9, 1] *= 300
    parent = trees(np.random.default_rng(1), 3, N) if kind == "trees" else None
    q = q.to(dtype)
    good = check_attention(pr, q, parent=parent).clone()
    special = [(0, 7, 0, float("nan")), (1, 20, 7, float("inf")), (2, 59, 3, -float("inf")), (0, 33, 5, float("nan")), (2, 0, 1, float("inf"))]
    for b, i, h, x in special:
        q[b, i, h, 5] = x
    out = kv.tree_attention(q, pr.c, 0, None if parent is None else i32(parent))
    for b, i, h, _ in special:
        assert out[b, i, h].isnan().all(), (b, i, h)
        out[b, i, h] = good[b, i, h]
    assert torch.equal(out, good)


def test_captured_calls_of_many_rows_share_a_workspace():
    """Two graphs with one workspace and one status tensor, replayed in turn on new lengths and rows of q."""
    N, B = 40, 3
    pr = Pair(pages=200, heads=2, d=64, page=32, seqs=B, width=40, seed=105)
    pr.grow([700, 20, 130])
    pr.resize([2 * N] * B)
    pr.append(B, 2 * N)
    qs = [torch.randn((B, n, 8, 64), device=DEV).to(torch.bfloat16) for n in (N, N // 2)]
    parents = [i32(trees(np.random.default_rng(1), B, N)), None]
    outs = [torch.full(q.shape, 7.25, dtype=q.dtype, device=DEV) for q in qs]
    ws, st, count = kv.attention_workspace(qs[0], pr.c), torch.full((B,), -7, dtype=torch.int32, device=DEV), i32([N] * B)
    graphs = []
    for q, p, o in zip(qs, parents, outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            kv.tree_attention(q, pr.c, 0, p, count=count, out=o, status=st, workspace=ws)
    for step in range(3):
        count.copy_(i32([N, 7 * step, N - step]))
        for q in qs:
            q.normal_()
        lens = [700 + step, 20, 130 + 2 * step]          # rows behind the committed ones are there
        pr.m.len[:] = lens
        pr.c.seq_len.copy_(i32(lens))
        for g, q, p, o in zip(graphs, qs, parents, outs):
            o.fill_(7.25)
            g.replay()
            torch.cuda.synchronize()
            want = check_attention(pr, q, parent=None if p is None else host(p), count=host(count))
            assert torch.equal(o, want) and (host(st) == 0).all()

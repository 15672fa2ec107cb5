"""The 4-bit KV cache without a GPU: the model's number formats against their definition, and the
refusals of every entry point, which return before any CUDA call."""
import ctypes

import numpy as np
import pytest

from oracle import kv_oracle as ko
from paper_2601_15498_b200 import kv_cache, mars

P = ctypes.c_void_p(4096)
N = None


def cache(**kw):
    c = dict(pages=4096, scales=4096, block_table=4096, seq_len=4096, seq_pages=4096, page_refs=4096, free_bits=4096,
             layers=2, num_pages=10, kv_heads=2, head_dim=128, page_size=32, seqs=4, table_width=6)
    c.update(kw)
    return ctypes.byref(kv_cache._CacheStruct(*c.values()))


@pytest.fixture(scope="module")
def lib():
    return mars.lib()


def test_tables_of_the_model():
    assert len(ko.E4M3) == 127 and ko.E4M3[-1] == 448 and ko.E4M3[1] == 2.0 ** -9 and ko.E4M3[8] == 2.0 ** -6
    assert (np.diff(ko.E4M3) > 0).all()
    # every border of E2M1 goes to the even code
    for x, code in ((0.25, 0), (0.75, 2), (1.25, 2), (1.75, 4), (2.5, 4), (3.5, 6), (5.0, 6), (7.0, 7), (1e9, 7)):
        assert ko.nearest(x, ko.E2M1) == code
    import torch
    x = torch.cat([torch.rand(4000) * 450, torch.rand(4000) * 0.02, torch.tensor(ko.E4M3, dtype=torch.float32)])
    want = x.clamp(max=448).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(ko.nearest(x.numpy(), ko.E4M3), want)


def test_model_quantises_within_half_a_step():
    rng = np.random.default_rng(0)
    x = (rng.standard_normal((50, 64)) * np.exp2(rng.integers(-4, 5, (50, 1)))).astype(np.float32)
    c, s = ko.quantise(x, 0.5)
    y = ko.values(c, s, 0.5)
    scale = np.repeat(ko.E4M3[s] * 0.5, 16, -1)
    # a scale is off by at most 2^-4 of itself (0.0625), so amax/s <= 6 * 17/16: steps of 2 up to 6, half a
    # step 1, and what saturates at 6 is off by at most 6/16 < 1
    assert (np.abs(y - x) <= scale * 1.0 * (1 + 1e-6)).all()
    z, zs = ko.quantise(np.zeros((1, 16), np.float32), 1.0)
    assert (z == 0).all() and (zs == 0).all()
    n, ns = ko.quantise(np.array([[np.nan] * 8 + [3.0] * 8], np.float32), 1.0)
    assert (ko.values(n, ns, 1.0)[0] == [0.0] * 8 + [3.0] * 8).all()


def test_cache_descriptor_is_checked(lib):
    call = lambda c: lib.mars_kv_resize(c, P, N, N)  # noqa: E731
    assert call(N) == 1
    for f in ("pages", "scales", "block_table", "seq_len", "seq_pages", "page_refs", "free_bits"):
        assert call(cache(**{f: 0})) == 1, f
        assert call(cache(**{f: 4097})) == 1, f
    assert call(cache(pages=4104)) == 1
    for f in ("layers", "num_pages", "kv_heads", "seqs", "table_width"):
        assert call(cache(**{f: 0})) == 1, f
        assert call(cache(**{f: -3})) == 1, f
    for f, bad in (("head_dim", 96), ("head_dim", 256), ("page_size", 48), ("page_size", 8), ("page_size", 256),
                   ("seqs", 8193), ("table_width", 1 << 26), ("num_pages", (1 << 30) + 1), ("kv_heads", 1025)):
        assert call(cache(**{f: bad})) == 3, (f, bad)
    assert lib.mars_kv_resize(cache(), N, N, N) == 1


def test_pool_bytes(lib):
    size = lib.mars_kv_pool_bytes
    assert size(2, 10, 3, 128, 32) == 2 * 10 * 3 * 32 * 144
    assert size(32, 100000, 8, 128, 128) == 32 * 100000 * 8 * 128 * 144          # beyond 32 bits
    for bad in ((0, 1, 1, 64, 16), (1, 0, 1, 64, 16), (1, 1, 0, 64, 16), (1, 1, 1, 80, 16), (1, 1, 1, 64, 20)):
        assert size(*bad) == 0


def test_append_refusals(lib):
    call = lib.mars_kv_append
    args = lambda **k: [k.get(n, d) for n, d in (  # noqa: E731
        ("c", cache()), ("layer", 0), ("k", P), ("kr", 256), ("kh", 128), ("v", P), ("vr", 256), ("vh", 128), ("dt", 0),
        ("B", 1), ("N", 1), ("count", N), ("status", N), ("stream", N))]
    for bad in (dict(k=N), dict(v=N), dict(B=0), dict(N=0), dict(B=5), dict(layer=2), dict(layer=-1),
                dict(k=ctypes.c_void_p(4104)), dict(kr=257), dict(vh=4)):
        assert call(*args(**bad)) == 1, bad
    for bad in (dict(dt=3), dict(dt=-1), dict(N=(1 << 24) + 1)):
        assert call(*args(**bad)) == 3, bad


def test_attention_refusals(lib):
    call = lib.mars_tree_attention
    need = lib.mars_tree_attention_workspace_bytes(2, 4, 8, 2, 128)
    assert need > 0 and need % 4 == 0
    for bad in ((0, 1, 8, 2, 128), (1, 0, 8, 2, 128), (1, 1, 7, 2, 128), (1, 1, 8, 2, 96), (1, 1, 0, 2, 64)):
        assert lib.mars_tree_attention_workspace_bytes(*bad) == 0, bad
    args = lambda **k: [k.get(n, d) for n, d in (  # noqa: E731
        ("c", cache()), ("layer", 1), ("q", P), ("qr", 1024), ("qh", 128), ("dt", 0), ("Hq", 8), ("B", 2), ("N", 4),
        ("parent", P), ("count", N), ("scale", 0.1), ("flags", 0), ("out", P), ("outr", 1024), ("outh", 128),
        ("status", N), ("ws", P), ("wb", need), ("stream", N))]
    for bad in (dict(q=N), dict(out=N), dict(B=0), dict(B=5), dict(N=0), dict(layer=2), dict(Hq=7), dict(Hq=0),
                dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(qr=1025),
                dict(qh=4), dict(outr=0), dict(outh=0), dict(q=ctypes.c_void_p(4098)), dict(outr=12)):
        assert call(*args(**bad)) == 1, bad
    for bad in (dict(dt=1), dict(dt=3), dict(N=1025), dict(flags=1), dict(flags=128)):
        assert call(*args(**bad)) == 3, bad
    for bad in (dict(ws=N), dict(wb=need - 1), dict(ws=ctypes.c_void_p(4100))):
        assert call(*args(**bad)) == 2, bad


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group", [1, 3, 4, 8])
def test_workspace_never_falls_with_the_nodes(lib, d, group):
    size = [lib.mars_tree_attention_workspace_bytes(B, n, 2 * group, 2, d) for n in range(1, 300) for B in (1, 64)]
    assert size[0::2] == size[1::2] and size[0] > 0 and (np.diff(size[0::2]) >= 0).all()


def test_commit_fork_gather_refusals(lib):
    assert lib.mars_kv_commit(cache(), P, 4, N, 2, P, N, N) == 1
    assert lib.mars_kv_commit(cache(), P, 4, P, 2, N, N, N) == 1
    assert lib.mars_kv_commit(cache(), P, 0, P, 2, P, N, N) == 1
    assert lib.mars_kv_commit(cache(), P, 4, P, 0, P, N, N) == 1
    assert lib.mars_kv_commit(cache(), P, 4, P, 5, P, N, N) == 1
    assert lib.mars_kv_fork(cache(), N, P, 1, P, N) == 1
    assert lib.mars_kv_fork(cache(), P, N, 1, P, N) == 1
    assert lib.mars_kv_fork(cache(), P, P, 1, N, N) == 1
    assert lib.mars_kv_fork(cache(), P, P, 0, P, N) == 1
    assert lib.mars_kv_fork(cache(), P, P, 8193, P, N) == 3
    g = lib.mars_kv_gather
    assert g(cache(), 0, 1, 2, N, N, 4, N, P, 0, N) == 1
    assert g(cache(), 0, 1, 2, N, N, 4, P, N, 0, N) == 1
    assert g(cache(), 1, 2, 2, N, N, 4, P, P, 0, N) == 1
    assert g(cache(), 0, 1, 5, N, N, 4, P, P, 0, N) == 1
    assert g(cache(), 0, 1, 2, N, N, 0, P, P, 0, N) == 1
    assert g(cache(), 0, 1, 2, N, N, 4, ctypes.c_void_p(4104), P, 0, N) == 1
    assert g(cache(), 0, 1, 2, N, N, 4, P, P, 7, N) == 3


def test_binding_checks_tensors():
    import torch
    t = lambda *s, dt=torch.int32: torch.zeros(s, dtype=dt)  # noqa: E731
    good = dict(pages=t(1, 4, 2, 32 * 72, dt=torch.uint8), scales=t(1, 2, 2, dt=torch.float32), block_table=t(3, 5),
                seq_len=t(3), seq_pages=t(3), page_refs=t(4), free_bits=t(1), head_dim=64, page_size=32)
    with pytest.raises(mars.MarsError, match="device memory"):
        kv_cache.KVCache(**good)
    for k, bad in (("scales", t(1, 2, 2)), ("seq_len", t(4)), ("page_refs", t(8)[::2]), ("head_dim", 128)):
        with pytest.raises(mars.MarsError, match="contiguous"):
            kv_cache.KVCache(**{**good, k: bad})
    with pytest.raises(mars.MarsError, match="one stride"):
        kv_cache._rows(t(3, 4, 2, 64, dt=torch.float32)[:, :3], 2, 64, -1, "k")
    with pytest.raises(mars.MarsError, match="must be"):
        kv_cache._rows(t(3, 4, 2, 64), 2, 64, -1, "k")
    with pytest.raises(mars.MarsError, match="int32"):
        kv_cache._i32(t(4), 3, -1, "count")
    assert kv_cache._rows(t(3, 4, 9, 64, dt=torch.float32)[:, :, 2:4], 2, 64, -1, "k")[1:] == (576, 64)


def test_tables_whose_requests_pass_32_bits_are_refused(lib):
    """mars_kv_resize adds up pages in 32 bits: at most seqs * table_width of them can be asked for."""
    for seqs, width in ((8192, 1 << 18), (32, 1 << 26), (8192, 1 << 26), (8191, 262177)):
        c = cache(seqs=seqs, table_width=width, page_size=16)
        assert seqs * width >= 1 << 31
        assert lib.mars_kv_resize(c, P, N, N) == 3, (seqs, width)
        assert lib.mars_kv_fork(c, P, P, 1, P, N) == 3, (seqs, width)
    # the largest that is taken: refused for its missing argument only
    for seqs, width in ((8192, (1 << 18) - 1), (31, 1 << 26), (1, 1 << 26)):
        assert lib.mars_kv_resize(cache(seqs=seqs, table_width=width, page_size=16), N, N, N) == 1, (seqs, width)


def test_pools_whose_bytes_pass_63_bits_are_refused(lib):
    """Sizes that are each in range, but whose product is no 63-bit count."""
    big = dict(layers=4096, num_pages=1 << 30, kv_heads=1024, head_dim=128, page_size=128)
    fits = dict(big, layers=400)
    for kw in (big, dict(big, layers=500), dict(big, head_dim=64, layers=1000)):
        assert kw["layers"] * kw["num_pages"] * kw["kv_heads"] * kw["page_size"] * kw["head_dim"] * 9 // 8 > (1 << 63) - 1
        assert lib.mars_kv_pool_bytes(*kw.values()) == 0, kw
        assert lib.mars_kv_resize(cache(**kw), N, N, N) == 3, kw
        assert lib.mars_kv_gather(cache(**kw), 0, 1, 2, N, N, 0, P, P, 0, N) == 3, kw
    want = fits["layers"] * fits["num_pages"] * fits["kv_heads"] * fits["page_size"] * 144
    assert want < 1 << 63 and lib.mars_kv_pool_bytes(*fits.values()) == want
    assert lib.mars_kv_resize(cache(**fits), N, N, N) == 1

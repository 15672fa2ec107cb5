"""Refusals of the score calls, which return before any CUDA call."""
import ctypes
import math

import numpy as np
import pytest
import torch

from paper_2601_15498_b200 import mars

P, Q, N = ctypes.c_void_p(4096), ctypes.c_void_p(8192), None
INVALID, WORKSPACE, UNSUPPORTED = 1, 2, 3


@pytest.fixture(scope="module")
def lib():
    return mars.lib()


def call(fn, defaults, **kw):
    assert set(kw) <= set(defaults)
    return fn(*{**defaults, **kw}.values())


def test_logprob_refusals(lib):
    d = dict(logits=P, ld=100, dt=mars.FP32, n=4, row_ids=N, rows=4, V=100, T=1.0, tok=P, J=2, k=3, logprob=P, entropy=N,
             stats=N, top_id=P, top_logprob=P, stream=N)
    f = lambda **k: call(lib.mars_token_logprobs, d, **k)  # noqa: E731
    for k in ("logits", "tok", "logprob", "top_id", "top_logprob"):
        assert f(**{k: N}) == INVALID, k
    for k, bad in (("ld", 99), ("n", 0), ("n", 5), ("rows", 0), ("rows", 3), ("V", 0), ("V", 101), ("J", -1), ("k", -1), ("k", 101)):
        assert f(**{k: bad}) == INVALID, (k, bad)
    for t in (0.0, -1.0, math.nan, math.inf):
        assert f(T=t) == INVALID
    assert f(logits=ctypes.c_void_p(4097)) == INVALID
    for k, bad in (("dt", 2), ("J", 1025), ("k", 33), ("T", 1e-45)):
        assert f(**{k: bad}) == UNSUPPORTED, (k, bad)
    assert f(V=1 << 30, ld=1 << 31, rows=(1 << 27) + 1, n=(1 << 27) + 1) == UNSUPPORTED


def test_gradient_refusals(lib):
    d = dict(logits=P, ld=100, dt=mars.BF16, rows=4, V=100, T=1.0, tok=P, J=2, stats=P, entropy=P, g=P, h=P, grad=Q,
             ld_grad=100, stream=N)
    f = lambda **k: call(lib.mars_token_logprobs_backward, d, **k)  # noqa: E731
    for k in ("logits", "tok", "stats", "entropy", "g", "grad"):
        assert f(**{k: N}) == INVALID, k
    for k, bad in (("ld", 99), ("ld_grad", 99), ("rows", 0), ("V", 0), ("J", 0), ("T", 0.0), ("T", math.nan)):
        assert f(**{k: bad}) == INVALID, (k, bad)
    assert f(grad=P, ld_grad=104) == INVALID                     # in place with another stride
    assert f(grad=ctypes.c_void_p(8193)) == INVALID
    for k, bad in (("dt", 2), ("J", 1025), ("T", 1e-45)):
        assert f(**{k: bad}) == UNSUPPORTED, (k, bad)
    assert f(rows=1 << 27, V=1 << 20, ld=1 << 20, ld_grad=1 << 20) == UNSUPPORTED


def test_quantise_refusals(lib):
    d = dict(x=P, ldx=100, dt=mars.BF16, rows=4, K=100, q=Q, ldq=112, scale=P, stream=N)
    f = lambda **k: call(lib.mars_quantize_rows, d, **k)  # noqa: E731
    for k in ("x", "q", "scale"):
        assert f(**{k: N}) == INVALID, k
    for k, bad in (("ldx", 99), ("ldq", 96), ("ldq", 104), ("rows", 0), ("K", 0), ("q", ctypes.c_void_p(8200)), ("x", ctypes.c_void_p(4097))):
        assert f(**{k: bad}) == INVALID, (k, bad)
    assert f(dt=mars.FP32, x=ctypes.c_void_p(4098)) == INVALID
    for k, bad in (("dt", 3), ("rows", 1 << 31)):
        assert f(**{k: bad}) == UNSUPPORTED, (k, bad)
    assert f(K=(1 << 17) + 1, ldx=1 << 18, ldq=1 << 18) == UNSUPPORTED


def test_project_refusals_and_workspace(lib):
    size = lib.mars_project_int8_workspace_bytes
    need = size(40, 1000, 512)
    assert need % 256 == 0 and need > 0
    assert size(1, 1000, 512) <= need <= size(256, 1000, 512) and size(3840, 151936, 4096) == size(256, 1000, 512)
    for bad in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (1, 1, (1 << 17) + 1), (1, (1 << 28) + 1, 1), ((1 << 24) + 1, 1, 1), (1 << 24, 1 << 28, 1)):
        assert size(*bad) == 0, bad
    d = dict(xq=P, ldx=512, xs=P, wq=P, ldw=512, ws=P, bias=N, M=40, V=1000, K=500, out=P, ldo=1000, dt=mars.BF16, flags=0,
             work=Q, bytes=need, stream=N)
    f = lambda **k: call(lib.mars_project_int8, d, **k)  # noqa: E731
    for k in ("xq", "xs", "wq", "ws", "out"):
        assert f(**{k: N}) == INVALID, k
    for k, bad in (("ldx", 496), ("ldx", 520), ("ldw", 496), ("ldw", 520), ("ldo", 999), ("M", 0), ("V", 0), ("K", 0),
                   ("xq", ctypes.c_void_p(4104)), ("wq", ctypes.c_void_p(4104)), ("out", ctypes.c_void_p(4097))):
        assert f(**{k: bad}) == INVALID, (k, bad)
    for k, bad in (("dt", 2), ("flags", 1), ("flags", 128)):
        assert f(**{k: bad}) == UNSUPPORTED, (k, bad)
    for k, bad in (("work", N), ("work", ctypes.c_void_p(8192 + 128)), ("bytes", need - 1)):
        assert f(**{k: bad}) == WORKSPACE, (k, bad)


@pytest.mark.parametrize("kind", ["numpy", "torch", "list", "uint64", "strided"])
def test_ids_beyond_32_bits_stay_outside(kind):
    ids = [0, 5, -1, 2 ** 31 - 1, 2 ** 31, 2 ** 32, 2 ** 32 + 5, 2 ** 62 + 7] + ([] if kind == "uint64" else [-2 ** 31 - 1, -2 ** 32, -2 ** 40 + 3])
    x = {"numpy": lambda: np.array(ids), "torch": lambda: torch.tensor(ids), "list": lambda: ids,
         "uint64": lambda: np.array([max(i, 0) for i in ids] + [2 ** 63 + 5], dtype=np.uint64),
         "strided": lambda: torch.tensor(ids)[:, None].expand(len(ids), 3)[:, 1]}[kind]()
    t = mars._dev_i32(x, torch.device("cpu"))
    assert t.dtype == torch.int32 and t.is_contiguous()
    for got, i in zip(t.tolist(), ids):
        want = max(i, 0) if kind == "uint64" else i
        assert got == want if -2 ** 31 <= want < 2 ** 31 else (got == 2 ** 31 - 1 if want > 0 else got == -2 ** 31)
    assert kind != "uint64" or t[-1] < 0

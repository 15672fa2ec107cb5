"""Refusals of the score calls, which return before any CUDA call."""
import ctypes
import math

import pytest

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

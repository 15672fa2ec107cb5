"""ctypes binding of the output side of libmars (mars_scores.h; argument marshalling only).

The output projection with weights in 8 bits, quantised once::

    wq, ws = scores.quantize_rows(w_vocab)
    work = scores.project_workspace(tokens, V, K, device)
    logits = scores.project_int8(*scores.quantize_rows(hidden), wq, ws, workspace=work)      # [tokens, V]

After a verification, the log probabilities, entropies and alternatives of what it emitted::

    out = mars.verify_tree(logits, tok, parent, theta=0.9)
    got = scores.emitted_logprobs(logits, out, k=5)           # [B, Dcap + 1], [B, Dcap + 1, 5]

and for a model that learns from such rows::

    logprob, entropy = scores.logprobs(logits, tok)           # differentiable by logits
    loss = -(advantage * logprob.sum(1) + 0.01 * entropy).mean()
    loss.backward()

Every call is asynchronous on the current stream of its tensors' device.
"""
from __future__ import annotations

import torch

from . import mars
from .mars import MarsError, _check, _dev_f32, _dev_i32, lib

MAX_TOKENS, MAX_TOP = 1024, 32
PROJECT_COUNTER_BYTES = 16384

_LOGIT_DTYPES = {torch.bfloat16: mars.BF16, torch.float32: mars.FP32}
_ROW_DTYPES = {torch.bfloat16: mars.BF16, torch.float32: mars.FP32, torch.float16: 2}
_I32, _F32, _I8 = torch.int32, torch.float32, torch.int8

# The calls below run once a decode step or more, so their host time counts: attributes are read once, devices
# compared by index, the stream is taken as a raw handle, outputs come from the cheapest allocating call.

def _call(fn, index: int, *args) -> None:
    """fn(*args, stream) with device `index` current; raises on a refusal."""
    stream = torch._C._cuda_getCurrentRawStream(index)
    if torch._C._cuda_getDevice() == index:
        code = fn(*args, stream)
    else:
        with torch.cuda.device(index):
            code = fn(*args, stream)
    if code:
        _check(code, fn.__name__)


def _ptr(t):
    return None if t is None else t.data_ptr()


def _logits(logits, V):
    """(dtype code, rows, row stride, V, device index)."""
    index, dtype = logits.get_device(), logits.dtype
    if index < 0 or logits.dim() != 2 or dtype not in _LOGIT_DTYPES:
        raise MarsError("logits must be [rows, >= V] of bfloat16 or float32 in device memory")
    rows, width = logits.shape
    ld, inner = logits.stride()
    if inner != 1 and width != 1:
        raise MarsError("logits must have unit inner stride")
    V = width if V is None else int(V)
    if V > width:
        raise MarsError(f"logits have {width} columns, not {V}")
    # a single row has no second one to be apart from
    return _LOGIT_DTYPES[dtype], rows, max(ld, V) if rows == 1 else ld, V, index


def _tokens(tok, rows: int, logits):
    """(int32 [rows, J] beside the logits, J) of tok [rows], [rows, J] or None."""
    if tok is None:
        return None, 0
    if type(tok) is not torch.Tensor or tok.dtype is not _I32 or tok.get_device() != logits.get_device() or not tok.is_contiguous():
        tok = _dev_i32(tok, logits.device)
    shape = tok.shape
    if len(shape) not in (1, 2) or shape[0] != rows:
        raise MarsError(f"tok must be [{rows}] or [{rows}, J], got {list(shape)}")
    return tok, 1 if len(shape) == 1 else shape[1]


def _out1(out, name: str, n: int, dtype, device, index: int):
    """out[name] of n entries, checked, or a new tensor."""
    t = None if out is None else out.get(name)
    if t is None:
        return torch.empty_strided((n,), (1,), dtype=dtype, device=device)
    return _checked(t, name, (n,), dtype, index)


def _out2(out, name: str, n: int, m: int, dtype, device, index: int):
    """The same for [n, m]."""
    t = None if out is None else out.get(name)
    if t is None:
        return torch.empty_strided((n, m), (m, 1), dtype=dtype, device=device)
    return _checked(t, name, (n, m), dtype, index)


def _checked(t, name: str, shape, dtype, index: int):
    if t.shape != shape or t.dtype is not dtype or t.get_device() != index or not t.is_contiguous():
        raise MarsError(f"{name} must be a contiguous {dtype} tensor {list(shape)} on device {index}")
    return t


def _codes(q, scale, name: str):
    """(rows, K, row stride, device index) of a pair of codes and scales."""
    index = q.get_device()
    if index < 0 or q.dim() != 2 or q.dtype is not _I8:
        raise MarsError(f"{name}: codes must be int8 [rows, K] in device memory")
    rows, K = q.shape
    ld, inner = q.stride()
    if inner != 1 and K != 1:
        raise MarsError(f"{name}: codes must have unit inner stride")
    if scale.dtype is not _F32 or scale.shape != (rows,) or not scale.is_contiguous() or scale.get_device() != index:
        raise MarsError(f"{name}: scales must be contiguous float32, one a row, beside the codes")
    # a single row has no second one to be apart from
    return rows, K, ld if rows > 1 else -(-K // 16) * 16, index


def quantize_rows(x: torch.Tensor, out=None):
    """mars_quantize_rows on the current stream: x [rows, K] (bfloat16, float16 or float32, unit inner stride) as
    (codes int8 [rows, K] in rows of a multiple of 16 bytes, scales float32 [rows]); `out` = such a pair."""
    index, dt = x.get_device(), _ROW_DTYPES.get(x.dtype)
    if index < 0 or dt is None or x.dim() != 2 or (x.stride(1) != 1 and x.shape[1] != 1):
        raise MarsError("x must be [rows, K] of bfloat16, float16 or float32 with unit inner stride in device memory")
    R, K = x.shape
    if out is None:
        ldq = -(-K // 16) * 16
        q = torch.empty_strided((R, ldq), (ldq, 1), dtype=_I8, device=x.device)
        if ldq != K:
            q = q[:, :K]
        scale = torch.empty_strided((R,), (1,), dtype=_F32, device=x.device)
    else:
        q, scale = out
        r, k, ldq, i = _codes(q, scale, "out")
        if (r, k, i) != (R, K, index):
            raise MarsError("out must have the shape and device of x")
    ldx = x.stride(0)
    _call(lib().mars_quantize_rows, index, x.data_ptr(), max(ldx, K) if R == 1 else ldx, dt, R, K, q.data_ptr(), ldq, scale.data_ptr())
    return q, scale


def project_workspace(tokens: int, V: int, K: int, device) -> torch.Tensor:
    """A workspace for project_int8 calls of up to so many tokens (V and K do not matter to its size), its counters
    zeroed; it serves any number of calls that do not overlap.  Its first int32 is the last call's status: 0, or 3
    (timeout) where a wait on the device gave up and logits are NaN."""
    need = int(lib().mars_project_int8_workspace_bytes(tokens, V, K))
    if need == 0:
        raise MarsError("unsupported sizes")
    work = torch.empty((need,), dtype=torch.uint8, device=device)
    work[:PROJECT_COUNTER_BYTES].zero_()
    return work


def project_int8(xq: torch.Tensor, x_scale: torch.Tensor, wq: torch.Tensor, w_scale: torch.Tensor, bias=None,
                 dtype=torch.bfloat16, out: torch.Tensor | None = None, workspace: torch.Tensor | None = None) -> torch.Tensor:
    """mars_project_int8 on the current stream: logits [tokens, V] of codes xq [tokens, K] and wq [V, K] with
    their scales (quantize_rows of the hidden states, and once of the weights).  `out` [tokens, >= V] (its dtype
    is used).  `workspace` comes from project_workspace and is used by these calls only; without one, a call
    allocates and clears its own.  Logits that a wait which gave up left uncomputed are NaN."""
    M, K, ldx, index = _codes(xq, x_scale, "xq")
    V, wk, ldw, wi = _codes(wq, w_scale, "wq")
    if wk != K or wi != index:
        raise MarsError("xq and wq must have the same number of columns and device")
    if bias is not None:
        bias = _checked(_dev_f32(bias, xq.device), "bias", (V,), _F32, index)
    if out is None:
        if dtype not in _LOGIT_DTYPES:
            raise MarsError("logits are bfloat16 or float32")
        out = torch.empty_strided((M, V), (V, 1), dtype=dtype, device=xq.device)
    dt, rows, ldo, width, oi = _logits(out, None)
    if rows != M or width < V or oi != index:
        raise MarsError(f"out must be [{M}, >= {V}] beside the codes")
    flags = mars.COUNTERS_ZERO
    if workspace is None:
        flags = 0
        need = int(lib().mars_project_int8_workspace_bytes(M, V, K))
        if need == 0:
            raise MarsError("unsupported sizes")
        workspace = torch.empty_strided((need,), (1,), dtype=torch.uint8, device=xq.device)
    elif workspace.get_device() != index or not workspace.is_contiguous():
        raise MarsError("workspace must be a contiguous tensor beside the codes")
    _call(lib().mars_project_int8, index, xq.data_ptr(), ldx, x_scale.data_ptr(), wq.data_ptr(), ldw, w_scale.data_ptr(),
          _ptr(bias), M, V, K, out.data_ptr(), ldo, dt, flags, workspace.data_ptr(), workspace.nbytes)
    return out


def token_logprobs(logits: torch.Tensor, tok=None, temperature: float = 1.0, k: int = 0, rows=None,
                   V: int | None = None, out: dict | None = None) -> dict:
    """mars_token_logprobs on the current stream.  logits [n, >= V] (bfloat16 or float32, unit inner stride),
    tok [rows, J], [rows] or None, `rows` int32 [rows] (logits row of each output row, -1 for none) or None
    (all).  Returns {"logprob" (shape of tok), "entropy" [rows], "stats" [rows, 2], and with k > 0 "top_id",
    "top_logprob" [rows, k]}, in the tensors of `out` where it has them."""
    dt, n, ld, V, index = _logits(logits, V)
    dev = logits.device
    R = n
    if rows is not None:
        rows = _dev_i32(rows, dev)
        R = rows.numel()
    tok, J = _tokens(tok, R, logits)
    entropy, stats = _out1(out, "entropy", R, _F32, dev, index), _out2(out, "stats", R, 2, _F32, dev, index)
    got = {"entropy": entropy, "stats": stats}
    logprob = top_id = top_logprob = None
    if tok is not None:
        logprob = (_out1(out, "logprob", R, _F32, dev, index) if tok.dim() == 1 else
                   _out2(out, "logprob", R, J, _F32, dev, index))
        got["logprob"] = logprob
    if k > 0:
        top_id, top_logprob = _out2(out, "top_id", R, k, _I32, dev, index), _out2(out, "top_logprob", R, k, _F32, dev, index)
        got["top_id"], got["top_logprob"] = top_id, top_logprob
    _call(lib().mars_token_logprobs, index, logits.data_ptr(), ld, dt, n, _ptr(rows), R, V, float(temperature), _ptr(tok), J, int(k),
          _ptr(logprob), entropy.data_ptr(), stats.data_ptr(), _ptr(top_id), _ptr(top_logprob))
    return got


def token_logprobs_backward(logits: torch.Tensor, tok, forward: dict, grad_logprob, grad_entropy=None,
                            temperature: float = 1.0, V: int | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """mars_token_logprobs_backward on the current stream: the gradient by `logits` (columns 0 .. V-1, dtype of
    the logits; a new dense [rows, V] tensor, or `out`, which may be the logits).  `forward` is what token_logprobs
    returned for these logits; grad_logprob has the shape of tok, grad_entropy [rows] or None.  Logits whose row stride
    is no multiple of 16 bytes want an `out` of the same stride (a dense one takes two to four times as long)."""
    dt, R, ld, V, index = _logits(logits, V)
    tok, J = _tokens(tok, R, logits)
    g = _dev_f32(grad_logprob, logits.device)
    h = None if grad_entropy is None else _dev_f32(grad_entropy, logits.device)
    stats, entropy = _checked(forward["stats"], "forward['stats']", (R, 2), _F32, index), forward.get("entropy")
    # (a number of weights is not enough: [J, rows] would give every row those of others; in one dimension they are row by row)
    if tok is None or (g.shape != (R, J) and g.shape != (R * J,)) or (h is not None and (h.numel() != R or entropy is None)):
        raise MarsError("grad_logprob must have the shape of tok, grad_entropy one value a row")
    if J == 0 and h is not None:         # no tokens, the entropy's gradient alone: a place without a token
        tok, g, J = torch.full((R, 1), -1, dtype=_I32, device=logits.device), torch.zeros((R, 1), dtype=_F32, device=logits.device), 1
    if entropy is not None:
        _checked(entropy, "forward['entropy']", (R,), _F32, index)
    if out is None:
        out = torch.empty_strided((R, V), (V, 1), dtype=logits.dtype, device=logits.device)
    gdt, rows, ld_grad, width, gi = _logits(out, None)
    if gdt != dt or rows != R or width < V or gi != index:
        raise MarsError("out must be [rows, >= V] of the logits' dtype beside them")
    _call(lib().mars_token_logprobs_backward, index, logits.data_ptr(), ld, dt, R, V, float(temperature), tok.data_ptr(), J,
          stats.data_ptr(), _ptr(entropy), g.data_ptr(), _ptr(h), out.data_ptr(), ld_grad)
    return out


class _Logprobs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, tok, temperature):
        got = token_logprobs(logits, tok, temperature)
        ctx.save_for_backward(logits, tok, got["stats"], got["entropy"])
        ctx.temperature = temperature
        return got["logprob"], got["entropy"]

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, grad_logprob, grad_entropy):
        logits, tok, stats, entropy = ctx.saved_tensors
        return token_logprobs_backward(logits, tok, {"stats": stats, "entropy": entropy}, grad_logprob, grad_entropy,
                                       ctx.temperature), None, None


def logprobs(logits: torch.Tensor, tok, temperature: float = 1.0):
    """(log probabilities of tok [rows, J] or [rows], entropies [rows]) of logits [rows, V], differentiable by
    the logits (once).  Rows are not picked by index here: gather those that a loss needs."""
    return _Logprobs.apply(logits, _dev_i32(tok, logits.device), float(temperature))


def emitted_logprobs(logits: torch.Tensor, verified: dict, temperature: float = 1.0, k: int = 0, V: int | None = None,
                     chain: bool = False) -> dict:
    """token_logprobs of the tokens that a verification emitted, from its logits [B*N, ld] and its result:
    out_tokens[b, i] was judged by, or drawn from, the row of node path_nodes[b, i] (with `chain`, for the
    results of the chain calls, which have no path: of row i).  Results are [B, W] (and [B, W, k]) for
    out_tokens [B, W]; places behind a sequence's out_len hold no token.  Not differentiable (see logprobs)."""
    tok = verified["out_tokens"]
    B, W = tok.shape
    if logits.shape[0] % B:
        raise MarsError("logits must hold N rows for each sequence of the verification")
    N = logits.shape[0] // B
    first = torch.arange(0, B * N, N, device=tok.device, dtype=_I32)[:, None]
    if chain:
        node = torch.arange(W, device=tok.device, dtype=_I32)[None]
        rows = torch.where(node < verified["out_len"][:, None], node + first, -1)
    else:
        path = verified["path_nodes"]
        rows = torch.where(path < 0, -1, path + first)
    got = token_logprobs(logits, tok.reshape(-1), temperature, k, rows=rows.view(-1), V=V)
    return {name: t.view(B, W, *t.shape[1:]) for name, t in got.items()}

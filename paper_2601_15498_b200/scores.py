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
from .mars import MarsError, _check, _dev_f32, _dev_i32, _dtype_code, _logits_args, lib

MAX_TOKENS, MAX_TOP = 1024, 32

_ROW_DTYPES = {torch.bfloat16: mars.BF16, torch.float32: mars.FP32, torch.float16: 2}


# The calls below run once a decode step or more, so their host time counts: devices are compared by index, the
# stream is taken as a raw handle, and the current device is only changed where it has to be.

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


def _tokens(tok, rows: int, device):
    """(int32 [rows, J] on `device`, J) of tok [rows], [rows, J] or None."""
    if tok is None:
        return None, 0
    tok = _dev_i32(tok, device)
    if tok.dim() not in (1, 2) or tok.shape[0] != rows:
        raise MarsError(f"tok must be [{rows}] or [{rows}, J], got {list(tok.shape)}")
    return tok, 1 if tok.dim() == 1 else tok.shape[1]


def _into(out, name: str, shape, dtype, device):
    """out[name], checked, or a new tensor."""
    t = None if out is None else out.get(name)
    if t is None:
        return torch.empty(shape, dtype=dtype, device=device)
    if t.shape != shape or t.dtype is not dtype or t.device != device or not t.is_contiguous():
        raise MarsError(f"out[{name!r}] must be a contiguous {dtype} tensor {list(shape)} on {device}")
    return t


def quantize_rows(x: torch.Tensor, out=None):
    """mars_quantize_rows on the current stream: x [rows, K] (bfloat16, float16 or float32, unit inner stride) as
    (codes int8 [rows, K] in rows of a multiple of 16 bytes, scales float32 [rows]); `out` = such a pair."""
    if not x.is_cuda or x.dim() != 2 or x.stride(1) != 1 or x.dtype not in _ROW_DTYPES:
        raise MarsError("x must be [rows, K] of bfloat16, float16 or float32 with unit inner stride in device memory")
    R, K = x.shape
    if out is None:
        out = (torch.empty((R, -(-K // 16) * 16), dtype=torch.int8, device=x.device)[:, :K],
               torch.empty((R,), dtype=torch.float32, device=x.device))
    q, scale = out
    _codes(q, scale, "out")
    if q.shape != x.shape or q.device != x.device:
        raise MarsError("out must have the shape and device of x")
    _call(lib().mars_quantize_rows, x.get_device(), x.data_ptr(), x.stride(0), _ROW_DTYPES[x.dtype], R, K, q.data_ptr(), q.stride(0),
          scale.data_ptr())
    return q, scale


def _codes(q, scale, name: str) -> None:
    if q.dim() != 2 or q.dtype != torch.int8 or q.stride(1) != 1 or not q.is_cuda:
        raise MarsError(f"{name}: codes must be int8 [rows, K] with unit inner stride in device memory")
    if scale.dtype != torch.float32 or tuple(scale.shape) != q.shape[:1] or not scale.is_contiguous() or scale.device != q.device:
        raise MarsError(f"{name}: scales must be contiguous float32, one a row, beside the codes")


def project_workspace(tokens: int, V: int, K: int, device) -> torch.Tensor:
    """A zeroed workspace for project_int8 calls of these sizes; it serves any number of calls that do not
    overlap."""
    need = int(lib().mars_project_int8_workspace_bytes(tokens, V, K))
    if need == 0:
        raise MarsError("unsupported sizes")
    return torch.zeros((need,), dtype=torch.uint8, device=device)


def project_int8(xq: torch.Tensor, x_scale: torch.Tensor, wq: torch.Tensor, w_scale: torch.Tensor, bias=None,
                 dtype=torch.bfloat16, out: torch.Tensor | None = None, workspace: torch.Tensor | None = None) -> torch.Tensor:
    """mars_project_int8 on the current stream: logits [tokens, V] of codes xq [tokens, K] and wq [V, K] with
    their scales (quantize_rows of the hidden states, and once of the weights).  `out` [tokens, >= V] (its dtype
    is used).  `workspace` comes from project_workspace and is used by these calls only; without one, a call
    allocates and clears its own."""
    dev = xq.device
    _codes(xq, x_scale, "xq")
    _codes(wq, w_scale, "wq")
    (M, K), V = xq.shape, wq.shape[0]
    if wq.shape[1] != K or wq.device != dev:
        raise MarsError("xq and wq must have the same number of columns and device")
    if bias is not None:
        bias = _dev_f32(bias, dev)
        if tuple(bias.shape) != (V,):
            raise MarsError(f"bias must be [{V}]")
    if out is None:
        out = torch.empty((M, V), dtype=dtype, device=dev)
    if out.dim() != 2 or out.shape[0] != M or out.shape[1] < V or out.stride(1) != 1 or out.device != dev:
        raise MarsError(f"out must be [{M}, >= {V}] with unit inner stride beside the codes")
    flags = mars.COUNTERS_ZERO
    if workspace is None:
        flags = 0
        need = int(lib().mars_project_int8_workspace_bytes(M, V, K))
        if need == 0:
            raise MarsError("unsupported sizes")
        workspace = torch.empty((need,), dtype=torch.uint8, device=dev)
    elif workspace.device != dev or not workspace.is_contiguous():
        raise MarsError("workspace must be a contiguous tensor beside the codes")
    _call(lib().mars_project_int8, xq.get_device(), xq.data_ptr(), xq.stride(0), x_scale.data_ptr(), wq.data_ptr(), wq.stride(0),
          w_scale.data_ptr(), _ptr(bias), M, V, K, out.data_ptr(), out.stride(0), _dtype_code(out), flags,
          workspace.data_ptr(), workspace.nbytes)
    return out


def token_logprobs(logits: torch.Tensor, tok=None, temperature: float = 1.0, k: int = 0, rows=None,
                   V: int | None = None, out: dict | None = None) -> dict:
    """mars_token_logprobs on the current stream.  logits [n, >= V] (bfloat16 or float32, unit inner stride),
    tok [rows, J], [rows] or None, `rows` int32 [rows] (logits row of each output row, -1 for none) or None
    (all).  Returns {"logprob" (shape of tok), "entropy" [rows], "stats" [rows, 2], and with k > 0 "top_id",
    "top_logprob" [rows, k]}, in the tensors of `out` where it has them."""
    dev = logits.device
    dt, ld, V = _logits_args(logits, logits.shape[0], V)
    n = logits.shape[0]
    rows = None if rows is None else _dev_i32(rows, dev)
    R = n if rows is None else rows.numel()
    tok, J = _tokens(tok, R, dev)
    got = {"entropy": _into(out, "entropy", (R,), torch.float32, dev), "stats": _into(out, "stats", (R, 2), torch.float32, dev)}
    if tok is not None:
        got["logprob"] = _into(out, "logprob", tok.shape, torch.float32, dev)
    if k:
        got["top_id"] = _into(out, "top_id", (R, k), torch.int32, dev)
        got["top_logprob"] = _into(out, "top_logprob", (R, k), torch.float32, dev)
    _call(lib().mars_token_logprobs, logits.get_device(), logits.data_ptr(), ld, dt, n, _ptr(rows), R, V, float(temperature), _ptr(tok), J,
          int(k), _ptr(got.get("logprob")), got["entropy"].data_ptr(), got["stats"].data_ptr(), _ptr(got.get("top_id")),
          _ptr(got.get("top_logprob")))
    return got


def token_logprobs_backward(logits: torch.Tensor, tok, forward: dict, grad_logprob, grad_entropy=None,
                            temperature: float = 1.0, V: int | None = None, out: torch.Tensor | None = None) -> torch.Tensor:
    """mars_token_logprobs_backward on the current stream: the gradient by `logits` (columns 0 .. V-1, dtype of
    the logits; a new [rows, V] tensor, or `out`, which may be the logits).  `forward` is what token_logprobs
    returned for these logits; grad_logprob has the shape of tok, grad_entropy [rows] or None."""
    dev = logits.device
    dt, ld, V = _logits_args(logits, logits.shape[0], V)
    R = logits.shape[0]
    tok, J = _tokens(tok, R, dev)
    g = _dev_f32(grad_logprob, dev)
    h = None if grad_entropy is None else _dev_f32(grad_entropy, dev)
    stats, entropy = forward["stats"], forward.get("entropy")
    if tok is None or g.numel() != R * J or (h is not None and (h.numel() != R or entropy is None)):
        raise MarsError("grad_logprob must have the shape of tok, grad_entropy one value a row")
    for t, shape in ((stats, (R, 2)), (entropy, (R,))):
        if t is not None and (tuple(t.shape) != shape or t.dtype != torch.float32 or t.device != dev or not t.is_contiguous()):
            raise MarsError("forward is not the result of token_logprobs on these logits")
    if out is None:
        out = torch.empty((R, V), dtype=logits.dtype, device=dev)
    elif out.dim() != 2 or out.shape[0] != R or out.shape[1] < V or out.stride(1) != 1 or out.dtype != logits.dtype or out.device != dev:
        raise MarsError("out must be [rows, >= V] of the logits' dtype with unit inner stride")
    _call(lib().mars_token_logprobs_backward, logits.get_device(), logits.data_ptr(), ld, dt, R, V, float(temperature), tok.data_ptr(), J,
          stats.data_ptr(), _ptr(entropy), g.data_ptr(), _ptr(h), out.data_ptr(), out.stride(0))
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
    the logits (once)."""
    return _Logprobs.apply(logits, _dev_i32(tok, logits.device), float(temperature))


def emitted_logprobs(logits: torch.Tensor, verified: dict, temperature: float = 1.0, k: int = 0, V: int | None = None) -> dict:
    """token_logprobs of the tokens that a tree verification emitted, from its logits [B*N, ld] and its result:
    out_tokens[b, i] was judged by, or drawn from, the row of node path_nodes[b, i].  Results are
    [B, Dcap + 1] (and [B, Dcap + 1, k]); places behind a sequence's out_len hold no token."""
    path, tok = verified["path_nodes"], verified["out_tokens"]
    B, W = path.shape
    if logits.shape[0] % B:
        raise MarsError("logits must hold N rows for each sequence of the verification")
    first = torch.arange(0, logits.shape[0], logits.shape[0] // B, device=path.device, dtype=torch.int32)[:, None]
    got = token_logprobs(logits, tok.reshape(-1), temperature, k, rows=torch.where(path < 0, -1, path + first).view(-1), V=V)
    return {name: t.view(B, W, *t.shape[1:]) for name, t in got.items()}

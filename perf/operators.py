"""Measured cases of the paged 4-bit KV cache: attention of draft nodes over it, and the calls that
fill it, compact it after a verification, fork it and hand its pages out.

``run`` computes them with plain torch operations, or, with ``own`` set, through the library's
entry points; ``exact`` evaluates the definitions in 64 bits.

Layout of the cache (shared by both sides): pool uint8 [layers, pages, kv_heads, page bytes]; a page
is page_size / 16 blocks of 16 tokens; a block is K codes [16, d/2], V codes [16, d/2], K scales
[16, d/16], V scales [16, d/16].  A code is a 4-bit E2M1 number (low nibble = even element), a scale
an E4M3 number for 16 neighbouring elements; value = code * scale * head scale.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ------------------------------------------------------------------------------------------ cases

def listed():
    return [
        # one sequence verifying a chain of 5 drafts (6 nodes), every head with its own K and V
        {"name": "attend_one_chain", "op": "attend", "B": 1, "N": 6, "kv_heads": 32, "group": 1, "d": 128, "page": 16,
         "dtype": "bf16", "tree": False, "len_lo": 1017, "len_hi": 1017, "ragged": False, "pick": 1},
        # a serving batch without drafts: one token a sequence, long and uneven contexts
        {"name": "attend_tokens", "op": "attend", "B": 64, "N": 1, "kv_heads": 8, "group": 4, "d": 128, "page": 64,
         "dtype": "bf16", "tree": False, "len_lo": 300, "len_hi": 32768, "ragged": False, "pick": 2},
        # the tree verification batch: 64 trees of 60 nodes over long contexts
        {"name": "attend_trees", "op": "attend", "B": 64, "N": 60, "kv_heads": 8, "group": 4, "d": 128, "page": 64,
         "dtype": "bf16", "tree": True, "len_lo": 2000, "len_hi": 12000, "ragged": True, "pick": 3},
        # chains of 7 drafts (8 nodes) for 64 sequences, fp16
        {"name": "attend_chains", "op": "attend", "B": 64, "N": 8, "kv_heads": 8, "group": 4, "d": 128, "page": 32,
         "dtype": "fp16", "tree": False, "len_lo": 777, "len_hi": 16001, "ragged": True, "pick": 4},
        # prompts read in one pass, heads of 64, nothing or little cached before them
        {"name": "attend_prompts", "op": "attend", "B": 4, "N": 2048, "kv_heads": 4, "group": 4, "d": 64, "page": 32,
         "dtype": "fp16", "tree": False, "len_lo": 0, "len_hi": 2100, "ragged": True, "pick": 5},
        # the K and V of 64 trees, slices of a fused projection, into the cache and read back
        {"name": "append_trees", "op": "append", "B": 64, "N": 60, "kv_heads": 8, "group": 4, "d": 128, "page": 64,
         "dtype": "bf16", "len_lo": 2000, "len_hi": 2500, "ragged": True, "pick": 6},
        # whole prompts into the cache
        {"name": "append_prompts", "op": "append", "B": 16, "N": 4096, "kv_heads": 8, "group": 1, "d": 128, "page": 64,
         "dtype": "bf16", "len_lo": 0, "len_hi": 100, "ragged": True, "pick": 7},
        # one sequence's tree: append, keep the accepted path
        {"name": "commit_one", "op": "commit", "B": 1, "N": 60, "layers": 1, "kv_heads": 8, "group": 1, "d": 128,
         "page": 16, "dtype": "bf16", "len_lo": 501, "len_hi": 501, "ragged": False, "pick": 8},
        # the same for 64 sequences and a few layers
        {"name": "commit_trees", "op": "commit", "B": 64, "N": 60, "layers": 4, "kv_heads": 8, "group": 1, "d": 128,
         "page": 64, "dtype": "bf16", "len_lo": 300, "len_hi": 900, "ragged": True, "pick": 9},
        # one prompt continued eight ways
        {"name": "fork_one_prompt", "op": "fork", "src": 1, "ways": 7, "layers": 32, "kv_heads": 8, "d": 128, "page": 64,
         "len_lo": 1999, "len_hi": 1999, "pick": 10},
        # 32 sequences continued two ways each
        {"name": "fork_batch", "op": "fork", "src": 32, "ways": 2, "layers": 32, "kv_heads": 8, "d": 128, "page": 64,
         "len_lo": 100, "len_hi": 9000, "pick": 11},
        # page bookkeeping of a large server between two steps: most sequences take room for the next
        # tree, some end, some wait
        {"name": "resize_server", "op": "resize", "seqs": 2048, "page": 64, "len_lo": 10, "len_hi": 16000, "N": 60,
         "pick": 12},
    ]


def _odd(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "append", "commit", "fork", "resize"])
    pick = rng.randrange(1 << 30)
    if op == "resize":
        lo, page = rng.randrange(1, 200), rng.choice([16, 32, 64, 128])
        return {"op": op, "seqs": _odd(rng, 1, 2048), "page": page, "len_lo": lo,
                "len_hi": max(lo, _odd(rng, 1, page * 250)), "N": _odd(rng, 1, 64), "pick": pick}
    if op == "fork":
        lo = rng.randrange(0, 400)
        return {"op": op, "src": _odd(rng, 1, 24), "ways": rng.randrange(1, 4), "layers": _odd(rng, 1, 24),
                "kv_heads": rng.choice([1, 2, 5, 8]), "d": rng.choice([64, 128]), "page": rng.choice([16, 32, 64, 128]),
                "len_lo": lo, "len_hi": _odd(rng, lo + 1, 4000), "pick": pick}
    c = {"op": op, "kv_heads": rng.choice([1, 2, 3, 4, 8]), "group": rng.choice([1, 2, 4, 5, 8]),
         "d": rng.choice([64, 128]), "page": rng.choice([16, 32, 64, 128]), "dtype": rng.choice(["bf16", "fp16"]),
         "ragged": rng.random() < 0.6, "pick": pick}
    if op == "append":
        c["B"] = _odd(rng, 1, 64)
        c["N"] = _odd(rng, 1, max(1, 60000 // c["B"]) if rng.random() < 0.3 else 64)
        c["len_lo"] = rng.randrange(0, 300)
        c["len_hi"] = c["len_lo"] + rng.randrange(0, 300)
    elif op == "commit":
        c["B"] = _odd(rng, 1, 64)
        c["N"] = _odd(rng, 1, 64)
        c["layers"] = rng.randrange(1, 5)
        c["group"] = 1
        c["len_lo"] = rng.randrange(0, 300)
        c["len_hi"] = c["len_lo"] + rng.randrange(0, 300)
    else:
        c["tree"] = rng.random() < 0.5
        c["N"] = _odd(rng, 1, 128) if c["tree"] else _odd(rng, 1, 2048)
        c["B"] = _odd(rng, 1, max(1, min(64, 4096 // c["N"])))
        c["len_lo"] = rng.choice([0, 0, 1, rng.randrange(0, 600)])
        c["len_hi"] = max(c["len_lo"], _odd(rng, 1, max(1, min(32768, 400000 // c["B"]))))
        while work(c)["flops"] > 2e11:
            c["N"] = max(1, c["N"] // 2)
            c["len_hi"] = max(c["len_lo"], c["len_hi"] // 2)
    return c


def _lens(case, n):
    r = np.random.RandomState(case["pick"] % (1 << 31))
    lo, hi = case["len_lo"], case["len_hi"]
    a = np.exp(r.uniform(math.log(lo + 1), math.log(hi + 1.999), n)).astype(np.int64) - 1
    a = np.clip(a, lo, hi)
    a[0] = hi
    return [int(x) for x in a]


def _counts(case, n):
    r = np.random.RandomState((case["pick"] + 1) % (1 << 31))
    N = case["N"]
    if not case.get("ragged"):
        return [N] * n
    c = r.randint(max(1, N // 2), N + 1, n)
    if n > 1:
        c[-1] = r.randint(0, N + 1)
    return [int(x) for x in c]


def _trees(case, B):
    """A tree a sequence: a node's parent is one of the few nodes before it, levels stay shallow."""
    r = np.random.RandomState((case["pick"] + 2) % (1 << 31))
    N = case["N"]
    par = np.full((B, N), -1, np.int32)
    depth = np.zeros((B, N), np.int64)
    for i in range(1, N):
        p = (r.uniform(0, 1, B) ** 1.5 * i).astype(np.int64)
        deep = np.take_along_axis(depth, p[:, None], 1)[:, 0] >= 6
        p[deep] = 0
        par[:, i] = p
        depth[:, i] = np.take_along_axis(depth, p[:, None], 1)[:, 0] + 1
    return par


def _paths(case, B, counts):
    """An accepted path a sequence (root first, node numbers rising) and its number of drafts."""
    r = np.random.RandomState((case["pick"] + 3) % (1 << 31))
    W = 9
    path = np.full((B, W), -1, np.int32)
    acc = np.full((B,), -1, np.int32)
    for b in range(B):
        n = counts[b]
        if n == 0:
            continue
        a = int(r.randint(0, min(W - 1, n - 1) + 1))
        acc[b] = a
        path[b, 0] = 0
        if a:
            path[b, 1:a + 1] = np.sort(r.choice(np.arange(1, n), a, replace=False))
    return path, acc


def _visible(case, b, n, par):
    """Visible draft nodes, summed over the n nodes of sequence b."""
    if not case["tree"]:
        return n * (n + 1) // 2
    depth = [1] * n
    for i in range(1, n):
        depth[i] = depth[par[b, i]] + 1
    return sum(depth)


def work(case):
    op = case["op"]
    if op == "resize":
        lens = _lens(case, case["seqs"])
        held = sum(-(-x // case["page"]) for x in lens)
        # every sequence's length, page count and request; the tables' touched entries; the free set
        return {"bytes": case["seqs"] * 16 + held // 8 * 8 + held // 4, "flops": 0}
    rowb = case["d"] * 9 // 16 * 2
    if op == "fork":
        lens = _lens(case, case["src"])
        tail = sum(x % case["page"] for x in lens)
        el = case["layers"] * case["kv_heads"] * rowb
        # each source's ragged rows once, each copy once, and the copies read back as 16-bit values
        return {"bytes": tail * el + case["ways"] * tail * (2 * el + case["layers"] * case["kv_heads"] * case["d"] * 4)
                + case["ways"] * sum(x // case["page"] for x in lens) * 12, "flops": 0}
    B = case["B"]
    lens, n = _lens(case, B), _counts(case, B)
    H, d = case["kv_heads"], case["d"]
    if op == "append":
        # rows in, packed rows out, packed rows in, values out
        return {"bytes": sum(n) * H * (d * 4 + 2 * rowb + d * 4), "flops": 0}
    if op == "commit":
        _, acc = _paths(case, B, n)
        kept = int((acc + 1).sum())
        L = case["layers"]
        return {"bytes": L * H * (sum(n) * (d * 4 + rowb) + kept * (2 * rowb + rowb + d * 4)), "flops": 0}
    par = _trees(case, B) if case["tree"] else None
    pairs = sum(n[b] * lens[b] + _visible(case, b, n[b], par) for b in range(B))
    kv = sum((lens[b] + n[b]) if n[b] else 0 for b in range(B)) * H * rowb
    qo = sum(n) * H * case["group"] * d * 2 * 2
    return {"bytes": kv + qo, "flops": 4 * d * pairs * H * case["group"]}


# -------------------------------------------------------------------------------- making the inputs

def _fill_pages(pool, g, scales):
    """Random K and V in every page of the pool: normal values, a few loud channels, packed."""
    L, P, H, pb = pool.shape
    d = _fill_pages.d
    page = pb * 8 // (9 * d)
    nb = page // 16
    step = max(1, (1 << 25) // (H * page * d))
    for lay in range(L):
        loud = [1 + 6 * (torch.rand((H, 1, d), generator=g, device=DEV) > 0.97).float() for _ in range(2)]
        for p0 in range(0, P, step):
            n = min(step, P - p0)
            blk = pool[lay, p0:p0 + n].view(n, H, nb, 18 * d)
            for kv in range(2):
                x = torch.randn((n, H, page, d), generator=g, device=DEV) * loud[kv]
                c, s = _quantise(x, scales[lay, kv].view(1, H, 1, 1))
                c = (c[..., 0::2] | (c[..., 1::2] << 4)).view(n, H, nb, 8 * d)
                blk[..., 8 * d * kv:8 * d * (kv + 1)] = c
                blk[..., 16 * d + d * kv:16 * d + d * (kv + 1)] = s.reshape(n, H, nb, d)


def _new_cache(case, layers, seqs, need, g, fill=True, spare=3):
    """A pool whose sequence b holds need[b] tokens' pages, in shuffled order."""
    page, H, d = case["page"], case["kv_heads"], case["d"]
    per = [-(-x // page) for x in need]
    P = sum(per) + spare
    W = max(max(per), 1) + 1
    s = {"pool": torch.empty((layers, P, H, page * d * 9 // 8), dtype=torch.uint8, device=DEV)}
    # scales calibrated once per layer, kind and head, kept at powers of two
    s["scales"] = torch.exp2(torch.randint(-3, 2, (layers, 2, H), generator=g, device=DEV).float())
    if fill:
        _fill_pages.d = d
        _fill_pages(s["pool"], g, s["scales"])
    order = torch.randperm(P, generator=g, device=DEV).to(torch.int32)
    table = torch.full((seqs, W), -1, dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(per):
        table[b, :n] = order[at:at + n]
        at += n
    refs = torch.zeros((P,), dtype=torch.int32, device=DEV)
    refs[order[:at].long()] = 1
    s["table"], s["refs"] = table, refs
    s["held"] = torch.tensor(per + [0] * (seqs - len(per)), dtype=torch.int32, device=DEV)
    s["free"] = _pack_bits(refs == 0)
    return s


def _pack_bits(free):
    n = free.numel()
    w = torch.zeros(((n + 31) // 32 * 32,), dtype=torch.int64, device=free.device)
    w[:n] = free.long()
    w = (w.view(-1, 32) << torch.arange(32, device=free.device)).sum(1)
    return torch.where(w >= 1 << 31, w - (1 << 32), w).to(torch.int32)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _cache(s, case):
    """The framework's handle on the state's tensors."""
    from paper_2601_15498_b200 import kv_cache
    return kv_cache.KVCache(pages=s["pool"], block_table=s["table"], seq_len=s["len"], seq_pages=s["held"],
                            page_refs=s["refs"], free_bits=s["free"], scales=s["scales"], head_dim=case["d"],
                            page_size=case["page"])


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed) * 1000003 + case["pick"] % 1000003)
    op = case["op"]
    if op == "resize":
        return _prepare_resize(case, g)
    if op == "fork":
        return _prepare_fork(case, g)
    B, N, H, d = case["B"], case["N"], case["kv_heads"], case["d"]
    lens, counts = _lens(case, B), _counts(case, B)
    dt = DTYPES[case["dtype"]]
    layers = case.get("layers", 1)
    s = _new_cache(case, layers, B, [lens[b] + N for b in range(B)], g, fill=op == "attend")
    if op != "attend":
        s["pool"].zero_()
    s["case"], s["lens"], s["counts"] = case, lens, counts
    s["len"], s["count"] = _i32(lens), _i32(counts)
    Hq = H * case["group"]
    # q, k and v as slices of one fused projection's output
    s["qkv"] = [torch.randn((B, N, Hq + 2 * H, d), generator=g, device=DEV).to(dt) for _ in range(layers)]
    if op == "attend":
        s["q"] = s["qkv"][0][:, :, :Hq]
        s["out"] = torch.zeros((B, N, Hq, d), dtype=dt, device=DEV)
        s["parent_host"] = _trees(case, B) if case["tree"] else None
        s["parent"] = torch.as_tensor(s["parent_host"], device=DEV) if case["tree"] else None
        s["mask"] = _ancestors(s["parent"], N)
    else:
        s["k"] = [x[:, :, Hq:Hq + H] for x in s["qkv"]]
        s["v"] = [x[:, :, Hq + H:] for x in s["qkv"]]
        for lay in range(layers):
            s["v"][lay].mul_(torch.exp2(torch.randint(-6, 7, (B, N, 1, 1), generator=g, device=DEV).float()).to(dt))
        rows = N
        if op == "commit":
            path, acc = _paths(case, B, counts)
            s["path"], s["acc"] = torch.as_tensor(path, device=DEV), torch.as_tensor(acc, device=DEV)
            s["path_host"], s["acc_host"] = path, acc
            s["kept"] = _i32([int(x) + 1 for x in acc])
            s["new_len"] = torch.zeros_like(s["len"])
            rows = path.shape[1]
        s["got"] = [torch.zeros((layers, B, rows, H, d), dtype=dt, device=DEV) for _ in range(2)]
    if own:
        from paper_2601_15498_b200 import kv_cache
        s["cache"] = _cache(s, case)
        if op == "attend":
            s["work"] = kv_cache.attention_workspace(s["q"], s["cache"])
    return s


def _ancestors(parent, N):
    """Who sees whom among the draft nodes, as a program that keeps a tree mask would hold it."""
    if parent is None:
        return torch.ones((1, N, N), dtype=torch.bool, device=DEV).tril()
    B = parent.shape[0]
    m = torch.eye(N, dtype=torch.bool, device=DEV).repeat(B, 1, 1)
    rows = torch.arange(B, device=DEV)
    for i in range(1, N):
        m[:, i] |= m[rows, parent[:, i].long()]
    return m


def _prepare_fork(case, g):
    S, ways = case["src"], case["ways"]
    lens = _lens(case, S)
    page = case["page"]
    s = _new_cache(case, case["layers"], S * (1 + ways), lens, g, spare=S * ways + 5)
    s["case"], s["lens"] = case, lens
    s["len"] = _i32(lens + [0] * (S * ways))
    src = [i for i in range(S) for _ in range(ways)]
    dst = [S + i for i in range(S * ways)]
    s["src"], s["dst"] = _i32(src), _i32(dst)
    # where the copied rows begin, for reading them back
    full = [lens[i] // page * page for i in src]
    s["start"] = _i32([0] * S + full)
    s["count"] = _i32([0] * S + [lens[i] - f for i, f in zip(src, full)])
    s["starts"], s["counts"] = [0] * S + full, [0] * S + [lens[i] - f for i, f in zip(src, full)]
    s["srcs"] = src
    s["got"] = [torch.zeros((case["layers"], S * (1 + ways), page, case["kv_heads"], case["d"]),
                            dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    _keep_meta(s)
    if own:
        s["cache"] = _cache(s, case)
    return s


def _prepare_resize(case, g):
    n = case["seqs"]
    c = {"page": case["page"], "kv_heads": 1, "d": 64}
    r = np.random.RandomState((case["pick"] + 4) % (1 << 31))
    lens = _lens(case, n)
    kind = r.uniform(0, 1, n)
    extra = [-1 if k < 0.1 else -2 if k < 0.2 else 0 if k < 0.25 else case["N"] for k in kind]
    s = _new_cache(c, 1, n, lens, g, fill=False, spare=n * (case["N"] // case["page"] + 1) // 2 + 1)
    wide = torch.full((n, s["table"].shape[1] + case["N"] // case["page"] + 1), -1, dtype=torch.int32, device=DEV)
    wide[:, :s["table"].shape[1]] = s["table"]
    s["table"] = wide
    s["case"], s["len"], s["extra"] = dict(c, op="resize"), _i32(lens), _i32(extra)
    s["status"] = torch.zeros((n,), dtype=torch.int32, device=DEV)
    _keep_meta(s)
    if own:
        s["cache"] = _cache(s, c)
    return s


def _keep_meta(s):
    """One buffer holds the tables, and a snapshot of it that a pass starts from."""
    names = ("table", "refs", "held", "free", "len")
    flat = torch.cat([s[k].reshape(-1) for k in names])
    at = 0
    for k in names:
        n, shape = s[k].numel(), s[k].shape
        s[k] = flat[at:at + n].view(shape)
        at += n
    s["meta"], s["meta0"] = flat, flat.clone()


# ------------------------------------------------------------------------------------- plain forms

def _e4m3(x):
    return x.clamp(max=448.0).to(torch.float8_e4m3fn)


def _quantise(x, g):
    """Codes (uint8 0..15) and scale bytes of rows x [..., d]; g broadcasts over the last axis."""
    x = torch.nan_to_num(x.float(), nan=0.0, posinf=math.inf, neginf=-math.inf)
    y = x.unflatten(-1, (-1, 16))
    a = y.abs().amax(-1)
    s8 = _e4m3(a / 6.0 / g)
    sg = (s8.float() * g).unsqueeze(-1)
    t = torch.where(sg > 0, y.abs() / sg, torch.zeros_like(y))
    c = (t > 0.25).to(torch.uint8)
    for edge, strict in ((0.75, 0), (1.25, 1), (1.75, 0), (2.5, 1), (3.5, 0), (5.0, 1)):
        c += (t > edge) if strict else (t >= edge)
    c |= (y < 0).to(torch.uint8) << 3
    return c.flatten(-2), s8.view(torch.uint8)


def _split(pages, d):
    """Codes and scales of pages [..., page bytes] as tokens: codes uint8 [..., page, d], scales fp32."""
    blk = pages.unflatten(-1, (-1, 18 * d))
    out = []
    for kv in range(2):
        c = blk[..., 8 * d * kv:8 * d * (kv + 1)].unflatten(-1, (16, d // 2))
        c = torch.stack((c & 15, c >> 4), -1).flatten(-2)
        s = blk[..., 16 * d + d * kv:16 * d + d * (kv + 1)].contiguous().view(torch.float8_e4m3fn).float()
        out += [c.flatten(-3, -2), s.unflatten(-1, (16, d // 16)).flatten(-3, -2)]
    return out


def _values(pages, d, scales):
    """K and V in fp32 [pages, H, page, d] of pages [pages, H, page bytes]; scales [2, H]."""
    lut = torch.tensor([*E2M1, *[-x for x in E2M1]], device=pages.device)
    kc, ks, vc, vs = _split(pages, d)
    out = []
    for c, sc, g in ((kc, ks, scales[0]), (vc, vs, scales[1])):
        x = lut[c.long()].unflatten(-1, (-1, 16)) * sc.unsqueeze(-1)
        out.append(x.flatten(-2) * g.view(1, -1, 1, 1))
    return out


def _rows(s, layer, b, first, n):
    """K and V rows first .. first+n-1 of sequence b in fp32, [n, H, d]."""
    case = s["case"]
    page, d = case["page"], case["d"]
    p0, p1 = first // page, -(-(first + n) // page)
    ids = s["table"][b, p0:p1].long()
    out = []
    for x in _values(s["pool"][layer, ids], d, s["scales"][layer]):
        x = x.permute(0, 2, 1, 3).reshape(-1, case["kv_heads"], d)
        out.append(x[first - p0 * page:first - p0 * page + n])
    return out


def _plain_attend(s):
    case = s["case"]
    H, d, G = case["kv_heads"], case["d"], case["group"]
    for b, (ln, n) in enumerate(zip(s["lens"], s["counts"])):
        if n == 0:
            continue
        k, v = _rows(s, 0, b, 0, ln + n)
        q = s["q"][b, :n].float().view(n, H, G, d).permute(1, 2, 0, 3).reshape(H, G * n, d)
        sc = torch.bmm(q, k.permute(1, 2, 0)) * (1.0 / math.sqrt(d))
        sc = sc.view(H, G, n, ln + n)
        m = s["mask"][b if s["mask"].shape[0] > 1 else 0, :n, :n]
        sc[..., ln:].masked_fill_(~m, -math.inf)
        p = torch.exp(sc - sc.amax(-1, keepdim=True))
        o = torch.bmm(p.view(H, G * n, ln + n), v.permute(1, 0, 2)) / p.sum(-1).view(H, G * n, 1)
        s["out"][b, :n] = o.view(H, G, n, d).permute(2, 0, 1, 3).reshape(n, H * G, d).to(s["out"].dtype)
    return s["out"]


def _plain_append(s, layer):
    case = s["case"]
    page, d, H = case["page"], case["d"], case["kv_heads"]
    pool = s["pool"][layer]
    blk = pool.view(pool.shape[0], H, page // 16, 18 * d)
    B, N = s["k"][layer].shape[:2]
    i = torch.arange(N, device=DEV)
    live = i < s["count"].view(B, 1)
    b, i = live.nonzero(as_tuple=True)
    pos = s["len"].long()[b] + i
    pid = s["table"][b, pos // page].long()
    sub, slot = (pos % page) // 16, pos % 16
    for kv, x in enumerate((s["k"][layer], s["v"][layer])):
        c, sc = _quantise(x[b, i], s["scales"][layer, kv].view(H, 1))
        c = c[..., 0::2] | (c[..., 1::2] << 4)
        codes = blk[..., 8 * d * kv:8 * d * (kv + 1)].unflatten(-1, (16, d // 2))
        codes[pid, :, sub, slot] = c
        by = blk[..., 16 * d + d * kv:16 * d + d * (kv + 1)].unflatten(-1, (16, d // 16))
        by[pid, :, sub, slot] = sc


def _plain_gather(s, starts, counts):
    case = s["case"]
    for layer in range(s["pool"].shape[0]):
        for b, (st, n) in enumerate(zip(starts, counts)):
            if n == 0:
                continue
            for out, x in zip(s["got"], _rows(s, layer, b, st, n)):
                out[layer, b, :n] = x.to(out.dtype)
    return s["got"]


def _move(s, b, src, dst):
    """Rows at positions src of sequence b to positions dst, in every layer."""
    case = s["case"]
    page, d = case["page"], case["d"]
    pool = s["pool"]
    blk = pool.view(*pool.shape[:3], page // 16, 18 * d)
    t = s["table"][b].long()
    at = [(t[p // page], (p % page) // 16, p % 16) for p in (src, dst)]
    for lo, hi in ((0, 8 * d), (8 * d, 16 * d), (16 * d, 17 * d), (17 * d, 18 * d)):
        part = blk[..., lo:hi].unflatten(-1, (16, -1))
        part[:, at[1][0], :, at[1][1], at[1][2]] = part[:, at[0][0], :, at[0][1], at[0][2]]


def _plain_commit(s):
    for b, a in enumerate(s["acc_host"]):
        if a > 0:
            src = s["len"][b].long() + s["path"][b, 1:int(a) + 1].long()
            dst = s["len"][b].long() + torch.arange(1, int(a) + 1, device=DEV)
            _move(s, b, src, dst)
    torch.add(s["len"], s["acc"] + 1, out=s["new_len"])
    return s["new_len"]


def _plain_take(s, need):
    """The lowest free pages for need[r] pages of each request in order: first place of each request
    in the list of free pages, and who is served."""
    free = ((s["free"].view(-1, 1) >> torch.arange(32, dtype=torch.int32, device=DEV)) & 1).view(-1)[:s["refs"].numel()]
    pages = free.nonzero()[:, 0]
    upto = need.cumsum(0)
    return pages, upto - need, upto <= pages.numel()


def _plain_fork(s):
    case = s["case"]
    page = case["page"]
    src, dst = s["src"].long(), s["dst"].long()
    ln = s["len"][src]
    full, tail = ln // page, (ln % page > 0).to(torch.int32)
    pages, first, _ = _plain_take(s, tail.long())
    W = s["table"].shape[1]
    col = torch.arange(W, device=DEV)
    shared = torch.where(col < full.view(-1, 1), s["table"][src], -1)
    new = pages[first.clamp(max=pages.numel() - 1)].to(torch.int32)
    last = (col == full.view(-1, 1)) & (tail.view(-1, 1) > 0)
    old = s["table"][dst]
    row = torch.where(last, new.view(-1, 1), torch.where(shared >= 0, shared, old))
    ids = shared[shared >= 0].long()
    s["refs"].index_add_(0, ids, torch.ones_like(ids, dtype=torch.int32))
    got = tail > 0
    s["refs"][new[got].long()] = 1
    s["free"].copy_(_pack_bits(s["refs"] == 0))
    from_page = s["table"][src, full.long().clamp(max=W - 1)].long()
    s["table"][dst] = row
    s["held"][dst] = full + tail
    s["len"][dst] = ln
    d, H = case["d"], case["kv_heads"]
    pool = s["pool"]
    for k, (a, n) in enumerate(zip(s["srcs"], s["counts"][case["src"]:])):
        if n:
            cols = pool.view(*pool.shape[:3], page // 16, 18 * d)
            to, fr = new[k].long(), from_page[k]
            for lo, hi in ((0, 8 * d), (8 * d, 16 * d), (16 * d, 17 * d), (17 * d, 18 * d)):
                part = cols[..., lo:hi].unflatten(-1, (16, -1))
                for blk in range(-(-n // 16)):
                    m = min(16, n - 16 * blk)
                    part[:, to, :, blk, :m] = part[:, fr, :, blk, :m]


def _plain_resize(s):
    page = s["case"]["page"]
    ex, ln, held = s["extra"], s["len"], s["held"]
    want = torch.where(ex == -1, 0, torch.where(ex == -2, held, (ln + ex.clamp(min=0) + page - 1) // page))
    W = s["table"].shape[1]
    col = torch.arange(W, device=DEV)
    drop = (col < held.view(-1, 1)) & (col >= want.view(-1, 1))
    ids = s["table"][drop].long()
    s["refs"].index_add_(0, ids, -torch.ones_like(ids, dtype=torch.int32))
    s["free"].copy_(_pack_bits(s["refs"] == 0))
    need = (want - held).clamp(min=0).long()
    pages, first, ok = _plain_take(s, need)
    ok = ok | (need == 0)
    take = (col >= held.view(-1, 1)) & (col < want.view(-1, 1)) & ok.view(-1, 1)
    place = (first.view(-1, 1) + col - held.view(-1, 1))[take]
    s["table"].masked_fill_(drop, -1)
    s["table"][take] = pages[place].to(torch.int32)
    s["refs"][pages[place]] = 1
    s["free"].copy_(_pack_bits(s["refs"] == 0))
    s["status"].copy_(torch.where(ok, 0, 7))
    held.copy_(torch.where(ok, want, held))
    ln.masked_fill_(ex == -1, 0)


# ---------------------------------------------------------------------------------------- one pass

def _meta(s):
    return {k: s[k] for k in ("table", "refs", "held", "free", "len")}


def run(s):
    op = s["case"]["op"]
    if own:
        return _run_own(s, op)
    if op == "attend":
        return _plain_attend(s)
    if op == "append":
        _plain_append(s, 0)
        return _plain_gather(s, s["lens"], s["counts"])
    if op == "commit":
        for layer in range(len(s["k"])):
            _plain_append(s, layer)
        return [_plain_commit(s), _plain_gather(s, s["lens"], [int(a) + 1 for a in s["acc_host"]])]
    s["meta"].copy_(s["meta0"])
    if op == "fork":
        _plain_fork(s)
        return [_meta(s), _plain_gather(s, s["starts"], s["counts"])]
    _plain_resize(s)
    return [_meta(s), s["status"]]


def _run_own(s, op):
    from paper_2601_15498_b200 import kv_cache as kv
    c = s["cache"]
    if op == "attend":
        return kv.tree_attention(s["q"], c, 0, s["parent"], count=s["count"], out=s["out"], workspace=s["work"])
    if op == "append":
        kv.append(c, 0, s["k"][0], s["v"][0], count=s["count"])
        return list(kv.gather(c, 0, 1, c.seq_len, s["count"], out=s["got"]))
    if op == "commit":
        for layer, (k, v) in enumerate(zip(s["k"], s["v"])):
            kv.append(c, layer, k, v, count=s["count"])
        kv.commit(c, s["path"], s["acc"], new_len=s["new_len"])
        return [s["new_len"], list(kv.gather(c, 0, c.layers, c.seq_len, s["kept"], out=s["got"]))]
    s["meta"].copy_(s["meta0"])
    if op == "fork":
        kv.fork(c, s["src"], s["dst"])
        return [_meta(s), list(kv.gather(c, 0, c.layers, s["start"], s["count"], out=s["got"]))]
    kv.resize(c, s["extra"], status=s["status"])
    return [_meta(s), s["status"]]


# ---------------------------------------------------------------------------- definitions in 64 bits

def _decode64(nibble):
    """E2M1 by its fields: sign, two exponent bits (bias 1), one mantissa bit."""
    n = nibble.to(torch.int64)
    e, m = (n >> 1) & 3, (n & 1).double()
    mag = torch.where(e == 0, m * 0.5, (1 + m * 0.5) * torch.exp2((e - 1).double()))
    return torch.where(n >= 8, -mag, mag)


def _scale64(byte):
    """E4M3 (no sign in use) by its fields, bias 7."""
    n = byte.to(torch.int64)
    e, m = (n >> 3) & 15, (n & 7).double()
    return torch.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * torch.exp2((e - 7).double()))


def _token64(s, layer, b, h, pos):
    """K and V of one head at positions pos in 64 bits, [len(pos), d]."""
    case = s["case"]
    page, d = case["page"], case["d"]
    pid = s["table"][b].long()[pos // page]
    raw = s["pool"][layer, pid, h]                                  # one page a position
    off = (pos % page) // 16 * (18 * d)
    slot = pos % 16
    res = []
    for kv in range(2):
        ci = (off + 8 * d * kv + slot * (d // 2)).view(-1, 1) + torch.arange(d // 2, device=DEV)
        si = (off + 16 * d + d * kv + slot * (d // 16)).view(-1, 1) + torch.arange(d // 16, device=DEV)
        byte = raw.gather(1, ci)
        x = torch.empty((pos.numel(), d), dtype=torch.float64, device=DEV)
        x[:, 0::2], x[:, 1::2] = _decode64(byte & 15), _decode64(byte >> 4)
        x *= _scale64(raw.gather(1, si)).repeat_interleave(16, 1)
        res.append(x * s["scales"][layer, kv, h].double())
    return res


def _round_to(x, values):
    """Nearest of `values` (ascending, in 64 bits); ties to the even place in the list."""
    v = torch.tensor(values, dtype=torch.float64, device=x.device)
    hi = torch.searchsorted(v, x.clamp(max=values[-1]).contiguous()).clamp(max=len(values) - 1)
    lo = (hi - 1).clamp(min=0)
    up, down = v[hi] - x, x - v[lo]
    pick = torch.where(up < down, hi, torch.where(down < up, lo, torch.where(hi % 2 == 0, hi, lo)))
    return v[pick]


def _stored64(x, g):
    """What rows x [..., d] become in the cache; g broadcasts over the last axis."""
    y = x.double().unflatten(-1, (-1, 16))
    a = y.abs().amax(-1, keepdim=True)
    table = [m * 2.0 ** -9 for m in range(8)] + [(1 + m / 8) * 2.0 ** (e - 7) for e in range(1, 16) for m in range(8)][:-1]
    s = _round_to(a / 6 / g.double().unsqueeze(-1), table) * g.double().unsqueeze(-1)
    t = torch.where(s > 0, y.abs() / s, torch.zeros_like(y))
    return (torch.sign(y) * _round_to(t, list(E2M1)) * s).flatten(-2)


def exact(case, seed):
    op = case["op"]
    if op == "resize":
        return None
    s = prepare(case, seed)
    H, d = case["kv_heads"], case["d"]
    if op == "fork":
        got = [torch.zeros(x.shape, dtype=torch.float64, device=DEV) for x in s["got"]]
        S = case["src"]
        for k, a in enumerate(s["srcs"]):
            n, st = s["counts"][S + k], s["starts"][S + k]
            if n:
                pos = st + torch.arange(n, device=DEV)
                for layer in range(case["layers"]):
                    for h in range(H):
                        for out, x in zip(got, _token64(s, layer, a, h, pos)):
                            out[layer, S + k, :n, h] = x
        return [{k: None for k in ("table", "refs", "held", "free", "len")}, got]
    if op == "attend":
        out = torch.zeros(s["out"].shape, dtype=torch.float64, device=DEV)
        G = case["group"]
        for b, (ln, n) in enumerate(zip(s["lens"], s["counts"])):
            if n == 0:
                continue
            see = torch.ones((n, ln + n), dtype=torch.bool, device=DEV)
            if case["tree"]:
                par = s["parent_host"][b]
                anc = np.zeros((n, n), bool)
                for i in range(n):
                    j = i
                    while j >= 0:
                        anc[i, j] = True
                        j = par[j]
                see[:, ln:] = torch.as_tensor(anc, device=DEV)
            else:
                see[:, ln:] = torch.arange(n, device=DEV).view(-1, 1) >= torch.arange(n, device=DEV)
            for h in range(H):
                k, v = _token64(s, 0, b, h, torch.arange(ln + n, device=DEV))
                for j in range(h * G, h * G + G):
                    z = s["q"][b, :n, j].double() @ k.T / math.sqrt(d)
                    z.masked_fill_(~see, -math.inf)
                    out[b, :n, j] = torch.softmax(z, -1) @ v
        return out
    B, rows = s["got"][0].shape[1:3]
    got = [torch.zeros(x.shape, dtype=torch.float64, device=DEV) for x in s["got"]]
    for layer in range(len(s["k"])):
        for kv, x in enumerate((s["k"][layer], s["v"][layer])):
            y = _stored64(x, s["scales"][layer, kv].view(1, 1, H, 1))
            for b in range(B):
                if op == "append":
                    got[kv][layer, b, :s["counts"][b]] = y[b, :s["counts"][b]]
                else:
                    a = int(s["acc_host"][b])
                    if a >= 0:
                        got[kv][layer, b, :a + 1] = y[b, torch.as_tensor(s["path_host"][b, :a + 1], device=DEV).long()]
    return got if op == "append" else [None, got]

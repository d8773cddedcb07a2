"""The decode side's operators on a paged KV cache, as cases that can be timed and compared.

Three kinds of call that a decode worker makes on the cache that it has received:

``attend``   attention of one new token per request over one layer of the paged cache: grouped
             heads with separate K and V, or the latent rows of multi-head latent attention; all
             tokens, or a sliding window with a few first tokens that stay visible.
``turn``     one turn of the scheduler: finished requests free their pages, some rows fork others
             (beams, samples of one prompt), every live request is extended by its new tokens.
``compact``  the pages in use move to the lowest page ids, the tables follow.
``copy``     a list of pages is copied to other pages, in all layers.

``run`` computes them in their plain form, in elementary torch operations, or, where ``own`` is
true, by the library's entry points.
"""
import math

import numpy as np
import torch

own = False

_TORCH = {"bf16": torch.bfloat16, "fp16": torch.float16, "e4m3": torch.float8_e4m3fn}


# ---------------------------------------------------------------------------------- the cases

def _attend(name, **kw):
    case = dict(name=name, kind="attend", R=4, lo=1, hi=256, H=8, G=8, D=128, Dv=0, P=16, type="bf16", io="bf16",
                window=0, sinks=0, style="page", empty=0)
    case.update(kw)
    return case


def _pages(name, kind, **kw):
    case = dict(name=name, kind=kind, R=4, lo=1, hi=256, L=2, F=2, H=8, D=128, P=16, style="page", free=1, forks=1, new=1, n=3)
    case.update(kw)
    return case


def listed():
    return [
        # the tiny grouped-head shape: four short requests, a call that is all latency
        _attend("gqa_short", R=4, lo=17, hi=255),
        # the 8B-shaped layer: sixteen ragged requests of a serving batch, four query heads a group
        _attend("gqa_ragged", R=16, lo=512, hi=4096, G=4),
        # one user with a very long prompt on the 70B-shaped layer, cache in 8 bits, an odd length
        _attend("gqa_long_8bit", R=1, lo=131071, hi=131071, type="e4m3"),
        # a windowed layer of the model with 8 x 64 heads and a 128-token window, four first tokens kept
        _attend("window_short", R=2, lo=100, hi=400, D=64, window=128, sinks=4, type="fp16", io="fp16"),
        # the same layer under a full batch, and a pool with the heads split inside the page
        _attend("window_batch", R=128, lo=1, hi=8000, D=64, window=128, sinks=4, type="fp16", io="fp16", style="head"),
        # latent rows on one of eight ranks that share the heads: 16 heads, a small batch
        _attend("latent_16_heads", R=6, lo=200, hi=1500, H=1, G=16, D=576, Dv=512, P=64),
        # latent rows with all 128 heads, the ragged serving batch
        _attend("latent_batch", R=32, lo=1024, hi=8192, H=1, G=128, D=576, Dv=512, P=64),
        # the scheduler's turn on a handful of requests
        _pages("turn_short", "turn", R=6, lo=17, hi=255, free=2, forks=2),
        # the turn of a serving batch: a dozen requests end, a dozen beams fork, all grow
        _pages("turn_batch", "turn", R=64, lo=100, hi=600, L=8, free=12, forks=12, new=2),
        # a small pool with holes
        _pages("compact_short", "compact", R=4, lo=17, hi=255, free=1),
        # a pool half of whose requests have ended, compacted before it is handed over in one piece
        _pages("compact_batch", "compact", R=32, lo=100, hi=900, L=8, free=16),
        # pages of latent rows copied within the pool: a shared prompt made private
        _pages("copy_latent", "copy", L=8, F=1, H=1, D=576, P=64, n=255),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "window", "latent", "latent", "turn", "turn", "compact", "copy"])
    if kind in ("attend", "window"):
        t = rng.choice(["bf16", "bf16", "fp16", "e4m3"])
        case = _attend(None, R=_log(rng, 1, 96), H=rng.choice([1, 2, 4, 5, 8, 16]), G=rng.choice([1, 2, 3, 4, 6, 7, 8, 8, 12, 16, 24]),
                       D=rng.choice([64, 64, 80, 96, 128, 128, 128, 192, 256]), P=rng.choice([1, 8, 16, 16, 24, 32, 64, 256]), type=t,
                       io=t if t != "e4m3" else rng.choice(["bf16", "fp16"]), style=rng.choice(["page", "page", "head", "padded"]))
        # the padded plain form and the pool stay below the largest listed case
        most = 60_000_000 // (case["H"] * case["D"] * case["R"])
        case["hi"] = max(2, min(_log(rng, 2, 100_000), most))
        case["lo"] = rng.randint(1, case["hi"])
        if kind == "window":
            case["window"], case["sinks"] = _log(rng, 1, 2000), rng.choice([0, 0, 1, 4, 5, 128])
    elif kind == "latent":
        case = _attend(None, R=_log(rng, 1, 48), H=1, G=rng.choice([1, 8, 16, 16, 24, 32, 64, 96, 128, 128]), P=rng.choice([1, 16, 32, 64, 64, 100]),
                       style=rng.choice(["page", "page", "padded"]))
        case["type"] = case["io"] = rng.choice(["bf16", "bf16", "fp16"])
        case["D"], case["Dv"] = rng.choice([(576, 512), (576, 512), (576, 512), (288, 256), (192, 128), (320, 320)])
        case["hi"] = max(2, min(_log(rng, 2, 60_000), 80_000_000 // (576 * case["R"])))
        case["lo"] = rng.randint(1, case["hi"])
        if rng.random() < 0.2:
            case["window"], case["sinks"] = _log(rng, 1, 2000), rng.choice([0, 4])
    else:
        case = _pages(None, kind, R=rng.randint(2, 96), L=rng.choice([1, 2, 4, 8]), P=rng.choice([1, 8, 16, 16, 24, 64]),
                      style=rng.choice(["page", "page", "head", "padded"]))
        if rng.random() < 0.3:
            case.update(F=1, H=1, D=576, style="page")
        else:
            case.update(H=rng.choice([1, 2, 8]), D=rng.choice([64, 80, 128]))
        most = 500_000_000 // (case["R"] * case["L"] * case["F"] * case["H"] * case["D"] * 2)
        case["hi"] = max(2, min(_log(rng, 2, 4000), most))
        case["lo"] = rng.randint(1, case["hi"])
        case["free"], case["new"] = rng.randint(1, max(1, case["R"] // 2)), rng.choice([1, 1, 2, 7])
        case["forks"] = rng.randint(1, case["free"])
        case["n"] = _log(rng, 1, max(1, min(400, 150_000_000 // (case["L"] * case["F"] * case["H"] * case["D"] * 2 * case["P"]))))
    if kind in ("attend", "window", "latent"):
        case["empty"] = rng.choice([0, 0, 0, 1])  # a batch padded with a row that holds nothing
    return {k: v for k, v in case.items() if k != "name"}


# --------------------------------------------------------------------------------- the inputs

def _lengths(case, seed):
    rng = np.random.Generator(np.random.PCG64([seed, 1]))
    sl = rng.integers(case["lo"], case["hi"] + 1, size=case["R"]).astype(np.int64)
    if case.get("empty"):
        sl[rng.integers(0, case["R"])] = 0
    return sl, rng


def _tables(sl, P, pool_pages, maxp, rng):
    """A block table over a random permutation of the pool, -1 past each row's last page."""
    pages = -(-sl // P)
    perm = rng.permutation(pool_pages)[:int(pages.sum())]
    bt = np.full((len(sl), maxp), -1, np.int64)
    col = np.arange(maxp)[None, :]
    bt[col < pages[:, None]] = perm
    return bt


def _pool_pages(c):
    """Pages of a pool that holds every request at its longest, the forks and what is added."""
    return c["R"] * -(-c["hi"] // c["P"]) + c["forks"] + c["R"] * (1 + c["new"] // c["P"]) + 2


def _pool(L, N, F, P, H, D, dtype, style, seed):
    """The pool as a flat buffer of elements, and a view [L, N, F, P, H, D] of it."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + 11)
    pad = 16 if style == "padded" else 0  # elements between two tokens' rows
    shape = (L, N, F, H, P, D) if style == "head" else (L, N, F, P, H * D + pad)
    n = math.prod(shape)
    flat = torch.empty(n, dtype=dtype, device="cuda")
    step = 1 << 27
    for at in range(0, n, step):
        some = torch.randn(min(step, n - at), generator=g, device="cuda", dtype=torch.float16 if dtype != torch.bfloat16 else dtype)
        flat[at:at + step] = some.to(dtype)
    if style == "head":
        return flat, flat.view(shape).permute(0, 1, 2, 4, 3, 5)
    return flat, flat.view(shape)[..., :H * D].unflatten(-1, (H, D))


def _int(x, kind=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(x)).to(device="cuda", dtype=kind)


def prepare(case, seed):
    c = dict(case)
    sl, rng = _lengths(c, seed)
    P = c["P"]
    if c["kind"] == "attend":
        F = 1 if c["Dv"] else 2
        maxp = int(-(-c["hi"] // P))
        N = int((-(-sl // P)).sum()) * 5 // 4 + 2
        bt = _tables(sl, P, N, maxp, rng)
        flat, view = _pool(1, N, F, P, c["H"], c["D"], _TORCH[c["type"]], c["style"], seed)
        Hq, Dv = c["H"] * c["G"], c["Dv"] or c["D"]
        g = torch.Generator(device="cuda")
        g.manual_seed(seed * 104729 + 5)
        q = torch.randn((c["R"], Hq, c["D"]), generator=g, device="cuda").to(_TORCH[c["io"]])
        return dict(case=c, flat=flat, view=view, block_table=_int(bt), seq_lens=_int(sl), total=int(sl.sum()), q=q,
                    out=torch.empty((c["R"], Hq, Dv), dtype=q.dtype, device="cuda"),
                    lse=torch.empty((c["R"], Hq), dtype=torch.float32, device="cuda"),
                    scale=c["D"] ** -0.5, scales=(0.75, 1.25) if c["type"] == "e4m3" else (1.0, 1.0))
    R, F = c["R"], c["F"]
    maxp = int(-(-(c["hi"] + c["new"]) // P))
    if c["kind"] == "copy":
        N = 2 * c["n"] + c["n"] // 2 + 2
        flat, view = _pool(c["L"], N, F, P, c["H"], c["D"], torch.bfloat16, c["style"], seed)
        ids = rng.permutation(N)
        return dict(case=c, flat=flat, view=view, src=_int(ids[:c["n"]]), dst=_int(ids[c["n"]:2 * c["n"]]))
    N = _pool_pages(c)
    bt = _tables(sl, P, N, maxp, rng)
    ended = rng.permutation(R)[:c["free"]]
    ref = np.zeros(N, np.int64)
    np.add.at(ref, bt[bt >= 0], 1)
    if c["kind"] == "compact":  # the ended requests are gone already: their pages are the holes
        gone = bt[ended]
        np.add.at(ref, gone[gone >= 0], -1)
        bt[ended], sl[ended] = -1, 0
    flat, view = _pool(c["L"], N, F, P, c["H"], c["D"], torch.bfloat16, c["style"], seed)
    s = dict(case=c, flat=flat, view=view, block_table=_int(bt), seq_lens=_int(sl), ref=_int(ref))
    for k in ("block_table", "seq_lens", "ref"):
        s[k + "_out"] = torch.empty_like(s[k])
    s["num_used"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    s["page_map"] = torch.zeros(N, dtype=torch.int32, device="cuda")
    if c["kind"] == "turn":
        live = np.setdiff1d(np.arange(R), ended)
        children = ended[:c["forks"]]
        parents = rng.choice(live if len(live) else ended, size=len(children))
        new = np.zeros(R, np.int64)
        new[live] = c["new"]
        if len(live):
            new[children] = c["new"]
        s.update(ended=_int(ended), parents=_int(parents), children=_int(children), new=_int(new))
    return s


# ------------------------------------------------------------------------------ the plain forms

def _rows(table, index):
    """table[index], also for elements that torch does not index (8-bit floats)."""
    if table.element_size() == 1:
        return table.view(torch.uint8)[index].view(table.dtype)
    return table[index]


def _plain_attend(s):
    c = s["case"]
    P, W, H, G = c["P"], c["window"], c["H"], c["G"]
    R, maxp = s["block_table"].shape
    n_all = s["seq_lens"].long()[:, None]
    first = (n_all - W).clamp(min=0) if W else torch.zeros_like(n_all)
    sinks = first.clamp(max=c["sinks"])
    n = sinks + n_all - first                                    # visible tokens of each request
    at = torch.arange(min(maxp * P, W + c["sinks"]) if W else maxp * P, device="cuda")[None, :]
    seen = at < n
    token = torch.where(at < sinks, at, at - sinks + first).masked_fill(~seen, 0)
    page = s["block_table"].long().gather(1, token // P).masked_fill(~seen, 0)
    pool = s["view"][0]
    k = _rows(pool[:, 0], (page, token % P)).float() * s["scales"][0]           # [R, n, H, D]
    v = k[..., :c["Dv"]] if c["Dv"] else _rows(pool[:, 1], (page, token % P)).float() * s["scales"][1]
    v = v.masked_fill(~seen[:, :, None, None], 0.0)
    q = s["q"].float().unflatten(1, (H, G))
    score = torch.einsum("rhgd,rnhd->rhgn", q, k) * s["scale"]
    score = score.masked_fill(~seen[:, None, None, :], -math.inf)
    top = score.amax(-1, keepdim=True)
    top = top.masked_fill(top == -math.inf, 0.0)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    out = torch.einsum("rhgn,rnhd->rhgd", p, v) / total.masked_fill(n[:, None, None] == 0, 1.0)
    lse = (top + torch.log(total)).squeeze(-1)
    return [out.flatten(1, 2).to(s["q"].dtype), lse.flatten(1, 2)]


def _plain_turn(s):
    P = s["case"]["P"]
    bt, sl, ref = s["block_table"].clone(), s["seq_lens"].clone(), s["ref"].clone()
    col = torch.arange(bt.shape[1], device="cuda")[None, :]

    def count(rows, mask, by):  # every page named by rows[mask] is used `by` times more
        ref.index_add_(0, rows.clamp(min=0).flatten().long(), mask.flatten().to(ref.dtype) * by)

    # the ended requests give their pages back
    rows = s["ended"].long()
    count(bt[rows], col < -(-sl[rows] // P)[:, None], -1)
    bt[rows], sl[rows] = -1, 0
    # the children share their parents' full pages and get a page of their own for the rest
    parents, children = s["parents"].long(), s["children"].long()
    full, tail = (sl[parents] // P)[:, None], sl[parents] % P
    need = tail > 0
    free = torch.argsort((ref > 0).int(), stable=True).to(ref.dtype)  # the lowest free pages come first
    fresh = free[(need.cumsum(0) - 1).clamp(min=0)]
    old = bt[parents]
    mine = torch.where(col < full, old, torch.where((col == full) & need[:, None], fresh[:, None], -1))
    count(mine, mine >= 0, 1)
    bt[children], sl[children] = mine, sl[parents]
    which = need.nonzero().squeeze(1)
    src, dst = old.gather(1, full.clamp(max=bt.shape[1] - 1).long()).squeeze(1)[which].long(), fresh[which].long()
    keep = (torch.arange(P, device="cuda")[None, :] < tail[which, None])[None, :, None, :, None, None]
    view = s["view"]
    view[:, dst] = torch.where(keep, view[:, src], view[:, dst])
    # every request grows by its new tokens
    have, want = -(-sl // P), -(-(sl + s["new"]) // P)
    start = (want - have).cumsum(0) - (want - have)
    free = torch.argsort((ref > 0).int(), stable=True).to(ref.dtype)
    grown = (col >= have[:, None]) & (col < want[:, None])
    bt = torch.where(grown, free[(start[:, None] + col - have[:, None]).clamp(0, len(free) - 1).long()], bt)
    count(bt, grown, 1)
    sl += s["new"]
    return [bt, sl, ref, s["flat"].view(torch.int16)]


def _plain_compact(s):
    P = s["case"]["P"]
    bt, ref = s["block_table"], s["ref"]
    used = ref > 0
    n = used.sum()
    page = torch.arange(len(ref), device="cuda")
    holes = (~used & (page < n)).nonzero().squeeze(1)
    movers = (used & (page >= n)).nonzero().squeeze(1)
    s["view"][:, holes] = s["view"][:, movers]
    to = torch.where(used, page, -1).to(torch.int32)
    to[movers] = holes.to(torch.int32)
    ref = ref.clone()
    ref[holes], ref[movers] = ref[movers], 0
    inside = torch.arange(bt.shape[1], device="cuda")[None, :] < -(-s["seq_lens"] // P)[:, None]
    bt = torch.where(inside, to[bt.clamp(min=0).long()], bt)
    return [bt, s["seq_lens"].clone(), ref, n.to(torch.int32)[None], to, s["flat"].view(torch.int16)]


def _plain_copy(s):
    s["view"][:, s["dst"].long()] = s["view"][:, s["src"].long()]
    return [s["flat"].view(torch.int16)]


# ------------------------------------------------------------------------ the library's entry points

def _handle(s):
    """What a program builds once for a cache and keeps: the descriptors and a workspace."""
    from paper_2607_28633_b200 import binding as tk
    c, v = s["case"], s["view"]
    L, N, F, P, H, D = v.shape
    e = v.element_size()
    lo = tk.make_layout(L, F, H, D, e, P, N)
    lo.pool_layer_stride, lo.pool_page_stride, lo.pool_kv_stride, lo.pool_token_stride, lo.pool_head_stride = (x * e for x in v.stride()[:5])
    h = dict(tk=tk, lo=lo)
    if c["kind"] == "attend":
        h["batch"] = tk.make_batch(s["block_table"], s["seq_lens"], -1 if c["window"] else s["total"], window_tokens=c["window"])
        kind = {"bf16": tk.TOPKV_TYPE_BF16, "fp16": tk.TOPKV_TYPE_FP16, "e4m3": tk.TOPKV_TYPE_E4M3}
        h["att"] = tk.make_attention(s["q"], s["out"], kind[c["type"]], kind[c["io"]], s["scale"], value_dim=c["Dv"], sink_tokens=c["sinks"],
                                     k_scale=s["scales"][0], v_scale=s["scales"][1], lse=s["lse"])
        n = tk.check(tk.topkv_attend_workspace_bytes(lo, h["batch"], h["att"]))
    elif c["kind"] == "copy":
        return h
    else:
        out = (s["block_table_out"], s["seq_lens_out"], s["ref_out"])
        h["batch"] = tk.make_batch(s["block_table"], s["seq_lens"])
        h["tables"] = tk.make_page_tables(s["ref"], *out)
        h["batch_out"] = tk.make_batch(out[0], out[1])      # the later calls of a turn work in place
        h["tables_out"] = tk.make_page_tables(out[2], *out)
        n = tk.check(tk.topkv_page_workspace_bytes(lo, h["batch"], c["forks"]))
    h["ws"] = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    return h


def _own(s):
    h = s.get("handle")
    if h is None:
        h = s["handle"] = _handle(s)
    tk, lo, kind = h["tk"], h["lo"], s["case"]["kind"]
    stream = torch.cuda.current_stream().cuda_stream
    if kind == "attend":
        tk.check(tk.topkv_attend_layer(0, s["flat"], lo, h["batch"], h["att"], s["q"], s["out"], h["ws"], h["ws"].numel(), stream))
        return [s["out"], s["lse"]]
    if kind == "copy":
        tk.check(tk.topkv_copy_pages(0, lo.num_layers, s["flat"], lo, s["src"], s["dst"], s["src"].numel(), stream))
        return [s["flat"].view(torch.int16)]
    ws, tables = h["ws"], [s["block_table_out"], s["seq_lens_out"], s["ref_out"]]
    if kind == "turn":
        tk.check(tk.topkv_free_requests(lo, h["batch"], h["tables"], s["ended"], s["ended"].numel(), stream))
        tk.check(tk.topkv_fork_requests(s["flat"], lo, h["batch_out"], h["tables_out"], s["parents"], s["children"], s["parents"].numel(),
                                        ws, ws.numel(), stream))
        tk.check(tk.topkv_extend_requests(lo, h["batch_out"], h["tables_out"], s["new"], ws, ws.numel(), stream))
        return tables + [s["flat"].view(torch.int16)]
    tk.check(tk.topkv_compact_pages(s["flat"], lo, h["batch"], h["tables"], s["num_used"], s["page_map"], ws, ws.numel(), stream))
    return tables + [s["num_used"], s["page_map"], s["flat"].view(torch.int16)]


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    if kind == "attend":
        return _plain_attend(state)
    return {"turn": _plain_turn, "compact": _plain_compact, "copy": _plain_copy}[kind](state)


# ----------------------------------------------------------------------------------- the bounds

def work(case):
    """Each input read once, each output written once; lengths of one seed stand for the case's."""
    c = case
    sl, _ = _lengths(c, 0)
    P = c["P"]
    if c["kind"] == "attend":
        n = np.minimum(sl, c["window"] + c["sinks"]) if c["window"] else sl
        F, e, Dv = (1 if c["Dv"] else 2), (1 if c["type"] == "e4m3" else 2), c["Dv"] or c["D"]
        rows = c["R"] * c["H"] * c["G"]
        return {"bytes": int(n.sum()) * F * c["H"] * c["D"] * e + rows * (2 * c["D"] + 2 * Dv + 4) + int((-(-n // P)).sum()) * 4,
                "flops": 2 * int(n.sum()) * c["H"] * c["G"] * (c["D"] + Dv)}
    page = c["L"] * c["F"] * P * c["H"] * c["D"] * 2
    if c["kind"] == "copy":
        return {"bytes": 2 * c["n"] * page + 8 * c["n"], "flops": 0}
    pages = -(-sl // P)
    rng = _lengths(c, 0)[1]
    tables = 2 * 4 * (int(pages.sum()) + c["R"] + _pool_pages(c))
    if c["kind"] == "turn":
        return {"bytes": tables + 2 * c["forks"] * page // 2, "flops": 0}  # half a page is left over, on average
    N = _pool_pages(c)
    bt = _tables(sl, P, N, int(-(-(c["hi"] + c["new"]) // P)), rng)
    bt[rng.permutation(c["R"])[:c["free"]]] = -1
    used = int((bt >= 0).sum())
    return {"bytes": tables + 2 * page * int((bt >= used).sum()), "flops": 0}


def exact(case, seed):
    """One request at a time in 64 bits, from the definition: softmax(scale q.k) over the visible
    tokens, times their values. Calls that only move words have no computed numbers."""
    c = case
    if c["kind"] != "attend":
        return None
    s = prepare(c, seed)
    lens, bt = s["seq_lens"].tolist(), s["block_table"].long()
    pool, P = s["view"][0], c["P"]
    Hq, Dv = s["out"].shape[1:]
    out = torch.zeros((c["R"], Hq, Dv), dtype=torch.float64, device="cuda")
    lse = torch.full((c["R"], Hq), -math.inf, dtype=torch.float64, device="cuda")
    for r, n in enumerate(lens):
        i = torch.arange(n, device="cuda")
        if c["window"]:
            i = i[(i >= n - c["window"]) | (i < c["sinks"])]
        if len(i) == 0:
            continue
        where = (bt[r, i // P], i % P)
        for h in range(c["H"]):
            rows = slice(h * c["G"], (h + 1) * c["G"])
            k = _rows(pool[:, 0, :, h], where).double() * s["scales"][0]
            v = k[:, :c["Dv"]] if c["Dv"] else _rows(pool[:, 1, :, h], where).double() * s["scales"][1]
            score = s["q"][r, rows].double() @ k.T * s["scale"]
            lse[r, rows] = torch.logsumexp(score, 1)
            out[r, rows] = torch.softmax(score, 1) @ v
    return [out, lse]

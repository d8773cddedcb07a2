"""More operators of the decode side's paged cache, as cases that can be timed and compared.

``append``    new tokens' K and V are written into the paged cache, rotated by their positions on the
              way, and the queries of the same tokens are rotated.
``plan``      which requests of a batch begin with the same pages, from the block table.
``shared``    attention of one new token per request, where groups of requests share a long prefix:
              the prefix is read once for a group.
``bounds``    the bounds of each page's keys in 8 bits, which a cheap score of a page is made of.
``sparse``    for each request and KV head the pages with the best scores, and attention over them.

``run`` computes them in their plain form, in elementary torch operations, or, where ``own`` is
true, by the library's entry points.
"""
import math

import numpy as np
import torch

own = False

_TORCH = {"bf16": torch.bfloat16, "fp16": torch.float16, "e4m3": torch.float8_e4m3fn}
_127TH = float(np.float32(1) / np.float32(127))


# ---------------------------------------------------------------------------------- the cases

def _append(name, **kw):
    case = dict(name=name, kind="append", R=4, lo=17, hi=255, new_lo=1, new_hi=1, F=2, H=8, G=8, D=128, P=16, type="bf16", io="bf16",
                style="page", first=0, count=128, pairs=False, far=0, base=500000.0, grow=1.0, empty=0)
    case.update(kw)
    return case


def _shared(name, kind="shared", **kw):
    case = dict(name=name, kind=kind, groups=1, lone=0, members_lo=4, members_hi=4, prefix_lo=256, prefix_hi=256, lo=1, hi=60, H=8, G=8,
                D=128, P=16, type="bf16", io="bf16", style="page", empty=0)
    case.update(kw)
    return case


def _sparse(name, kind="sparse", **kw):
    case = dict(name=name, kind=kind, R=2, lo=2000, hi=3001, H=8, G=4, D=128, P=16, type="bf16", io="bf16", style="page", budget=32,
                firsts=1, lasts=2, window=0, empty=0)
    case.update(kw)
    return case


def listed():
    return [
        # one token for each of four short requests: a decode step's call, all latency
        _append("append_token", R=4),
        # ragged chunks of prompts into an 8-bit cache, positions far beyond a million, frequencies stretched
        _append("append_prompts", R=12, lo=2048, hi=6000, new_lo=1, new_hi=2047, G=4, type="e4m3", far=1_000_003, grow=8.0),
        # latent rows of a serving batch: only the last 64 of 576 elements turn, as neighbours; all 128 heads
        _append("append_latent", R=256, lo=1, hi=1500, F=1, H=1, G=128, D=576, P=64, first=512, count=64, pairs=True, base=10000.0),
        # a handful of requests: two prompts that some of them share, and one more
        _shared("plan_short", "plan", groups=2, lone=1, members_lo=2, members_hi=3),
        # a serving batch over a few long prompts
        _shared("plan_batch", "plan", groups=8, lone=20, members_lo=8, members_hi=40, prefix_lo=600, prefix_hi=6000, hi=1000),
        # four samples of one short prompt
        _shared("shared_short"),
        # beams and samples of six prompts in an 8-bit cache beside two requests that share nothing
        _shared("shared_beams", groups=6, lone=2, members_lo=3, members_hi=17, prefix_lo=500, prefix_hi=4000, hi=300, type="e4m3", G=4),
        # a full batch behind one long instruction
        _shared("shared_prompt", members_lo=64, members_hi=64, prefix_lo=16384, prefix_hi=16384, lo=100, hi=1000),
        # the page that the newest token went to, in every request of a batch
        _sparse("bounds_step", "bounds", R=64, lo=200, hi=2000, window=1, type="e4m3"),
        # all pages of prompts that have just arrived
        _sparse("bounds_prompts", "bounds", R=16, lo=512, hi=4096),
        # two requests of a few thousand tokens, 512 of them seen
        _sparse("sparse_short"),
        # four very long requests of odd lengths, 2,048 tokens seen
        _sparse("sparse_long", R=4, lo=65537, hi=131071, budget=128, firsts=4, lasts=8),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "append", "append", "plan", "shared", "shared", "shared", "bounds", "sparse", "sparse"])
    t = rng.choice(["bf16", "bf16", "fp16", "e4m3"])
    common = dict(H=rng.choice([1, 2, 4, 5, 8, 8, 16]), G=rng.choice([1, 2, 3, 4, 4, 6, 7, 8, 8, 12, 16, 24]), D=rng.choice([64, 64, 80, 96, 128, 128, 128, 192, 256]),
                  P=rng.choice([1, 8, 16, 16, 24, 32, 64, 256]), type=t, io=t if t != "e4m3" else rng.choice(["bf16", "fp16"]),
                  style=rng.choice(["page", "page", "head", "padded"]), empty=rng.choice([0, 0, 0, 1]))
    if kind == "append":
        case = _append(None, R=_log(rng, 1, 256), far=rng.choice([0, 0, 131_072, 1_000_003, 100_000_007]), base=rng.choice([10000.0, 500000.0, 1e6]),
                       pairs=rng.choice([False, False, True]), grow=rng.choice([1.0, 1.0, 4.0, 8.0, 40.0]), **common)
        if rng.random() < 0.25:
            case.update(F=1, H=1, G=rng.choice([1, 16, 64, 128]), D=576, first=512, count=64)
            if t == "e4m3":
                case["type"] = case["io"]
        else:
            case["count"] = rng.choice([case["D"], case["D"], case["D"] // 2, 16, 0])
            case["first"] = rng.choice([0, 0, case["D"] - case["count"]])
        # rows of K, V and Q together, and the pool that is handed back whole, stay below the listed ones
        case["R"] = max(1, min(case["R"], 60_000_000 // (case["F"] * case["H"] * case["D"] * case["P"])))
        rows = case["F"] * case["H"] + case["H"] * case["G"]
        case["new_hi"] = rng.choice([1, max(1, min(_log(rng, 1, 4096), 80_000_000 // (rows * case["D"] * case["R"])))])
        case["new_lo"] = rng.randint(0 if case["new_hi"] > 1 else 1, case["new_hi"])
        case["hi"] = case["new_hi"] + min(_log(rng, 1, 6000), max(1, 60_000_000 // (case["R"] * case["F"] * case["H"] * case["D"])))
        case["lo"] = rng.randint(case["new_hi"], case["hi"])
    elif kind in ("plan", "shared"):
        case = _shared(None, kind, **common)
        case["groups"], case["lone"] = _log(rng, 1, 12), rng.choice([0, 0, 1, 9])
        case["members_hi"] = _log(rng, 2, 64)
        case["members_lo"] = rng.randint(1, case["members_hi"])
        case["hi"] = _log(rng, 2, 2000)
        rows = case["groups"] * case["members_hi"] + case["lone"]
        case["hi"] = max(2, min(case["hi"], 100_000_000 // (case["H"] * case["D"] * rows)))
        most = max(64, 60_000_000 // (case["H"] * case["D"] * rows) - case["hi"])   # the plain form reads the prefix once a request
        case["prefix_hi"] = min(_log(rng, 32, 40_000), most)
        case["prefix_lo"] = rng.randint(1, case["prefix_hi"])
        case["lo"] = rng.randint(0 if kind == "plan" else 1, case["hi"])
    else:
        case = _sparse(None, kind, R=_log(rng, 1, 48), **common)
        case["P"] = rng.choice([1, 8, 16, 16, 16, 24, 32, 64, 64])
        case["hi"] = max(2, min(_log(rng, 2, 140_000), 300_000_000 // (case["H"] * case["D"] * case["R"])))
        case["lo"] = rng.randint(1, case["hi"])
        case["budget"] = max(1, _log(rng, 16, 4096) // case["P"])
        case["firsts"] = rng.choice([0, 1, 1, 4])
        case["lasts"] = rng.choice([1, 1, 2, 5, 8])
        if kind == "bounds":
            case["hi"] = min(case["hi"], 20_000)
            case["lo"] = min(case["lo"], case["hi"])
            case["window"] = rng.choice([0, 0, 1, 1, 40])
    return {k: v for k, v in case.items() if k != "name"}


# --------------------------------------------------------------------------------- the inputs

def _rng(seed):
    return np.random.Generator(np.random.PCG64([seed, 1]))


def _int(x, kind=torch.int32):
    return torch.from_numpy(np.ascontiguousarray(x)).to(device="cuda", dtype=kind)


def _normal(shape, g, dtype):
    """Standard normal values, made in parts: 8-bit floats have no generator of their own."""
    n = math.prod(shape)
    flat = torch.empty(n, dtype=dtype, device="cuda")
    step = 1 << 27
    for at in range(0, n, step):
        some = torch.randn(min(step, n - at), generator=g, device="cuda", dtype=torch.bfloat16 if dtype == torch.bfloat16 else torch.float16)
        flat[at:at + step] = some.to(dtype)
    return flat.view(shape)


def _pool(c, N, g):
    """The pool of one layer as a flat buffer of elements, and a view [N, F, P, H, D] of it."""
    F, P, H, D = c.get("F", 2), c["P"], c["H"], c["D"]
    pad = 16 if c["style"] == "padded" else 0  # elements between two tokens' rows
    flat = _normal((N, F, H, P, D) if c["style"] == "head" else (N, F, P, H * D + pad), g, _TORCH[c["type"]])
    view = flat.permute(0, 1, 3, 2, 4) if c["style"] == "head" else flat[..., :H * D].unflatten(-1, (H, D))
    return flat.view(-1), view


def _tables(sl, P, N, maxp, rng):
    """A block table over a random permutation of the pool, -1 past each row's last page."""
    pages = -(-sl // P)
    bt = np.full((len(sl), maxp), -1, np.int64)
    bt[np.arange(maxp)[None, :] < pages[:, None]] = rng.permutation(N)[:int(pages.sum())]
    return bt


def _frequencies(c):
    """Of each pair, in radians a position: the geometric series of `base`, stretched by `grow`."""
    n = c["count"]
    return float(c["base"]) ** (-np.arange(0, n, 2, dtype=np.float64) / max(n, 1)) / c["grow"]


def _append_lengths(c, seed):
    """The case's lengths and new tokens: the same for every seed, which only says whose they are."""
    fixed, rng = _rng(0), _rng(seed)
    new = fixed.integers(c["new_lo"], c["new_hi"] + 1, size=c["R"])
    sl = np.maximum(fixed.integers(c["lo"], c["hi"] + 1, size=c["R"]), new)
    if c["empty"] and c["R"] > 1:
        sl[0] = 0  # a row that is left out: what it brings is not written
    whose = rng.permutation(c["R"])
    return sl[whose].astype(np.int64), new[whose].astype(np.int64), rng


def _prepare_append(c, seed):
    sl, new, rng = _append_lengths(c, seed)
    F, H, G, D, P = c["F"], c["H"], c["G"], c["D"], c["P"]
    N = int((-(-sl // P)).sum()) + 2
    bt = _tables(sl, P, N, int(-(-c["hi"] // P)), rng)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + 11)
    flat, view = _pool(c, N, g)
    T = int(new.sum())
    cu = np.concatenate([[0], np.cumsum(new)])
    row = np.repeat(np.arange(c["R"]), new)
    index = sl[row] - new[row] + np.arange(T) - cu[row]
    # one buffer for the projections' outcome: a token's queries, keys and values behind each other
    Hq, rows = H * G, H * G + F * H
    qkv = _normal((max(T, 1), rows, D), g, _TORCH[c["io"]])[:T]
    return dict(case=c, flat=flat, view=view, block_table=_int(bt), seq_lens=_int(sl), total=T, cu=_int(cu, torch.int64), one=c["new_hi"] == 1,
                q=qkv[:, :Hq], k=qkv[:, Hq:Hq + H], v=qkv[:, Hq + H:] if F == 2 else None, q_out=torch.zeros((T, Hq, D), dtype=qkv.dtype, device="cuda"),
                positions=_int(index + c["far"]), frequencies=_frequencies(c), turn=1.0 if c["grow"] == 1.0 else 0.1 * math.log(c["grow"]) + 1.0,
                scales=(0.5, 0.75) if c["type"] == "e4m3" else (1.0, 1.0))


def _groups(c, seed):
    """Lengths, rows of each group and shared pages of each; the seed says which rows these are."""
    fixed, rng = _rng(0), _rng(seed)
    size = [int(fixed.integers(c["members_lo"], c["members_hi"] + 1)) for _ in range(c["groups"])] + [1] * c["lone"]
    prefix = [int(fixed.integers(c["prefix_lo"], c["prefix_hi"] + 1)) // c["P"] for _ in size]
    R = sum(size)
    rows = np.split(rng.permutation(R), np.cumsum(size)[:-1])
    sl = np.zeros(R, np.int64)
    for m, n in zip(rows, prefix):
        sl[m] = n * c["P"] + fixed.integers(c["lo"], c["hi"] + 1, size=len(m))
    if c["empty"] and R > 1:
        sl[rows[0][0]] = 0
    return sl, rows, prefix, rng


def _most_tokens(c):
    return c["prefix_hi"] // c["P"] * c["P"] + c["hi"]


def _prepare_shared(c, seed):
    sl, rows, prefix, rng = _groups(c, seed)
    P, H, D = c["P"], c["H"], c["D"]
    pages = -(-sl // P)
    N = sum(n + int(np.maximum(pages[m] - n, 0).sum()) for m, n in zip(rows, prefix)) + 2
    ids, at = rng.permutation(N), 0
    bt = np.full((len(sl), int(-(-_most_tokens(c) // P))), -1, np.int64)
    for m, n in zip(rows, prefix):
        common, at = ids[at:at + n], at + n
        for r in m:
            k = min(n, int(pages[r]))
            bt[r, :k] = common[:k]
            bt[r, k:pages[r]], at = ids[at:at + pages[r] - k], at + int(pages[r]) - k
    s = dict(case=c, block_table=_int(bt), seq_lens=_int(sl), pages=N, plan=torch.zeros((6, len(sl)), dtype=torch.int32, device="cuda"))
    if c["kind"] == "plan":
        return s
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + 11)
    flat, view = _pool(c, N, g)
    q = _normal((len(sl), H * c["G"], D), g, _TORCH[c["io"]])
    s.update(flat=flat, view=view, q=q, out=torch.empty_like(q), lse=torch.empty(q.shape[:2], dtype=torch.float32, device="cuda"),
             scale=D ** -0.5, scales=(0.75, 1.25) if c["type"] == "e4m3" else (1.0, 1.0))
    return s


def _sparse_lengths(c, seed):
    fixed, rng = _rng(0), _rng(seed)
    sl = fixed.integers(c["lo"], c["hi"] + 1, size=c["R"]).astype(np.int64)
    if c["empty"] and c["R"] > 1:
        sl[0] = 0
    return rng.permutation(sl), rng


def _prepare_sparse(c, seed):
    sl, rng = _sparse_lengths(c, seed)
    P, H, D, R = c["P"], c["H"], c["D"], c["R"]
    N = int((-(-sl // P)).sum()) + 2
    bt = _tables(sl, P, N, int(-(-c["hi"] // P)), rng)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 7919 + 11)
    flat, view = _pool(c, N, g)
    # no page's bounds are known yet: nothing in the buffers counts
    s = dict(case=c, flat=flat, view=view, block_table=_int(bt), seq_lens=_int(sl), bounds=torch.zeros((N, H, 2, D), dtype=torch.int8, device="cuda"),
             steps=torch.zeros((N, H), dtype=torch.float32, device="cuda"))
    if c["kind"] == "bounds":
        return s
    _bounds_of(s, 0)
    q = _normal((R, H * c["G"], D), g, _TORCH[c["io"]])
    s.update(q=q, out=torch.empty_like(q), lse=torch.empty((R, H * c["G"]), dtype=torch.float32, device="cuda"),
             picked=torch.empty((R, H, c["budget"]), dtype=torch.int32, device="cuda"), scale=D ** -0.5,
             scales=(0.75, 1.25) if c["type"] == "e4m3" else (1.0, 1.0))
    return s


def prepare(case, seed):
    c = dict(case)
    if c["kind"] == "append":
        return _prepare_append(c, seed)
    return (_prepare_shared if c["kind"] in ("plan", "shared") else _prepare_sparse)(c, seed)


# ------------------------------------------------------------------------------ the plain forms

def _words(t):
    """8-bit floats as the bytes that torch can index and assign."""
    return t.view(torch.uint8) if t.element_size() == 1 else t


def _rows(table, index):
    return _words(table)[index].view(table.dtype)


def _turned(x, angle, c, m):
    """x [T, heads, D] with the elements first .. first + count - 1 rotated by angle [T, count / 2]."""
    n, first = c["count"], c["first"]
    if n == 0:
        return x
    cos, sin = (torch.cos(angle) * m).to(x.dtype)[:, None, :], (torch.sin(angle) * m).to(x.dtype)[:, None, :]
    part = x[..., first:first + n]
    a, b = (part[..., 0::2], part[..., 1::2]) if c["pairs"] else (part[..., :n // 2], part[..., n // 2:])
    u, w = a * cos - b * sin, a * sin + b * cos
    part = torch.stack([u, w], -1).flatten(-2) if c["pairs"] else torch.cat([u, w], -1)
    return torch.cat([x[..., :first], part, x[..., first + n:]], -1)


def _stored(x, dtype, scale):
    """Values as the cache holds them: divided by the scale, 8-bit ones kept within their range."""
    x = x / scale if scale != 1.0 else x
    return (x.clamp(-448.0, 448.0) if dtype == torch.float8_e4m3fn else x).to(dtype)


def _plain_append(s):
    c, T, P = s["case"], s["total"], s["case"]["P"]
    if T == 0:
        return [s["q_out"], s["flat"]]
    at = torch.arange(T, device="cuda")
    row = torch.searchsorted(s["cu"], at, right=True) - 1
    index = s["seq_lens"].long()[row] - (s["cu"][row + 1] - at)
    there = s["seq_lens"][row] > 0
    # positions can be far: the angles take 64 bits
    angle = s["positions"].double()[:, None] * torch.from_numpy(s["frequencies"]).cuda()[None, :]
    q = _turned(s["q"].float(), angle, c, s["turn"]).to(s["q_out"].dtype)
    s["q_out"].copy_(torch.where(there[:, None, None], q, s["q_out"]))
    row, index = row[there], index[there]
    page = s["block_table"].long()[row, index // P]
    view = _words(s["view"])
    view[page, 0, index % P] = _words(_stored(_turned(s["k"].float(), angle, c, s["turn"])[there], s["view"].dtype, s["scales"][0]))
    if s["v"] is not None:
        view[page, 1, index % P] = _words(_stored(s["v"].float()[there], s["view"].dtype, s["scales"][1]))
    return [s["q_out"], s["flat"]]


def _plain_plan(s):
    P, bt, sl = s["case"]["P"], s["block_table"], s["seq_lens"].long()
    R = len(sl)
    row, col = torch.arange(R, device="cuda"), torch.arange(bt.shape[1], device="cuda")
    full = sl // P
    key = torch.where(full > 0, bt[:, 0].long(), -1 - row)
    alike = key[:, None] == key[None, :]
    leader = torch.where(alike, row[None, :], R).amin(1)
    same = (bt == bt[leader]) & (col[None, :] < torch.minimum(full, full[leader])[:, None])
    common = torch.cumprod(same.long(), 1).sum(1) * P
    members = alike.sum(1)
    shared = torch.where(alike, common[None, :], 1 << 40).amin(1)
    shared = torch.where(members > 1, shared, 0)
    order = torch.argsort(leader * R + row)
    place = torch.empty_like(order)
    place[order] = row
    return [torch.stack([leader, common, shared, members, order, place]).to(torch.int32)]


def _softmax(score, k_seen, v):
    """softmax over the last axis of score [.., rows, n], where k_seen, times v [.., n, D]; and the log of the sum."""
    score = score.masked_fill(~k_seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    top = top.masked_fill(top == -math.inf, 0.0)
    p = torch.exp(score - top)
    total = p.sum(-1, keepdim=True)
    out = (p @ v) / total.masked_fill(total == 0, 1.0)
    return out, (top + torch.log(total)).squeeze(-1)


def _plain_shared(s):
    c, P = s["case"], s["case"]["P"]
    bt, n = s["block_table"].long(), s["seq_lens"].long()[:, None]
    at = torch.arange(bt.shape[1] * P, device="cuda")[None, :]
    seen = at < n
    page = bt.gather(1, (at // P).expand(len(bt), -1)).masked_fill(~seen, 0)
    spot = (at % P).expand(len(bt), -1)
    k = _rows(s["view"][:, 0], (page, spot)).float().permute(0, 2, 1, 3) * s["scales"][0]                    # [R, H, n, D]
    v = _rows(s["view"][:, 1], (page, spot)).float().masked_fill(~seen[:, :, None, None], 0.0).permute(0, 2, 1, 3) * s["scales"][1]
    q = s["q"].float().unflatten(1, (c["H"], c["G"]))
    out, lse = _softmax(q @ k.transpose(-1, -2) * s["scale"], seen[:, None, None, :], v)
    return [out.flatten(1, 2).to(s["q"].dtype), lse.flatten(1, 2)]


def _bounds_of(s, window):
    """Bounds and steps of the pages that hold the last `window` tokens of each request (0: all of them)."""
    c, P = s["case"], s["case"]["P"]
    bt, n = s["block_table"].long(), s["seq_lens"].long()[:, None]
    col = torch.arange(bt.shape[1], device="cuda")[None, :]
    here = (col * P < n) & ((col + 1) * P > ((n - window) if window else torch.zeros_like(n)))
    row, col = here.nonzero(as_tuple=True)
    if len(row) == 0:
        return
    page, held = bt[row, col], (n[row, 0] - col * P).clamp(max=P)
    # no more pages at a time than about 2 GB of keys in 32 bits
    step = max(1, (1 << 29) // (P * c["H"] * c["D"]))
    for at in range(0, len(page), step):
        ids, some = page[at:at + step], held[at:at + step]
        k = _rows(s["view"][:, 0], (ids,)).float()                                                        # [n, P, H, D]
        there = (torch.arange(P, device="cuda")[None, :] < some[:, None])[:, :, None, None]
        low, high = k.masked_fill(~there, math.inf).amin(1), k.masked_fill(~there, -math.inf).amax(1)
        most = torch.maximum(low.abs(), high.abs()).amax(-1)
        step_of = most * torch.tensor(_127TH, device="cuda")
        by = step_of[..., None].expand_as(low)
        usable = (by > 0) & torch.isfinite(by)
        lo8 = torch.floor(low / by).clamp(-127, 127).masked_fill(~usable, 0)
        hi8 = torch.ceil(high / by).clamp(-127, 127).masked_fill(~usable, 0)
        s["bounds"][ids] = torch.stack([lo8, hi8], 2).to(torch.int8)
        s["steps"][ids] = step_of


def _plain_bounds(s):
    _bounds_of(s, s["case"]["window"])
    return [s["bounds"], s["steps"]]


def _plain_select(s):
    c, P = s["case"], s["case"]["P"]
    H, G, K = c["H"], c["G"], c["budget"]
    bt, n = s["block_table"].long(), s["seq_lens"].long()
    pages = -(-n // P)
    col = torch.arange(bt.shape[1], device="cuda")
    seen = col[None, :] < pages[:, None]
    ids = bt.masked_fill(~seen, 0)
    # the queries in 8 bits, a step for each head
    q = s["q"].float().unflatten(1, (H, G))
    step = q.abs().amax(-1) * torch.tensor(_127TH, device="cuda")
    usable = (step > 0) & torch.isfinite(step)
    q8 = torch.round(q / step[..., None]).clamp(-127, 127).masked_fill(~usable[..., None], 0)
    step = step.masked_fill(~usable, 0)
    b, t = s["bounds"][ids].float(), s["steps"][ids].permute(0, 2, 1)                                         # [R, pages, H, 2, D]
    # whole numbers below 2^24: exact in 32 bits, whatever the order
    dot = torch.einsum("rhgd,rnhd->rhgn", q8.clamp(max=0), b[:, :, :, 0]) + torch.einsum("rhgd,rnhd->rhgn", q8.clamp(min=0), b[:, :, :, 1])
    score = (dot * (step[..., None] * t[:, :, None, :])).amax(2) + 0.0
    rank = torch.where(torch.isinf(t), math.inf, score)
    # the last pages before the first ones before the others, should the budget not hold them all
    last, firsts = col[None, :] >= pages[:, None] - c["lasts"], col[None, :] < c["firsts"]
    tier = torch.where(last, 2, torch.where(firsts, 1, 0))[:, None, :].expand_as(rank).masked_fill(~seen[:, None, :], -1)
    rank = torch.where(tier > 0, torch.where(tier == 2, col.float()[None, None, :], -col.float()[None, None, :]), rank)
    by_rank = torch.sort(rank.masked_fill(~seen[:, None, :], -math.inf), descending=True, stable=True).indices
    best = by_rank.gather(2, torch.sort(tier.gather(2, by_rank), descending=True, stable=True).indices)[..., :K]
    held = torch.arange(best.shape[2], device="cuda")[None, None, :] < pages[:, None, None]
    best = torch.sort(best.masked_fill(~held, 1 << 30)).values
    best = best.masked_fill(best == 1 << 30, -1)
    return torch.nn.functional.pad(best, (0, K - best.shape[2]), value=-1)


def _plain_sparse(s):
    c, P = s["case"], s["case"]["P"]
    H, G = c["H"], c["G"]
    best = _plain_select(s)                                                                              # [R, H, K]
    token = (best[..., None] * P + torch.arange(P, device="cuda")).flatten(2)                              # [R, H, K P]
    seen = (best >= 0).repeat_interleave(P, 2) & (token < s["seq_lens"].long()[:, None, None])
    token = token.masked_fill(~seen, 0)
    page = s["block_table"].long().gather(1, (token // P).flatten(1)).view_as(token).masked_fill(~seen, 0)
    head = torch.arange(H, device="cuda")[None, :, None].expand_as(token)
    k = _rows(s["view"][:, 0], (page, token % P, head)).float() * s["scales"][0]                            # [R, H, n, D]
    v = _rows(s["view"][:, 1], (page, token % P, head)).float().masked_fill(~seen[..., None], 0.0) * s["scales"][1]
    q = s["q"].float().unflatten(1, (H, G))
    out, lse = _softmax(q @ k.transpose(-1, -2) * s["scale"], seen[:, :, None, :], v)
    return [best.to(torch.int32), out.flatten(1, 2).to(s["q"].dtype), lse.flatten(1, 2)]


# ------------------------------------------------------------------------ the library's entry points

def _handle(s):
    """What a program builds once for a cache and keeps: the descriptors and a workspace."""
    from paper_2607_28633_b200 import binding as tk
    c, kind = s["case"], s["case"]["kind"]
    types = {"bf16": tk.TOPKV_TYPE_BF16, "fp16": tk.TOPKV_TYPE_FP16, "e4m3": tk.TOPKV_TYPE_E4M3}
    F, e = c.get("F", 2), 1 if c["type"] == "e4m3" else 2
    N = s["pages"] if kind == "plan" else s["view"].shape[0]
    lo = tk.make_layout(1, F, c["H"], c["D"], e, c["P"], N)
    if kind != "plan":
        lo.pool_page_stride, lo.pool_kv_stride, lo.pool_token_stride, lo.pool_head_stride = (x * e for x in s["view"].stride()[:4])
        lo.pool_layer_stride = N * lo.pool_page_stride
    h = dict(tk=tk, lo=lo, batch=tk.make_batch(s["block_table"], s["seq_lens"], window_tokens=c.get("window", 0)))
    if kind == "append":
        rotary = None
        if c["count"]:
            turns = torch.from_numpy(tk.topkv_rotary_turns(s["frequencies"]).view(np.int64)).cuda()
            rotary = tk.make_rotary(turns, tk.TOPKV_ROTARY_PAIRS if c["pairs"] else tk.TOPKV_ROTARY_HALVES, c["first"], s["turn"])
        # decode steps of one token a request need no offsets
        h["new"] = tk.make_new_tokens(s["k"], s["v"], types[c["type"]], types[c["io"]], q=s["q"], q_out=s["q_out"], rotary=rotary,
                                      cu_tokens=None if s["one"] else s["cu"], positions=s["positions"],
                                      k_scale=s["scales"][0], v_scale=s["scales"][1])
    elif kind in ("shared", "sparse"):
        h["att"] = tk.make_attention(s["q"], s["out"], types[c["type"]], types[c["io"]], s["scale"], k_scale=s["scales"][0], v_scale=s["scales"][1],
                                     lse=s["lse"])
    if kind == "shared":
        n = tk.check(tk.topkv_attend_shared_workspace_bytes(lo, h["batch"], h["att"]))
    elif kind == "sparse":
        h["pick"] = tk.make_page_choice(c["budget"], c["firsts"], c["lasts"], s["bounds"], s["steps"], s["picked"])
        n = tk.check(tk.topkv_page_choice_workspace_bytes(lo, h["batch"], h["att"], h["pick"]))
    else:
        return h
    h["ws"] = torch.empty(max(n, 16), dtype=torch.uint8, device="cuda")
    return h


def _own(s):
    h = s.get("handle")
    if h is None:
        h = s["handle"] = _handle(s)
    tk, lo, batch, kind = h["tk"], h["lo"], h["batch"], s["case"]["kind"]
    stream = torch.cuda.current_stream().cuda_stream
    if kind == "append":
        tk.check(tk.topkv_append_layer(0, s["flat"], lo, batch, h["new"], s["k"], s["v"], s["q"], s["q_out"], stream))
        return [s["q_out"], s["flat"]]
    if kind == "plan":
        tk.check(tk.topkv_plan_prefixes(lo, batch, 0, s["plan"], stream))
        return [s["plan"]]
    if kind == "bounds":
        tk.check(tk.topkv_bound_pages_layer(0, s["flat"], lo, batch, tk.TOPKV_TYPE_E4M3 if s["case"]["type"] == "e4m3" else
                                            tk.TOPKV_TYPE_BF16 if s["case"]["type"] == "bf16" else tk.TOPKV_TYPE_FP16, s["bounds"], s["steps"], stream))
        return [s["bounds"], s["steps"]]
    if kind == "shared":  # a plan serves all layers of a turn: a turn of one layer, which reads the table that it is given
        tk.check(tk.topkv_plan_prefixes(lo, batch, 0, s["plan"], stream))
        tk.check(tk.topkv_attend_shared_layer(0, s["flat"], lo, batch, h["att"], s["plan"], s["q"], s["out"], h["ws"], h["ws"].numel(), stream))
        return [s["out"], s["lse"]]
    tk.check(tk.topkv_choose_pages_layer(lo, batch, h["att"], h["pick"], s["q"], h["ws"], h["ws"].numel(), stream))
    tk.check(tk.topkv_attend_pages_layer(0, s["flat"], lo, batch, h["att"], h["pick"], s["q"], s["out"], h["ws"], h["ws"].numel(), stream))
    return [s["picked"], s["out"], s["lse"]]


def run(state):
    if own:
        return _own(state)
    return {"append": _plain_append, "plan": _plain_plan, "shared": _plain_shared, "bounds": _plain_bounds, "sparse": _plain_sparse}[state["case"]["kind"]](state)


# ----------------------------------------------------------------------------------- the bounds

def work(case):
    """Each input read once, each output written once; lengths of one seed stand for the case's."""
    c = case
    kind, H, G, D, P = c["kind"], c["H"], c["G"], c["D"], c["P"]
    e, Hq = 1 if c["type"] == "e4m3" else 2, H * G
    if kind == "append":
        sl, new, _ = _append_lengths(c, 0)
        T, kv = int(new[sl > 0].sum()), c["F"] * H * D
        return {"bytes": T * (kv * (2 + e) + Hq * D * 4 + 12) + 1, "flops": T * 3 * c["count"] * (H + Hq)}
    if kind in ("plan", "shared"):
        sl, rows, prefix, _ = _groups(c, 0)
        once = sum(max(min(n * P, int(sl[m].max())), 0) for m, n in zip(rows, prefix))  # tokens of the shared pages
        rest = sum(int(np.maximum(sl[m] - n * P, 0).sum()) for m, n in zip(rows, prefix))
        entries = 4 * (int((-(-sl // P)).sum()) + len(sl))
        if kind == "plan":
            return {"bytes": entries + 24 * len(sl), "flops": 0}
        return {"bytes": (once + rest) * 2 * H * D * e + len(sl) * Hq * (4 * D + 4) + entries, "flops": 4 * int(sl.sum()) * Hq * D}
    sl, _ = _sparse_lengths(c, 0)
    pages = -(-sl // P)
    if kind == "bounds":
        n, p = (sl, pages) if c["window"] == 0 else (np.minimum(sl, -(-c["window"] // P) * P), np.minimum(pages, -(-c["window"] // P)))
        return {"bytes": int(n.sum()) * H * D * e + int(p.sum()) * (H * (2 * D + 4) + 4), "flops": 0}
    seen = np.minimum(pages, c["budget"])
    tokens = np.minimum(sl, seen * P)
    return {"bytes": int(pages.sum()) * (H * (2 * D + 4) + 4) + int(tokens.sum()) * 2 * H * D * e + c["R"] * Hq * (4 * D + 4) + c["R"] * H * c["budget"] * 4,
            "flops": 4 * int(pages.sum()) * Hq * D + 4 * int(tokens.sum()) * Hq * D}


def _exact_append(c, s):
    q_out, pool = s["q_out"].double(), s["flat"].double()
    view = torch.as_strided(pool, s["view"].shape, s["view"].stride())
    lens, cu, bt, P = s["seq_lens"].tolist(), s["cu"].tolist(), s["block_table"].long(), c["P"]
    w, n, first = torch.from_numpy(s["frequencies"]).cuda(), c["count"], c["first"]
    one, two = (torch.arange(0, n, 2), torch.arange(1, n, 2)) if c["pairs"] else (torch.arange(n // 2), torch.arange(n // 2, n))
    one, two = one.cuda() + first, two.cuda() + first

    def turn(x, angle):
        x = x.double().clone()
        z = torch.polar(torch.full_like(angle, s["turn"]), angle)[:, None, :] * torch.complex(x[..., one], x[..., two])
        x[..., one], x[..., two] = z.real, z.imag
        return x

    for r, length in enumerate(lens):
        rows = torch.arange(cu[r], cu[r + 1], device="cuda")
        if length == 0 or len(rows) == 0:
            continue
        i = torch.arange(length - len(rows), length, device="cuda")
        angle = (i + c["far"]).double()[:, None] * w
        q_out[rows] = turn(s["q"][rows], angle)
        for plane, x in enumerate((turn(s["k"][rows], angle), None if s["v"] is None else s["v"][rows].double())):
            if x is not None:
                x = x / s["scales"][plane]
                view[bt[r, i // P], plane, i % P] = x.clamp(-448, 448) if c["type"] == "e4m3" else x
    return [q_out, pool]


def _exact_steps(c, s):
    steps, P = s["steps"].double(), c["P"]
    for r, n in enumerate(s["seq_lens"].tolist()):
        for j in () if n == 0 else range(max(n - c["window"], 0) // P if c["window"] else 0, -(-n // P)):
            page = s["block_table"][r, j].long()
            keys = s["view"][page, 0, :min(P, n - j * P)]
            steps[page] = keys.double().abs().amax((0, 2)) / 127
    return steps


def _exact_softmax(q, k, v, scale):
    score = q.double() @ k.double().T * scale
    return torch.softmax(score, 1) @ v.double(), torch.logsumexp(score, 1)


def exact(case, seed):
    """One request at a time in 64 bits, from the definitions. A plan has no computed
    values; which pages are seen is decided by whole numbers and two roundings to 32 bits."""
    c = case
    if c["kind"] == "plan":
        return None
    s = prepare(c, seed)
    if c["kind"] == "bounds":
        return [None, _exact_steps(c, s)]
    if c["kind"] == "append":
        return _exact_append(c, s)
    lens, bt, P, G = s["seq_lens"].tolist(), s["block_table"].long(), c["P"], c["G"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    for r, n in enumerate(lens):
        pages = -(-n // P)
        for h in range(c["H"] if n else 0):
            rows = slice(h * G, (h + 1) * G)
            i = torch.arange(n, device="cuda")
            if c["kind"] == "sparse":
                q = s["q"][r, rows].double()
                step = (q.abs().amax(1).float() * torch.tensor(_127TH, device="cuda"))
                q8 = torch.round((q.float() / step[:, None]).double())
                low, high = s["bounds"][bt[r, :pages], h].double().unbind(1)
                dot = torch.maximum(q8[:, None, :] * low, q8[:, None, :] * high).sum(-1) if pages * G * c["D"] < 1 << 28 else q8.clamp(max=0) @ low.T + q8.clamp(min=0) @ high.T
                score = (dot.float() * (step[:, None] * s["steps"][bt[r, :pages], h])).amax(0).tolist()
                firsts, lasts = set(range(min(c["firsts"], pages))), set(range(max(pages - c["lasts"], 0), pages))
                rank = sorted(range(pages), key=lambda j: (0, -j) if j in lasts else (1, j) if j in firsts else (2, -score[j], j))
                keep = torch.zeros(pages, dtype=torch.bool)
                keep[rank[:c["budget"]]] = True
                i = i[keep.cuda()[i // P]]
            where = (bt[r, i // P], i % P)
            k, v = (_rows(s["view"][:, f, :, h], where).double() * s["scales"][f] for f in (0, 1))
            out[r, rows], lse[r, rows] = _exact_softmax(s["q"][r, rows], k, v, s["scale"])
    return [None, out, lse] if c["kind"] == "sparse" else [out, lse]

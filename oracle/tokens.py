"""Calls around the decode side's attention written out from their definitions, in 64 bits or as plain
loops over host lists: rotated new tokens, shared prefixes, chosen pages. Test infrastructure like the rest
of this package; shares nothing with the library."""
from __future__ import annotations

import numpy as np

from . import Geom
from .decode import ERR_TABLE, HALF_STEP, decode_elements, row_offset, rows_of


# ---- rotated new tokens -----------------------------------------------------------------------------

def frequencies(count: int, base: float, kind: str = "none", factor: float = 1.0, original: float = 0.0,
                slow: float = 0.0, fast: float = 0.0) -> np.ndarray:
    out = []
    for j in range(count // 2):
        if kind == "base":
            f = (base * factor ** (count / (count - 2))) ** (-2 * j / count)
        else:
            f = base ** (-2 * j / count)
        if kind == "linear":
            f = f / factor
        if kind == "ramp":
            turns = original * f / (2 * np.pi)
            g = min(max((turns - slow) / (fast - slow), 0.0), 1.0)
            f = (1 - g) * f / factor + g * f
        out.append(f)
    return np.array(out)


def rotate(x: np.ndarray, position: int, freq: np.ndarray, first: int, pairs: bool, scale: float):
    """x [..., D] in 64 bits; returns the rotated vectors and, per element, |x| + |y| of its pair (0 outside
    the rotated part), which the error of the cosines is multiplied by."""
    y, size = np.array(x, np.float64), np.zeros_like(x)
    n = 2 * len(freq)
    for j, f in enumerate(freq):
        a, b = (first + 2 * j, first + 2 * j + 1) if pairs else (first + j, first + j + n // 2)
        c, s = np.cos(position * f) * scale, np.sin(position * f) * scale
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
        size[..., a] = size[..., b] = (np.abs(x[..., a]) + np.abs(x[..., b])) * abs(scale)
    return y, size


def stored_step(kind: str) -> tuple[float, float]:
    """Half a step of one rounding to `kind`, relative, and absolute below the normal numbers."""
    return HALF_STEP[kind], {"bf16": 2.0 ** -133, "fp16": 2.0 ** -25, "e4m3": 2.0 ** -10}[kind]


def places(P: int, num_pages: int, bt, sl, cu, num_rows: int):
    """For every row: (request, token, page, slot) or None, and the error bits."""
    R, maxp = bt.shape
    out, err = [None] * num_rows, 0
    for r in range(R):
        begin, end = (r, r + 1) if cu is None else (int(cu[r]), int(cu[r + 1]))
        s = int(sl[r])
        for t in range(begin, min(end, num_rows)):
            i = s - (end - t)
            if s == 0:
                continue
            if s < 0 or s > maxp * P or i < 0 or not 0 <= bt[r, i // P] < num_pages:
                err |= ERR_TABLE
                continue
            out[t] = (r, i, int(bt[r, i // P]), i % P)
    return out, err


def append(g: Geom, layer: int, bt, sl, cu, k, v, q, positions, freq, first, pairs, scale, k_scale, v_scale, kind: str, io: str):
    """Yields (pool offset or None, row of q, head, expected [D], tolerance [D]): what each written vector
    holds. k, v, q [rows][heads][D] in 64 bits.

    A cosine in 32 bits is off by the rounding of its angle, up to pi 2^-24, and 2 units of 2^-23; the two
    products and their sum by 2^-24 each, the division of a stored element by two more roundings: 2^-21 of
    |x| + |y| holds them all. The result is rounded once."""
    rows = len(k)
    where, err = places(g.P, g.num_pages, bt, sl, cu, rows)
    found = []
    for t, at in enumerate(where):
        if at is None:
            continue
        r, i, page, slot = at
        pos = i if positions is None else int(positions[t])
        for what, x, s in (("q", q, 1.0), ("k", k, k_scale), ("v", v, v_scale)):
            if x is None:
                continue
            y, size = rotate(x[t], pos, freq, first, pairs, scale) if what != "v" else (x[t], np.zeros_like(x[t]))
            size = np.where(size == 0, np.abs(x[t]) if s != 1.0 else 0.0, size)
            to = io if what == "q" else kind
            rel, least = stored_step(to)
            for h in range(x.shape[1]):
                e = 2.0 ** -21 * size[h] / abs(s)
                want = y[h] / s
                if to == "e4m3":
                    want = want.clip(-448, 448)
                off = None if what == "q" else row_offset(g, layer, page, 0 if what == "k" else 1, slot, h)
                found.append((off, t, h, want, e + rel * (np.abs(want) + e) + least))
    return found, err


# ---- shared prefixes ----------------------------------------------------------------------------------

def plan_prefixes(P: int, num_pages: int, bt, sl, min_tokens: int = 0) -> np.ndarray:
    """int32 [6][R]: leader, common, shared, members, order, place."""
    R, maxp = bt.shape
    full = [min(max(int(s), 0) // P, maxp) for s in sl]
    leader, common = [], []
    for r in range(R):
        lead = r
        if full[r] and 0 <= bt[r, 0] < num_pages:
            lead = next(x for x in range(r + 1) if full[x] and bt[x, 0] == bt[r, 0])
        n = 0
        while n < min(full[r], full[lead]) and bt[r, n] == bt[lead, n]:
            n += 1
        leader.append(lead)
        common.append(n * P)
    members = [leader.count(x) for x in leader]
    shared = [min(c for c, x in zip(common, leader) if x == leader[r]) for r in range(R)]
    shared = [s if m > 1 and s >= min_tokens else 0 for s, m in zip(shared, members)]
    order = sorted(range(R), key=lambda r: (leader[r], r))
    place = [order.index(r) for r in range(R)]
    return np.array([leader, common, shared, members, order, place], np.int32).reshape(6, R)


# ---- chosen pages ---------------------------------------------------------------------------------------
# Every operation below is one rounding to 32 bits, as the definition says, so the results are exact.

C127 = np.float32(1) / np.float32(127)


def bound_pages(g: Geom, layer: int, pool: np.ndarray, bt, sl, window: int, kind: str, bounds: np.ndarray, steps: np.ndarray) -> int:
    """Writes int8 bounds [pages][H][2][D] and float32 steps [pages][H]; returns error bits."""
    err = 0
    R, maxp = bt.shape
    for r in range(R):
        s = int(sl[r])
        if not 0 <= s <= maxp * g.P:
            err, s = err | ERR_TABLE, min(max(s, 0), maxp * g.P)
        for j in range(max(s - window, 0) // g.P if window else 0, -(-s // g.P)):
            page = int(bt[r, j])
            if not 0 <= page < g.num_pages:
                err |= ERR_TABLE
                continue
            tok = np.arange(j * g.P, min(s, (j + 1) * g.P))
            for h in range(g.h_kv):
                k = rows_of(g, layer, pool, bt[r], tok, 0, h, kind).astype(np.float32)
                step = (np.nan if np.isnan(k).any() else np.abs(k).max()) * C127
                steps[page, h] = step
                if not (step > 0 and np.isfinite(step)):
                    bounds[page, h] = 0
                    continue
                bounds[page, h, 0] = np.clip(np.floor(k.min(0) / step), -127, 127)
                bounds[page, h, 1] = np.clip(np.ceil(k.max(0) / step), -127, 127)
    return err


def choose_pages(P: int, bt, sl, q: np.ndarray, H: int, bounds, steps, budget: int, firsts: int, lasts: int) -> np.ndarray:
    """int32 [R][H][budget]."""
    R, maxp = bt.shape
    G = q.shape[1] // H
    out = np.full((R, H, budget), -1, np.int32)
    for r in range(R):
        pages = -(-min(max(int(sl[r]), 0), maxp * P) // P)
        for h in range(H):
            score = np.full(pages, -np.inf, np.float32)
            for a in range(h * G, (h + 1) * G):
                x = q[r, a].astype(np.float32)
                t = np.abs(x).max() * C127
                if not (t > 0 and np.isfinite(t)):
                    t, q8 = np.float32(0), np.zeros(len(x), np.int64)
                else:
                    q8 = np.clip(np.rint(x / t), -127, 127).astype(np.int64)
                ids = np.clip(bt[r, :pages], 0, len(steps) - 1)
                b = bounds[ids, h].astype(np.int64)                              # [pages][2][D]
                dot = (np.minimum(q8, 0) * b[:, 0] + np.maximum(q8, 0) * b[:, 1]).sum(1)
                with np.errstate(all="ignore"):
                    by = np.minimum(t * steps[ids, h], np.finfo(np.float32).max)
                    one = dot.astype(np.float32) * by
                    score = np.maximum(score, np.where(np.isfinite(steps[ids, h]), one, np.float32(np.inf)))
            last = range(max(pages - lasts, 0), pages)
            rank = sorted(range(pages), key=lambda j: (0, -j) if j in last else (1, j) if j < firsts else (2, -score[j], j))
            best = sorted(rank[:budget])
            out[r, h, :len(best)] = best
    return out


def of_chosen(P: int, bt_row, s: int, columns) -> tuple[np.ndarray, int]:
    """The table row and length of a request that has the chosen pages alone."""
    columns = [j for j in columns if j >= 0]
    pages = -(-s // P)
    n = (len(columns) - 1) * P + s - (pages - 1) * P if columns else 0
    return np.array([bt_row[j] for j in columns] or [-1], np.int32), n

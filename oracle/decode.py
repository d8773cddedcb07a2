"""The decode side's operators written out from their definitions: attention of one new token over
a paged cache in 64 bits, and the page operators as plain loops over host lists. Test
infrastructure like the rest of this package; shares nothing with the library."""
from __future__ import annotations

import numpy as np

from . import Geom


def _e4m3_table() -> np.ndarray:
    """Value of every 8-bit pattern: sign, 4 exponent bits (bias 7), 3 mantissa bits; no infinities,
    all ones is NaN."""
    v = np.empty(256)
    for b in range(256):
        e, f = (b >> 3) & 15, b & 7
        x = np.nan if (b & 127) == 127 else (f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7))
        v[b] = -x if b & 128 else x
    return v


E4M3 = _e4m3_table()
HALF_STEP = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11, "e4m3": 2.0 ** -4}   # relative, of one rounding


def decode_elements(raw: np.ndarray, kind: str) -> np.ndarray:
    """float64 values of a flat uint8 buffer."""
    if kind == "e4m3":
        return E4M3[raw]
    if kind == "fp16":
        return raw.view(np.float16).astype(np.float64)
    return (raw.view(np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def encode_elements(x: np.ndarray, kind: str) -> np.ndarray:
    """Nearest representable values (ties to even) as a uint8 buffer."""
    if kind == "e4m3":
        grid = E4M3[:127]                                       # 0 .. 448, ascending
        mag = np.minimum(np.abs(x), 448.0)
        hi = np.searchsorted(grid, mag).clip(1, 126)
        lo = hi - 1
        up = (grid[hi] - mag < mag - grid[lo]) | ((grid[hi] - mag == mag - grid[lo]) & (hi % 2 == 0))
        return (np.where(up, hi, lo) | np.where(np.signbit(x), 128, 0)).astype(np.uint8)
    if kind == "fp16":
        return x.astype(np.float16).view(np.uint8)
    u = x.astype(np.float32).view(np.uint32)
    return ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16).view(np.uint8)


def visible(s: int, window: int = 0, sinks: int = 0) -> np.ndarray:
    """Token numbers that the new token sees."""
    return np.array([i for i in range(s) if window == 0 or i >= s - window or i < sinks], dtype=np.int64)


def row_offset(g: Geom, layer: int, page: int, plane: int, t: int, head: int) -> int:
    return layer * g.S_layer + page * g.S_page + plane * g.S_kv + t * g.S_tok + head * g.S_head


def rows_of(g: Geom, layer: int, pool: np.ndarray, bt_row: np.ndarray, tokens: np.ndarray, plane: int, head: int,
            kind: str) -> np.ndarray:
    """float64 [tokens][d_h]."""
    n = g.d_h * g.b_p
    out = np.empty((len(tokens), n), dtype=np.uint8)
    for k, i in enumerate(tokens):
        a = row_offset(g, layer, int(bt_row[i // g.P]), plane, int(i % g.P), head)
        out[k] = pool[a:a + n]
    return decode_elements(out.reshape(-1), kind).reshape(len(tokens), g.d_h)


def attend(g: Geom, layer: int, pool: np.ndarray, bt, sl, q: np.ndarray, kind: str, io: str, scale: float,
           value_dim: int = 0, sinks: int = 0, k_scale: float = 1.0, v_scale: float = 1.0,
           weight_step: float | None = None):
    """q float64 [R][Hq][d_h] (values of type io). Returns out and lse in 64 bits, and a bound on how
    far a computation may be off that keeps scores and sums in 32 bits, rounds each weight once to
    16 bits (fp16 where the cache is not bf16) and the result once to ``io``:

    a dot product of n terms in 32 bits is off by at most n 2^-23 sum |terms| (2^-23, not 2^-24: the
    matrix units may cut instead of round), the scaled score by as much plus two roundings, so the
    weights by the factor e = that, in their sum as in the product with V; the sums over t tokens are
    off by t 2^-23 sum |terms|; a weight's rounding is u |w|, the result's half a step of io.
    exp and the power of two it is computed by add 2^-20 to a weight's factor. ``weight_step``: the
    relative rounding of a weight, if it is not that of one 16-bit value."""
    R, Hq, _ = q.shape
    H = g.h_kv
    G = Hq // H
    dv = value_dim if g.F == 1 else g.d_h
    out = np.zeros((R, Hq, dv))
    lse = np.full((R, Hq), -np.inf)
    tol_out, tol_lse = np.zeros_like(out), np.zeros_like(lse)
    u = HALF_STEP["bf16" if kind == "bf16" else "fp16"] if weight_step is None else weight_step
    ep = 2.0 ** -23
    for r in range(R):
        tok = visible(int(sl[r]), g.window, sinks)
        if len(tok) == 0:
            continue
        for h in range(H):
            k = rows_of(g, layer, pool, bt[r], tok, 0, h, kind) * k_scale
            v = k[:, :dv] if g.F == 1 else rows_of(g, layer, pool, bt[r], tok, 1, h, kind) * v_scale
            for a in range(h * G, (h + 1) * G):
                x = scale * (k @ q[r, a])
                m = x.max()
                w = np.exp(x - m)
                l = w.sum()
                out[r, a] = w @ v / l
                lse[r, a] = m + np.log(l)
                e = ((g.d_h + 4) * ep * abs(scale) * (np.abs(k) @ np.abs(q[r, a])).max() + 4 * ep * np.abs(x).max()
                     + 2.0 ** -20)
                spread = w @ np.abs(v) / l
                n = len(tok) + 64
                tol_out[r, a] = (HALF_STEP[io] * np.abs(out[r, a]) + (u + 2 * e + 2 * n * ep) * spread * 1.01
                                 + (2.0 ** -24 if io == "fp16" else 2.0 ** -133))   # below the smallest normal number
                tol_lse[r, a] = 2 * e + n * ep + 4 * ep * abs(lse[r, a])
    return out, lse, tol_out, tol_lse


# ---- page operators ---------------------------------------------------------------------------------
# Tables are numpy int32 arrays, changed in place; every function returns the error bits it raises.

ERR_TABLE, ERR_PAGES = 2, 8


def _pages(n: int, P: int) -> int:
    return -(-n // P)


def free_requests(P: int, bt, sl, ref, rows) -> int:
    err = 0
    R, maxp = bt.shape
    for r in rows:
        if not 0 <= r < R:
            err |= ERR_TABLE
            continue
        n, sl[r] = int(sl[r]), 0
        if n <= 0:
            err |= ERR_TABLE if n < 0 else 0
            continue
        if _pages(n, P) > maxp:
            err |= ERR_TABLE
        for p in bt[r, :min(_pages(n, P), maxp)]:
            if not 0 <= p < len(ref) or ref[p] <= 0:
                err |= ERR_TABLE
            else:
                ref[p] -= 1
        bt[r] = -1
    return err


def extend_requests(P: int, bt, sl, ref, new) -> int:
    err = 0
    R, maxp = bt.shape
    free = [p for p in range(len(ref)) if ref[p] <= 0]
    wanted = 0
    for r in range(R):
        n, k = int(sl[r]), int(new[r])
        if n < 0 or k < 0 or n + k > maxp * P:
            err |= ERR_TABLE
            continue
        need = _pages(n + k, P) - _pages(n, P)
        first, wanted = wanted, wanted + need
        if need and wanted > len(free):
            err |= ERR_PAGES
            continue
        for j in range(need):
            bt[r, _pages(n, P) + j] = free[first + j]
            ref[free[first + j]] = 1
        sl[r] = n + k
    return err


def fork_requests(g: Geom, pool, bt, sl, ref, parents, children) -> int:
    err = 0
    R, maxp = bt.shape
    bt0, sl0 = bt.copy(), sl.copy()
    free = [p for p in range(len(ref)) if ref[p] <= 0]
    seen, jobs = set(), []
    for a, c in zip(parents, children):
        a, c = int(a), int(c)
        first = c not in seen
        seen.add(c)
        ok = 0 <= a < R and 0 <= c < R and a != c and first and sl0[c] == 0 and 0 <= sl0[a] <= maxp * g.P
        if ok and sl0[a] % g.P:
            ok = 0 <= bt0[a, sl0[a] // g.P] < len(ref)
        if not ok:
            err |= ERR_TABLE
            continue
        jobs.append((a, c))
    rank = 0
    for a, c in jobs:
        n = int(sl0[a])
        full, tail = divmod(n, g.P)
        if tail:
            rank += 1
            if rank > len(free):
                err |= ERR_PAGES
                continue
        bt[c] = -1
        for j in range(full):
            bt[c, j] = bt0[a, j]
            if 0 <= bt0[a, j] < len(ref):
                ref[bt0[a, j]] += 1
            else:
                err |= ERR_TABLE
        if tail:
            p = free[rank - 1]
            bt[c, full], ref[p] = p, 1
            for layer in range(g.L):
                _move(g, pool, layer, int(bt0[a, full]), p, tail)
        sl[c] = n
    return err


def _move(g: Geom, pool, layer: int, src: int, dst: int, tokens: int):
    n = g.d_h * g.b_p
    for c in range(g.F):
        for t in range(tokens):
            for h in range(g.h_kv):
                a, b = row_offset(g, layer, src, c, t, h), row_offset(g, layer, dst, c, t, h)
                pool[b:b + n] = pool[a:a + n]


def copy_pages(g: Geom, pool, first_layer: int, num_layers: int, src, dst) -> int:
    err = 0
    for a, b in zip(src, dst):
        if not (0 <= a < g.num_pages and 0 <= b < g.num_pages):
            err |= ERR_TABLE
            continue
        for layer in range(first_layer, first_layer + num_layers):
            _move(g, pool, layer, int(a), int(b), g.P)
    return err


def compact_pages(g: Geom, pool, bt, sl, ref):
    """Returns (error bits, pages in use, map)."""
    err = 0
    R, maxp = bt.shape
    used = [p for p in range(len(ref)) if ref[p] > 0]
    n = len(used)
    holes = [p for p in range(n) if ref[p] <= 0]
    movers = [p for p in used if p >= n]
    to = np.full(len(ref), -1, np.int32)
    for p in used:
        to[p] = p
    for a, b in zip(movers, holes):
        to[a] = b
        for layer in range(g.L):
            _move(g, pool, layer, a, b, g.P)
        ref[b], ref[a] = ref[a], 0
    for r in range(R):
        if not 0 <= sl[r] <= maxp * g.P:
            err |= ERR_TABLE
        for j in range(min(_pages(max(int(sl[r]), 0), g.P), maxp)):
            p = bt[r, j]
            if not 0 <= p < len(ref) or to[p] < 0:
                err |= ERR_TABLE
            else:
                bt[r, j] = to[p]
    return err, n, to

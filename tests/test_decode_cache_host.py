"""session.DecodeCache on the CPU: the library's kernels are replaced by the oracle's loops, which work
on the memory that the calls name, so that what the class itself does (order, descriptors, offsets,
workspaces, refusals) is followed without a GPU."""
import contextlib
import ctypes
import gc
import weakref

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import __graft_entry__ as entry
from oracle import Geom, decode as od
from paper_2607_28633_b200 import binding as tk
from paper_2607_28633_b200 import session


def _at(addr, shape, dtype):
    """The array at an address that a descriptor names."""
    n = int(np.prod(shape)) * np.dtype(dtype).itemsize
    return np.frombuffer((ctypes.c_uint8 * n).from_address(addr), dtype=dtype).reshape(shape)


class _Library:
    """What the calls do, from the descriptors alone; error bits are gathered in `err`."""

    def __init__(self, g):
        self.g, self.err = g, 0

    def _tables(self, b, t):
        bt = _at(t.block_table_out, (b.num_requests, b.max_pages_per_req), np.int32)
        return bt, _at(t.seq_lens_out, (b.num_requests,), np.int32), _at(t.ref_counts_out, (self.g.num_pages,), np.int32)

    def extend(self, lo, b, t, new, ws, n, stream=None):
        self.err |= od.extend_requests(self.g.P, *self._tables(b, t), new.numpy())
        return 0

    def free(self, lo, b, t, rows, n, stream=None):
        self.err |= od.free_requests(self.g.P, *self._tables(b, t), rows.numpy()[:n])
        return 0

    def fork(self, pool, lo, b, t, parents, children, n, ws, nbytes, stream=None):
        self.err |= od.fork_requests(self.g, pool.numpy(), *self._tables(b, t), parents.numpy()[:n], children.numpy()[:n])
        return 0

    def plan(self, b, cu, stream=None):
        sl = _at(b.seq_lens, (b.num_requests,), np.int32).astype(np.int64)
        kept = np.minimum(sl, b.window_tokens) if b.window_tokens else sl
        _at(cu.data_ptr(), (b.num_requests + 1,), np.int64)[:] = np.concatenate([[0], np.cumsum(kept)])
        return 0

    def unpack(self, layer, pool, lo, b, wire, nbytes, stream=None):
        """The last window_tokens tokens of every request, from the wire rows that its prefix names."""
        g, R, W = self.g, b.num_requests, b.window_tokens
        if R > 1024 and not b.cu_seq_lens:
            return tk.TOPKV_ERR_INVALID_ARG
        row = g.F * g.h_kv * g.d_h * g.b_p
        sl = _at(b.seq_lens, (R,), np.int32)
        bt = _at(b.block_table, (R, b.max_pages_per_req), np.int32)
        kept = np.minimum(sl, W)
        cu = _at(b.cu_seq_lens, (R + 1,), np.int64) if b.cu_seq_lens else np.concatenate([[0], np.cumsum(kept)])
        at = layer * lo.wire_layer_stride
        slab = _at(wire + at, (nbytes - at,), np.uint8)
        out, n = pool.numpy(), g.d_h * g.b_p
        for r in range(R):
            for k in range(kept[r]):
                i = int(sl[r] - kept[r]) + k
                assert 0 <= bt[r, i // g.P] < g.num_pages and (cu[r] + k + 1) * row <= len(slab)
                src = slab[(cu[r] + k) * row:][:row].reshape(g.F, g.h_kv, n)
                for c in range(g.F):
                    for h in range(g.h_kv):
                        a = od.row_offset(g, layer, int(bt[r, i // g.P]), c, i % g.P, h)
                        out[a:a + n] = src[c, h]
        return 0


@pytest.fixture(scope="module", autouse=True)
def _built():
    entry.build()
    if torch.cuda.is_available():
        pytest.skip("the class is tested with the real library there")


@pytest.fixture
def make(monkeypatch):
    """make(g, bt, sl, **kw) -> (cache, library)"""
    class Idle:
        def synchronize(self):
            pass
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: Idle())

    def build(g, bt, sl, **kw):
        lib = _Library(g)
        for name, fn in (("extend_requests", lib.extend), ("free_requests", lib.free), ("fork_requests", lib.fork),
                         ("unpack_layer", lib.unpack), ("build_plan", lib.plan)):
            monkeypatch.setattr(tk, f"topkv_{name}", fn)
        monkeypatch.setattr(session.DecodeCache, "_on", lambda self, stream: contextlib.nullcontext(), raising=False)
        lo = tk.make_layout(g.L, g.F, g.h_kv, g.d_h, g.b_p, g.P, g.num_pages, wire_layer_stride=64 * g.F * g.h_kv * g.d_h * g.b_p)
        pool = torch.zeros(g.pool_bytes(), dtype=torch.uint8)
        return session.DecodeCache(pool, lo, torch.tensor(bt, dtype=torch.int32), torch.tensor(sl, dtype=torch.int32), **kw), lib
    return build


def _ints(*x):
    return torch.tensor(x, dtype=torch.int32)


GEOM = dict(L=2, F=2, h_kv=1, d_h=8, b_p=2, P=4)
ROW = 32   # bytes of a token's K and V


def _slab(*marks):
    """A wire slab of one token row per mark, all bytes the mark."""
    return torch.tensor(marks, dtype=torch.uint8)[:, None].expand(len(marks), ROW).contiguous()


def _mark(g, cache, layer, row, token):
    """The byte that fills a token's K and V (checked to be the same throughout)."""
    page = int(cache.block_table[row, token // g.P])
    got = {int(x) for c in range(g.F) for x in cache.pool[od.row_offset(g, layer, page, c, token % g.P, 0):][:16]}
    assert len(got) == 1
    return got.pop()


def _filled(g, cache, marks):
    """Every token of row r holds marks[r], in all layers."""
    for layer in range(g.L):
        for r, m in enumerate(marks):
            for i in range(int(cache.seq_lens[r])):
                for c in range(g.F):
                    a = od.row_offset(g, layer, int(cache.block_table[r, i // g.P]), c, i % g.P, 0)
                    cache.pool[a:a + 16] = m


def test_append_leaves_a_refused_request_as_it_was(make):
    """Five pages, all but one taken: of two requests that need a page the second gets none. Its last
    cached token stays, and what follows it in the slab goes where it belongs."""
    g = Geom(num_pages=5, **GEOM)
    cache, lib = make(g, [[0, -1], [1, -1], [2, 3]], [4, 4, 6])
    _filled(g, cache, [11, 12, 13])
    cache.extend(_ints(1, 1, 1), None)
    assert cache.seq_lens.tolist() == [5, 4, 7] and lib.err == od.ERR_PAGES
    for layer in range(2):
        cache.append(layer, _slab(101, 102, 103), None)
        assert [_mark(g, cache, layer, *x) for x in ((0, 4), (0, 3), (1, 3), (2, 6), (2, 5))] == [101, 11, 12, 103, 13]


def test_append_of_several_tokens_keeps_the_places_of_refused_and_new_requests(make):
    """Row 1 is new (length 0) and refused, row 3 short: each takes the wire rows that it asked for."""
    g = Geom(num_pages=5, **GEOM)
    cache, lib = make(g, [[0, -1], [-1, -1], [1, -1], [2, 3]], [3, 0, 1, 6], rows=5)
    _filled(g, cache, [11, 0, 13, 14])
    cache.extend(_ints(2, 2, 2, 2, 0), None)                 # row 0 takes the last free page, rows 2 and 3 need none
    assert cache.seq_lens.tolist() == [5, 0, 3, 8, 0] and lib.err == od.ERR_PAGES
    cache.append(0, _slab(1, 2, 3, 4, 5, 6, 7, 8), None, tokens=2)
    assert [_mark(g, cache, 0, 0, i) for i in range(5)] == [11, 11, 11, 1, 2]
    assert [_mark(g, cache, 0, 2, i) for i in range(3)] == [13, 5, 6]
    assert [_mark(g, cache, 0, 3, i) for i in range(8)] == [14] * 6 + [7, 8]


def test_append_leaves_a_request_without_new_tokens_as_it_was(make):
    g = Geom(num_pages=8, **GEOM)
    cache, _ = make(g, [[0, -1], [1, -1], [2, 3]], [4, 3, 6])
    _filled(g, cache, [11, 12, 13])
    for turn in range(2):                                    # also in the second turn, when row 1 grew in the first
        cache.extend(_ints(1, 1 - turn, 1), None)
        for layer in range(2):
            cache.append(layer, _slab(101, 102, 103), None)
    assert _mark(g, cache, 1, 1, 3) == 102
    cache.extend(_ints(0, 0, 0), None)
    cache.append(0, _slab(201, 202, 203), None)
    assert [_mark(g, cache, 0, *x) for x in ((0, 5), (1, 3), (2, 7))] == [101, 102, 103]


def test_append_after_the_refused_request_got_its_page(make):
    """The way out of a refusal: another request is freed and the refused one asks again; what the first
    call gave to the others is still to be written."""
    g = Geom(num_pages=4, **GEOM)
    cache, lib = make(g, [[0, -1], [1, -1], [2, 3]], [3, 4, 6])
    _filled(g, cache, [11, 12, 13])
    cache.extend(_ints(1, 1, 1), None)
    assert cache.seq_lens.tolist() == [4, 4, 7]
    cache.free(_ints(2), None)
    cache.extend(_ints(0, 1, 0), None)
    assert cache.seq_lens.tolist() == [4, 5, 0]
    cache.append(0, _slab(101, 102), None)
    assert [_mark(g, cache, 0, *x) for x in ((0, 3), (0, 2), (1, 4), (1, 3))] == [101, 11, 102, 12]


def test_append_before_any_extend_writes_every_request(make):
    g = Geom(num_pages=6, **GEOM)
    cache, _ = make(g, [[0, -1], [-1, -1], [2, 3]], [4, 0, 6])
    cache.append(1, _slab(1, 2), None)
    assert (_mark(g, cache, 1, 0, 3), _mark(g, cache, 1, 2, 5)) == (1, 2)
    cache.fork(_ints(2), _ints(1), None)
    cache.append(1, _slab(3, 4, 5), None)
    assert [_mark(g, cache, 1, r, n - 1) for r, n in ((0, 4), (1, 6), (2, 6))] == [3, 4, 5]


@pytest.mark.parametrize("seed", range(40))
def test_random_turns(make, seed):
    """Extensions that are refused in part, frees and forks in any order between them, then the appends:
    a model in plain Python keeps every token's mark and says which are written."""
    rng = np.random.default_rng(seed)
    R, P, N = 6, 4, int(rng.integers(9, 20))
    g = Geom(num_pages=N, **GEOM)
    sl = rng.integers(0, 7, size=R)
    bt, pos = np.full((R, 6), -1), 0
    for r in range(R):
        k = -(-sl[r] // P)
        if pos + k > N:
            sl[r] = k = 0
        bt[r, :k] = np.arange(pos, pos + k)
        pos += k
    cache, lib = make(g, bt, sl, max_forks=3)
    marks = [[int(x) for x in rng.integers(1, 250, size=n)] for n in sl]        # of the tokens whose K/V are there
    for layer in range(2):
        for r in range(R):
            for i, m in enumerate(marks[r]):
                for c in range(2):
                    a = od.row_offset(g, layer, int(bt[r, i // P]), c, i % P, 0)
                    cache.pool[a:a + 16] = m
    for turn in range(6):
        asked = [len(m) for m in marks]                      # what the caller believes the lengths to be
        owing = [0] * R                                      # new tokens of each row
        whole = [True] * R                                   # the last wish of the row was met
        ops = rng.integers(0, 4, size=int(rng.integers(0, 4))).tolist()
        ops.insert(int(rng.integers(0, len(ops) + 1)), 0)    # a turn has one extension at least
        if rng.random() < 0.5:
            ops.append(-1)                                   # its last one asks for nothing: refusals are known
        for op in ops:
            before = cache.seq_lens.tolist()
            if op <= 1:
                new = rng.integers(0, 3, size=R) * (op >= 0)
                cache.extend(torch.tensor(new, dtype=torch.int32), None)
                now = cache.seq_lens.tolist()
                for r in range(R):
                    asked[r], whole[r] = before[r] + int(new[r]), now[r] == before[r] + new[r]
                    owing[r] += now[r] - before[r]
            elif op == 2:
                rows = [int(x) for x in rng.integers(-1, R + 1, size=2)]
                cache.free(_ints(*rows), None)
                for r in rows:
                    if 0 <= r < R:
                        marks[r], asked[r], owing[r], whole[r] = [], 0, 0, True
            else:
                parents, children = ([int(x) for x in rng.integers(0, R, size=2)] for _ in range(2))
                cache.fork(_ints(*parents), _ints(*children), None)
                now = cache.seq_lens.tolist()
                old = [(list(marks[r]), asked[r], owing[r], whole[r]) for r in range(R)]
                for a, c in reversed(list(zip(parents, children))):             # the first that names a row is done
                    if now[c] != before[c]:
                        marks[c], asked[c], owing[c], whole[c] = list(old[a][0]), *old[a][1:]
        now = cache.seq_lens.tolist()
        tokens = int(rng.integers(1, 4))
        place, at, slab = [], 0, []
        for r in range(R):
            k = min(asked[r], tokens)
            place.append(at)
            at += k
            slab += [int(x) for x in rng.integers(1, 250, size=k)]
        for r in range(R):
            have = marks[r] + [None] * (now[r] - len(marks[r]))
            if owing[r] > 0 and whole[r]:
                k = min(now[r], tokens)
                have[now[r] - k:] = slab[place[r]:place[r] + k]
            marks[r] = have
        for layer in range(2):
            cache.append(layer, _slab(*(slab or [0])), None, tokens=tokens)
        for r in range(R):
            shared = [i for i in range(now[r]) if int(cache.ref_counts[int(cache.block_table[r, i // P])]) > 1]
            for layer in range(2):
                for i, m in enumerate(marks[r]):
                    if m is not None and i not in shared:
                        assert _mark(g, cache, layer, r, i) == m, (turn, layer, r, i)
        # tokens that were never written, or whose page is shared with a row that rewrote it, are taken as they lie
        marks = [[_mark(g, cache, 0, r, i) for i in range(now[r])] for r in range(R)]
        for r in range(R):                                   # (one byte per token from here on, the same in both layers)
            for i, m in enumerate(marks[r]):
                for c in range(2):
                    a = od.row_offset(g, 1, int(cache.block_table[r, i // P]), c, i % P, 0)
                    cache.pool[a:a + 16] = m


def test_append_to_more_rows_than_a_copy_counts_itself(make):
    """1,025 rows, before an extension and after one."""
    g = Geom(num_pages=6, **GEOM)
    bt, sl = np.full((1025, 2), -1), np.zeros(1025, np.int64)
    bt[3, 0], bt[1024, 0], sl[3], sl[1024] = 4, 2, 2, 3
    cache, _ = make(g, bt, sl)
    cache.append(0, _slab(1, 2), None)
    assert (_mark(g, cache, 0, 3, 1), _mark(g, cache, 0, 1024, 2)) == (1, 2)
    new = torch.zeros(1025, dtype=torch.int32)
    new[1024] = new[7] = 1
    cache.extend(new, None)
    cache.append(0, _slab(3, 4, 5), None)
    assert [_mark(g, cache, 0, r, i) for r, i in ((3, 1), (7, 0), (1024, 2), (1024, 3))] == [1, 4, 2, 5]
    cache.free(_ints(3), None)
    cache.append(1, _slab(6, 7), None)
    assert (_mark(g, cache, 1, 7, 0), _mark(g, cache, 1, 1024, 3)) == (6, 7)


def _attend(cache, lib, monkeypatch, needs, stream=None):
    """Attends once per workspace size; returns the workspaces that the calls were given."""
    seen = []
    monkeypatch.setattr(tk, "topkv_attend_layer", lambda layer, pool, lo, b, att, q, out, ws, n, stream=None: seen.append((ws, n)) or 0)
    R = len(cache.seq_lens)
    for need in needs:
        monkeypatch.setattr(tk, "topkv_attend_workspace_bytes", lambda lo, b, att, need=need: need)
        cache.attend(0, torch.zeros(R, 2, 8, dtype=torch.bfloat16), torch.zeros(R, 2, 8, dtype=torch.bfloat16), 1.0, stream)
    return seen


def test_a_workspace_that_a_call_was_given_stays(make, monkeypatch):
    """A captured graph keeps the address: a later call that needs more must not give that memory back."""
    g = Geom(num_pages=6, **GEOM)
    cache, lib = make(g, [[0, -1], [2, 3]], [4, 6])
    seen = [(weakref.ref(ws), ws.data_ptr(), n) for ws, n in _attend(cache, lib, monkeypatch, [100, 5000, 100, 0, 5000])]
    gc.collect()
    assert all(ws() is not None and n >= need for (ws, _, n), need in zip(seen, [100, 5000, 100, 0, 5000]))
    assert seen[0][1] == seen[2][1] and seen[1][1] == seen[4][1]     # and is the same for the same need


@pytest.mark.parametrize("stream", [None, 0, 12345])
def test_attend_takes_any_kind_of_stream(make, monkeypatch, stream):
    """A handle, or none, as the other calls do."""
    g = Geom(num_pages=6, **GEOM)
    cache, lib = make(g, [[0, -1], [2, 3]], [4, 6])
    used = []
    monkeypatch.setattr(session.DecodeCache, "_on", lambda self, s: used.append(s) or contextlib.nullcontext())
    assert len(_attend(cache, lib, monkeypatch, [100], stream)) == 1 and used == [stream]


def test_tensors_that_do_not_fit_the_cache_are_refused(make, monkeypatch):
    """The library sees addresses only: too few rows, another type or order would be read past its end
    or as other numbers."""
    g = Geom(num_pages=6, **GEOM)
    cache, lib = make(g, [[0, -1], [2, 3], [-1, -1]], [4, 6, 0])
    calls = []
    for name in ("attend_layer", "extend_requests", "free_requests", "fork_requests", "unpack_layer"):
        monkeypatch.setattr(tk, f"topkv_{name}", lambda *a, name=name: calls.append(name) or 0)
    new = _ints(1, 1, 1)
    for bad in (new[:2], new.long(), new.short(), _ints(1, 1, 1, 1), new[:, None].expand(3, 2), _ints(1, 0, 1, 0, 1, 0)[::2],
                new.float(), torch.zeros(3, dtype=torch.int32, device="meta")):
        with pytest.raises(ValueError):
            cache.extend(bad, None)
    for bad in (new.long(), _ints(1, 0, 1, 0)[::2], new.view(3, 1), torch.zeros(2, dtype=torch.int32, device="meta")):
        with pytest.raises(ValueError):
            cache.free(bad, None)
        with pytest.raises(ValueError):
            cache.fork(bad, bad, None)
        with pytest.raises(ValueError):
            cache.fork(bad.reshape(-1)[:1].int() if bad.device.type == "cpu" else _ints(0), bad.reshape(-1)[:1].long(), None)
    for kv, tokens in ((_slab(1, 2)[:, ::2], 1), (_slab(1, 2), 0), (_slab(1, 2), -1), (torch.zeros(64, dtype=torch.uint8, device="meta"), 1)):
        with pytest.raises(ValueError):
            cache.append(0, kv, None, tokens=tokens)
    q = lambda *s, dt=torch.bfloat16, dev="cpu": torch.zeros(*s, dtype=dt, device=dev)
    for a, b in ((q(2, 2, 8), q(2, 2, 8)), (q(4, 2, 8), q(4, 2, 8)), (q(3, 2, 16), q(3, 2, 16)), (q(3, 2, 8), q(3, 2, 4)),
                 (q(3, 2, 8), q(3, 2, 8, dt=torch.float16)), (q(3, 2, 8, dt=torch.int16), q(3, 2, 8, dt=torch.int16)),
                 (q(3, 2, 8, dev="meta"), q(3, 2, 8, dev="meta")), (q(3, 2, 8), q(3, 2, 8)[..., :0])):
        with pytest.raises(ValueError):
            cache.attend(0, a, b, 1.0, None)
    assert calls == []
    cache.extend(new, None), cache.free(_ints(0), None), cache.fork(_ints(0), _ints(2), None), cache.append(0, _slab(1, 2), None)
    cache.attend(0, q(3, 2, 8), q(3, 2, 8), 1.0, None)
    assert calls == ["extend_requests", "free_requests", "fork_requests", "unpack_layer", "attend_layer"]


def test_make_attention_checks_types_and_sizes():
    q = torch.zeros(3, 8, 64, dtype=torch.bfloat16)
    T = tk.TOPKV_TYPE_BF16
    for out, kw in ((q.half(), {}), (q[..., :32], {}), (q[..., :32], dict(value_dim=48)),
                    (q.to("meta"), {}), (q, dict(lse=torch.zeros(3, 8, device="meta")))):
        with pytest.raises(ValueError):
            tk.make_attention(q, out, T, T, 1.0, **kw)
    tk.make_attention(q, q[..., :32], T, T, 1.0, value_dim=32)
    tk.make_attention(q, torch.zeros_like(q), T, T, 1.0, value_dim=32)          # the rest of a wider row is left alone


def test_more_forks_than_the_workspace_holds_are_refused(make):
    g = Geom(num_pages=6, **GEOM)
    cache, lib = make(g, [[0, -1], [-1, -1], [-1, -1], [-1, -1]], [4, 0, 0, 0], max_forks=2)
    for parents, children in ((_ints(0, 0, 0), _ints(1, 2, 3)), (_ints(0, 0), _ints(1))):
        with pytest.raises(ValueError):
            cache.fork(parents, children, None)
    assert cache.seq_lens.tolist() == [4, 0, 0, 0]
    cache.fork(_ints(), _ints(), None)
    cache.fork(_ints(0, 0), _ints(1, 3), None)
    assert cache.seq_lens.tolist() == [4, 4, 0, 4]

"""A run of the calls together, as a decode worker makes them: prompts written with their rotation, samples
forked from them, turns of single tokens, attention to shared prefixes and to chosen pages, rows freed, the pool
compacted; every step against the oracle on what the pool then holds."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import decode as od, tokens as ot
from paper_2607_28633_b200 import binding as tk
from paper_2607_28633_b200 import session
from test_gpu_decode import TORCH, TYPE, _check, _geom, _layout

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    import __graft_entry__ as entry
    entry.build()
    return torch.device("cuda:0")


@pytest.fixture(autouse=True)
def clean(dev):
    tk.check(tk.topkv_reset_device_error_flags())
    before = tk.topkv_set_sharing_bytes(0)
    yield
    tk.topkv_set_sharing_bytes(before)
    assert tk.topkv_device_error_flags() == 0


class Run:
    def __init__(self, dev, kind, io, D, pairs, rows=6, G=3, H=2, L=2, P=8, pages=96, max_pages=24):
        self.rng = np.random.default_rng(3)
        self.kind, self.io, self.dev, self.D, self.Hq, self.H, self.L, self.pairs = kind, io, dev, D, H * G, H, L, pairs
        self.g = _geom(2, H, D, 1 if kind == "e4m3" else 2, P, pages, L=L)
        self.lo = _layout(self.g)
        self.pool = torch.zeros(self.g.L * self.g.S_layer, dtype=torch.uint8, device=dev)
        self.scales = (0.5, 0.75) if kind == "e4m3" else (1.0, 1.0)
        self.freq = ot.frequencies(D // 2, 10000.0)
        turns = torch.from_numpy(tk.topkv_rotary_turns(self.freq).view(np.int64)).to(dev)
        self.rotary = tk.make_rotary(turns, tk.TOPKV_ROTARY_PAIRS if pairs else tk.TOPKV_ROTARY_HALVES, D // 2)
        bt = torch.full((rows, max_pages), -1, dtype=torch.int32, device=dev)
        self.stream = torch.cuda.Stream(dev)
        self.cache = session.DecodeCache(self.pool, self.lo, bt, torch.zeros(rows, dtype=torch.int32, device=dev))
        self.rows = rows
        self.since = [0] * L  # the most tokens that a request has got since a layer's bounds were formed

    def ints(self, x, t=torch.int32):
        x = torch.from_numpy(np.asarray(x)).to(self.dev).to(t)
        torch.cuda.synchronize()
        return x

    def turn(self, new, one=False):
        """Extends by new[r] tokens and writes them, in all layers; what is written is checked."""
        c, new = self.cache, np.asarray(new)
        self.since = [n + int(new.max()) for n in self.since]
        T = self.rows if one else int(new.sum())
        cu = None if one else np.concatenate([[0], np.cumsum(new)])
        c.extend(self.ints(new), self.stream)
        written = []
        for layer in range(self.L):
            x = od.decode_elements(od.encode_elements(self.rng.normal(size=T * (self.Hq + 2 * self.H) * self.D), self.io), self.io).reshape(T, -1, self.D)
            d = self.ints(x, TORCH[self.io])
            q, k, v = d[:, :self.Hq], d[:, self.Hq:self.Hq + self.H], d[:, self.Hq + self.H:]
            q_out = torch.zeros_like(q)
            torch.cuda.synchronize()
            c.append_rotated(layer, k, v, self.stream, self.rotary, q, q_out, None if cu is None else self.ints(cu, torch.int64),
                             cache_type=TYPE[self.kind], k_scale=self.scales[0], v_scale=self.scales[1])
            written.append((x, q_out))
        self.stream.synchronize()
        pool, bt, sl = self.pool.cpu().numpy(), c.block_table.cpu().numpy(), c.seq_lens.cpu().numpy()
        for layer, (x, q_out) in enumerate(written):
            lens = sl if cu is not None else np.where(new > 0, sl, 0)
            found, err = ot.append(self.g, layer, bt, lens, cu, x[:, self.Hq:self.Hq + self.H], x[:, self.Hq + self.H:], x[:, :self.Hq], None, self.freq,
                                   self.D // 2, self.pairs, 1.0, *self.scales, self.kind, self.io)
            assert err == 0
            got = q_out.double().cpu().numpy()
            for off, t, h, want, tol in found:
                have = got[t, h] if off is None else od.decode_elements(pool[off:off + self.D * self.g.b_p].copy(), self.kind)
                assert (np.abs(have - want) <= tol).all()

    def attend(self, layer):
        c = self.cache
        q_h = od.decode_elements(od.encode_elements(self.rng.normal(size=self.rows * self.Hq * self.D), self.io), self.io).reshape(self.rows, self.Hq, self.D)
        q, scale = self.ints(q_h, TORCH[self.io]), self.D ** -0.5
        kw = dict(cache_type=TYPE[self.kind], k_scale=self.scales[0], v_scale=self.scales[1])
        pool, bt, sl = self.pool.cpu().numpy(), c.block_table.cpu().numpy(), c.seq_lens.cpu().numpy()
        want = lambda table, lens: od.attend(self.g, layer, pool, table, lens, q_h, self.kind, self.io, scale, k_scale=self.scales[0], v_scale=self.scales[1])
        out, lse = torch.zeros_like(q), torch.zeros(q.shape[:2], device=self.dev)
        torch.cuda.synchronize()
        # all tokens, shared ones once
        c.plan_prefixes(self.stream)
        c.attend_shared(layer, q, out, scale, self.stream, lse=lse, **kw)
        self.stream.synchronize()
        assert np.array_equal(c.plan.cpu().numpy(), ot.plan_prefixes(self.g.P, self.g.num_pages, bt, sl))
        _check((out.double().cpu().numpy(), lse.double().cpu().numpy()), want(bt, sl))
        # four pages a KV head
        chosen = torch.zeros((self.rows, self.H, 4), dtype=torch.int32, device=self.dev)
        torch.cuda.synchronize()
        c.bound_pages(layer, self.stream, tokens=max(self.since[layer], 1), cache_type=TYPE[self.kind])
        self.since[layer] = 0
        c.attend_chosen(layer, q, out, chosen, scale, self.stream, last_pages=2, lse=lse, **kw)
        self.stream.synchronize()
        bounds, steps = np.zeros((self.g.num_pages, self.H, 2, self.D), np.int8), np.zeros((self.g.num_pages, self.H), np.float32)
        ot.bound_pages(self.g, layer, pool, bt, sl, 0, self.kind, bounds, steps)
        lists = ot.choose_pages(self.g.P, bt, sl, q_h, self.H, bounds, steps, 4, 1, 2)
        assert np.array_equal(chosen.cpu().numpy(), lists)
        G = self.Hq // self.H
        for h in range(self.H):
            rows = [ot.of_chosen(self.g.P, bt[r], int(sl[r]), lists[r, h]) for r in range(self.rows)]
            table = np.full((self.rows, 4), -1, np.int32)
            for r, (x, _) in enumerate(rows):
                table[r, :len(x)] = x
            part = [x[:, h * G:(h + 1) * G] for x in want(table, [n for _, n in rows])]
            _check((out.double().cpu().numpy()[:, h * G:(h + 1) * G], lse.double().cpu().numpy()[:, h * G:(h + 1) * G]), part)


@pytest.mark.parametrize("kind, io, D, pairs", [("bf16", "bf16", 64, False), ("e4m3", "bf16", 64, True), ("fp16", "fp16", 96, True), ("e4m3", "fp16", 128, False)])
def test_a_decode_workers_run(dev, kind, io, D, pairs):
    run = Run(dev, kind, io, D, pairs)
    c = run.cache
    run.turn([61, 0, 9, 0, 0, 0])                                    # two prompts arrive
    run.attend(0)
    c.fork(run.ints([0, 0, 2]), run.ints([1, 3, 4]), run.stream)     # samples of them
    for step in range(3):
        run.turn([1, 1, 1, 1, step % 2, 0], one=True)
        run.attend(step % 2)
    run.turn([3, 0, 20, 1, 0, 40])                                   # chunks: a new prompt beside the others' tokens
    run.attend(1)
    c.free(run.ints([0, 2]), run.stream)                             # the first ones end, their samples stay
    run.attend(0)
    c.compact(run.stream)
    run.turn([0, 5, 33, 1, 1, 1])
    run.attend(0)
    run.attend(1)


def test_refused_requests_keep_what_they_have(dev):
    run = Run(dev, "bf16", "bf16", 64, False, pages=6, max_pages=4)
    run.turn([20, 8, 0, 0, 0, 0])                                    # 3 + 1 pages of 6
    before = run.pool.clone()
    c = run.cache
    c.extend(run.ints([1, 17, 0, 0, 0, 0]), run.stream)              # the second one wants 3 more: 2 are left
    x = torch.ones((6, 2, 64), dtype=torch.bfloat16, device=dev)
    q_out = torch.full((6, 6, 64), 7.0, dtype=torch.bfloat16, device=dev)
    q = torch.ones_like(q_out)
    torch.cuda.synchronize()
    for layer in range(2):
        c.append_rotated(layer, x, x, run.stream, run.rotary, q, q_out)
    run.stream.synchronize()
    assert tk.topkv_device_error_flags() == 8
    tk.check(tk.topkv_reset_device_error_flags())
    assert c.seq_lens.tolist() == [21, 8, 0, 0, 0, 0]
    assert (q_out[1:] == 7).all() and not (q_out[0] == 7).any()
    changed = (run.pool != before).nonzero().flatten().cpu().numpy()
    ok = {int(a) + i for layer in range(2) for plane in range(2) for h in range(2) for i in range(128)
          for a in [od.row_offset(run.g, layer, int(c.block_table[0, 2]), plane, 20 - 16, h)]}
    assert len(changed) and set(changed.tolist()) <= ok


def test_captured_turn_and_attention(dev):
    """Extension, append, plan, shared and sparse attention in one graph, replayed: as many eager turns."""
    out = {}
    for graph in (False, True):
        run = Run(dev, "bf16", "bf16", 64, False)
        c = run.cache
        run.turn([61, 0, 9, 0, 0, 0])
        c.fork(run.ints([0, 0]), run.ints([1, 3]), run.stream)
        for layer in range(2):
            c.bound_pages(layer, run.stream)
        g = torch.Generator(device=dev)
        g.manual_seed(1)
        new = run.ints([1, 1, 1, 1, 0, 0])
        k = torch.randn((6, 2, 64), generator=g, device=dev).to(torch.bfloat16)
        q = torch.randn((6, 6, 64), generator=g, device=dev).to(torch.bfloat16)
        q_out, a, b = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(q)
        chosen = torch.zeros((6, 2, 3), dtype=torch.int32, device=dev)

        def step(s):
            c.extend(new, s)
            c.plan_prefixes(s)
            for layer in range(2):
                c.append_rotated(layer, k, k, s, run.rotary, q, q_out)
                c.bound_pages(layer, s, tokens=1)
                c.attend_shared(layer, q_out, a, 0.125, s)
                c.attend_chosen(layer, q_out, b, chosen, 0.125, s)
        torch.cuda.synchronize()
        step(run.stream)                                            # workspaces are there then
        run.stream.synchronize()
        if graph:
            gr = torch.cuda.CUDAGraph()
            with torch.cuda.graph(gr, stream=run.stream):
                step(run.stream)
            for _ in range(5):
                gr.replay()
        else:
            for _ in range(5):
                step(run.stream)
        torch.cuda.synchronize()
        out[graph] = [x.clone() for x in (run.pool, c.seq_lens, c.block_table, a, b, chosen, q_out, c.bounds, c.steps)]
    assert all(torch.equal(x, y) for x, y in zip(out[False], out[True]))

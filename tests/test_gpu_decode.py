"""GPU tests of the decode side: attention of one new token over the paged cache against the oracle
in 64 bits (tolerances derived in oracle.decode.attend), and the page operators against the
oracle's loops, integer for integer and byte for byte."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import oracle
from oracle import Geom, decode as od
from paper_2607_28633_b200 import binding as tk

pytestmark = pytest.mark.gpu

TYPE = {"bf16": tk.TOPKV_TYPE_BF16, "fp16": tk.TOPKV_TYPE_FP16, "e4m3": tk.TOPKV_TYPE_E4M3}
TORCH = {"bf16": torch.bfloat16, "fp16": torch.float16}
NAN = {"bf16": (0xC1, 0x7F), "fp16": (0x01, 0x7E), "e4m3": (0x7F, 0xFF)}


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
    yield
    assert tk.topkv_device_error_flags() == 0


def _layout(g: Geom):
    lo = tk.make_layout(g.L, g.F, g.h_kv, g.d_h, g.b_p, g.P, g.num_pages, kind=tk.TOPKV_KIND_GQA)
    lo.pool_layer_stride, lo.pool_page_stride, lo.pool_kv_stride = g.S_layer, g.S_page, g.S_kv
    lo.pool_token_stride, lo.pool_head_stride = g.S_tok, g.S_head
    return lo


def _geom(F, H, D, E, P, pages, style="page", L=1, window=0):
    g = Geom(L=L, F=F, h_kv=H, d_h=D, b_p=E, P=P, num_pages=pages)
    if style == "padded":
        g.S_tok = H * D * E + 32
        g.S_kv = P * g.S_tok
        g.S_page = F * g.S_kv + 16
        g.S_layer = pages * g.S_page
    elif style == "head":
        g.S_tok = D * E
        g.S_head = P * g.S_tok
        g.S_kv = H * g.S_head
        g.S_page = F * g.S_kv
        g.S_layer = pages * g.S_page
    elif style == "plane":
        g.S_page = P * g.S_tok
        g.S_kv = pages * g.S_page
        g.S_layer = F * g.S_kv + 16
    g.window = window
    return g


def _table(sl, P, spare, extra_cols, rng):
    pages = -(-np.asarray(sl) // P)
    n = int(pages.sum()) + spare
    bt = np.full((len(sl), max(int(pages.max()), 1) + extra_cols), -1, np.int32)
    perm, pos = rng.permutation(n), 0
    for r, k in enumerate(pages):
        bt[r, :k] = perm[pos:pos + k]
        pos += k
    return bt, n


def _run(dev, g, lo, pool, bt, sl, q, kind, io, scale, Dv=0, sinks=0, ks=1.0, vs=1.0, T=-1, layer=0, stream=None,
         out_order="rh", flags=0, batch_window=None):
    """One call; returns out float64 and lse, with guard rows around out checked."""
    R, Hq, D = q.shape
    dv = Dv or D
    d_q = torch.from_numpy(q).to(dev).to(TORCH[io])
    if out_order == "rh":
        whole = torch.full((R + 2, Hq, dv), 7.0, dtype=TORCH[io], device=dev)
        out = whole[1:R + 1]
    else:
        whole = torch.full((Hq + 2, R, dv), 7.0, dtype=TORCH[io], device=dev)
        out = whole[1:Hq + 1].transpose(0, 1)
    lse = torch.full((R, Hq), 3.0, device=dev)
    b = tk.make_batch(torch.from_numpy(np.ascontiguousarray(bt)).to(dev), torch.from_numpy(np.asarray(sl, np.int32)).to(dev), T,
                      window_tokens=g.window if batch_window is None else batch_window, flags=flags)
    att = tk.make_attention(d_q, out, TYPE[kind], TYPE[io], scale, value_dim=Dv, sink_tokens=sinks, k_scale=ks,
                            v_scale=vs, lse=lse)
    n = tk.check(tk.topkv_attend_workspace_bytes(lo, b, att))
    ws = torch.full((n + 32,), 0xFF, dtype=torch.uint8, device=dev)           # NaN patterns: nothing is assumed
    torch.cuda.synchronize()
    tk.check(tk.topkv_attend_layer(layer, pool, lo, b, att, d_q, out, ws, n, stream))
    torch.cuda.synchronize()
    assert (whole[0] == 7).all() and (whole[-1] == 7).all() and (ws[n:] == 0xFF).all()
    return out.double().cpu().numpy(), lse.double().cpu().numpy()


def _cache(g, bt, sl, kind, sinks, rng, layer=0):
    """A pool of NaN patterns in which only what the new tokens see holds numbers."""
    pool = np.empty(g.L * g.S_layer, dtype=np.uint8)
    pool[0::2], pool[1::2] = NAN[kind]
    n = g.d_h * g.b_p
    for r, s in enumerate(sl):
        for i in od.visible(int(s), g.window, sinks):
            for c in range(g.F):
                for h in range(g.h_kv):
                    a = od.row_offset(g, layer, int(bt[r, i // g.P]), c, int(i % g.P), h)
                    pool[a:a + n] = od.encode_elements(rng.normal(size=g.d_h), kind)
    return pool


def _check(got, want):
    out, lse = got
    ref, ref_lse, tol, tol_lse = want
    assert np.isfinite(out).all()
    bad = np.abs(out - ref) > tol
    assert not bad.any(), (np.argwhere(bad)[:5], out[bad][:5], ref[bad][:5], tol[bad][:5])
    empty = ref_lse == -np.inf
    assert (lse[empty] == -np.inf).all() and (out[empty] == 0).all()
    assert (np.abs(lse - ref_lse)[~empty] <= tol_lse[~empty]).all()


def _case(dev, F, H, G, D, P, sl, kind="bf16", io=None, Dv=0, window=0, sinks=0, style="page", seed=0, layer=0, L=1,
          extra_cols=1, ks=1.0, vs=1.0, **kw):
    rng = np.random.default_rng(seed)
    io = io or (kind if kind != "e4m3" else "bf16")
    bt, pages = _table(sl, P, 2, extra_cols, rng)
    g = _geom(F, H, D, 1 if kind == "e4m3" else 2, P, pages, style, L, window)
    pool_h = _cache(g, bt, sl, kind, sinks, rng, layer)
    pool = torch.from_numpy(pool_h).to(dev)
    q = od.decode_elements(od.encode_elements(rng.normal(size=(len(sl), H * G, D)).reshape(-1), io), io).reshape(len(sl), H * G, D)
    scale = D ** -0.5
    got = _run(dev, g, _layout(g), pool, bt, sl, q, kind, io, scale, Dv, sinks, ks, vs, layer=layer, **kw)
    _check(got, od.attend(g, layer, pool_h, bt, sl, q, kind, io, scale, Dv, sinks, ks, vs))
    assert np.array_equal(pool.cpu().numpy(), pool_h)
    return got


# ------------------------------------------------------------------------- grouped heads

@pytest.mark.parametrize("kind", ["bf16", "fp16", "e4m3"])
@pytest.mark.parametrize("D", [16, 64, 80, 128, 192, 256])
def test_attend_head_dims_and_types(dev, kind, D):
    _case(dev, 2, 2, 4, D, 16, [1, 17, 64, 130], kind, ks=0.5 if kind == "e4m3" else 1.0, vs=2.0 if kind == "e4m3" else 1.0)


@pytest.mark.parametrize("sl", [[1], [0, 5, 0], [16, 15, 33, 64, 65], [255, 256], [0, 0], [257, 3, 900, 0, 64]])
def test_attend_lengths(dev, sl):
    _case(dev, 2, 2, 3, 64, 16, sl, seed=len(sl))


@pytest.mark.parametrize("H,G", [(1, 1), (1, 16), (1, 17), (3, 5), (8, 8), (2, 40), (16, 1), (5, 7)])
def test_attend_head_layouts(dev, H, G):
    _case(dev, 2, H, G, 64, 16, [70, 1, 333], seed=H * 100 + G)


@pytest.mark.parametrize("style", ["page", "padded", "head", "plane"])
@pytest.mark.parametrize("P", [1, 3, 16, 48, 512])
def test_attend_pools_and_pages(dev, style, P):
    _case(dev, 2, 2, 2, 72, P, [100, 500, 7], "fp16", style=style, seed=P, layer=1, L=2)


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 4), (64, 0), (100, 5), (128, 128), (300, 4), (5000, 3)])
def test_attend_window_and_sinks(dev, window, sinks):
    _case(dev, 2, 2, 4, 64, 16, [1, 2, 16, 64, 120, 257, 700, 0], "fp16", window=window, sinks=sinks, seed=window)


@pytest.mark.parametrize("kind,io", [("e4m3", "bf16"), ("e4m3", "fp16"), ("bf16", "bf16")])
@pytest.mark.parametrize("H,sl", [(1, [4000]), (2, [3000, 17, 999, 2048]), (8, [1500, 1, 0, 400])])
def test_attend_split_requests(dev, kind, io, H, sl):
    """Lengths that are cut between CTAs, from one request over all of them to several in one."""
    _case(dev, 2, H, 2, 64, 16, sl, kind, io, seed=sum(sl))


def test_attend_many_requests(dev):
    """More requests than threads look at, most of them short, a long one in the middle; the
    cut and the uncut way of sharing out the work give results within the same bound."""
    rng = np.random.default_rng(1)
    sl = rng.integers(0, 40, size=1500)
    sl[700] = 600
    _case(dev, 2, 1, 2, 16, 16, sl, "fp16", seed=9)
    _case(dev, 2, 1, 2, 16, 16, np.minimum(sl, 60), "fp16", seed=9)


def test_attend_same_bits_every_time_and_out_layouts(dev):
    kw = dict(kind="bf16", seed=4)
    a = _case(dev, 2, 2, 4, 128, 16, [2000, 30, 700], **kw)
    b = _case(dev, 2, 2, 4, 128, 16, [2000, 30, 700], out_order="hr", stream=torch.cuda.Stream(dev), **kw)
    c = _case(dev, 2, 2, 4, 128, 16, [2000, 30, 700], T=2730, flags=tk.TOPKV_FLAG_TABLES_SETTLED, **kw)
    for x in (b, c):
        assert np.array_equal(a[0], x[0]) and np.array_equal(a[1], x[1])


def _values_case(dev, k_rows, v_rows, q, kind="fp16", **kw):
    """One request, one head, D = 8 columns used of 16: explicit K, V and q."""
    n, D = len(k_rows), 16
    bt, pages = _table([n], 16, 1, 0, np.random.default_rng(3))
    g = _geom(2, 1, D, 2, 16, pages)
    pool = np.zeros(g.pool_bytes(), np.uint8)
    for i in range(n):
        for c, rows in ((0, k_rows), (1, v_rows)):
            a = od.row_offset(g, 0, int(bt[0, i // 16]), c, i % 16, 0)
            row = np.zeros(D)
            row[:len(rows[i])] = rows[i]
            pool[a:a + 2 * D] = od.encode_elements(row, kind)
    qq = np.zeros((1, 1, D))
    qq[0, 0, :len(q)] = q
    return g, pool, bt, [n], qq, _run(dev, g, _layout(g), torch.from_numpy(pool).to(dev), bt, [n], qq, kind, kind, 1.0, **kw)


def test_attend_extreme_values(dev):
    # one token far above many others whose weights are far below the largest: they still count
    n = 6000
    k = np.zeros((n, 1)); k[17] = 16.0
    v = np.ones((n, 1)); v[17] = 0.0
    g, pool, bt, sl, q, got = _values_case(dev, k, v, [1.0])
    _check(got, od.attend(g, 0, pool, bt, sl, q, "fp16", "fp16", 1.0))
    # the type's lowest value as a key, one token and all of them
    for n, rows in ((70, [3]), (70, range(70))):
        k = np.full((n, 1), 0.25)
        k[list(rows)] = -65504.0
        g, pool, bt, sl, q, got = _values_case(dev, k, np.arange(n)[:, None] / 8, [2.0])
        _check(got, od.attend(g, 0, pool, bt, sl, q, "fp16", "fp16", 1.0))
    # infinities and NaN in visible places act as in the formula
    k = np.full((70, 1), 0.25); k[5] = -np.inf
    *_, (out, lse) = _values_case(dev, k, np.ones((70, 1)), [2.0])
    assert abs(out[0, 0, 0] - 1) < 1e-3 and abs(lse[0, 0] - (0.5 + np.log(69))) < 1e-5
    k = np.full((70, 1), -np.inf)
    *_, (out, lse) = _values_case(dev, k, np.ones((70, 1)), [2.0])
    assert np.isnan(out[0, 0, 0])
    for bad in (np.inf, np.nan):
        k = np.zeros((400, 1)); k[333] = bad
        *_, (out, lse) = _values_case(dev, k, np.ones((400, 1)), [2.0])
        assert np.isnan(out[0, 0, 0]) and np.isnan(lse[0, 0])
        v = np.zeros((400, 1)); v[2] = bad
        *_, (out, lse) = _values_case(dev, np.zeros((400, 1)), v, [2.0])
        assert not np.isfinite(out[0, 0, 0]) and abs(lse[0, 0] - np.log(400)) < 1e-5


@pytest.mark.parametrize("big", [1e-30, 1e30])
def test_attend_8bit_cache_with_queries_beyond_fp16(dev, big):
    """bf16 queries of any magnitude over an 8-bit cache."""
    rng = np.random.default_rng(5)
    bt, pages = _table([90], 16, 1, 0, rng)
    g = _geom(2, 1, 64, 1, 16, pages)
    pool = _cache(g, bt, [90], "e4m3", 0, rng)
    q = rng.normal(size=(1, 3, 64)) * big
    q[0, 2] = 0
    q = od.decode_elements(od.encode_elements(q.reshape(-1), "bf16"), "bf16").reshape(q.shape)
    got = _run(dev, g, _layout(g), torch.from_numpy(pool).to(dev), bt, [90], q, "e4m3", "bf16", 0.1 / big)
    _check(got, od.attend(g, 0, pool, bt, [90], q, "e4m3", "bf16", 0.1 / big))


def test_attend_unusable_tables(dev):
    """Page ids outside the pool are skipped, lengths outside the row cut; both raise bit 2."""
    rng = np.random.default_rng(6)
    sl = [90, 40]
    bt, pages = _table(sl, 16, 1, 0, rng)
    g = _geom(2, 1, 64, 2, 16, pages)
    pool_h = _cache(g, bt, sl, "bf16", 0, rng)
    pool = torch.from_numpy(pool_h).to(dev)
    q = od.decode_elements(od.encode_elements(rng.normal(size=2 * 64), "bf16"), "bf16").reshape(2, 1, 64)
    for bad in (pages, -1, 1 << 30):
        broken = bt.copy()
        broken[0, 2] = bad
        out, lse = _run(dev, g, _layout(g), pool, broken, sl, q, "bf16", "bf16", 0.125)
        assert tk.topkv_device_error_flags() == 2
        tk.check(tk.topkv_reset_device_error_flags())
        rows = [i for i in range(90) if i // 16 != 2]           # what is left of request 0
        k, v = (od.rows_of(g, 0, pool_h, bt[0], np.array(rows), c, 0, "bf16") for c in (0, 1))
        w = np.exp(0.125 * k @ q[0, 0])
        assert np.abs(out[0, 0] - w @ v / w.sum()).max() < 2.0 ** -6 and abs(lse[0, 0] - np.log(w.sum())) < 1e-4
    out, lse = _run(dev, g, _layout(g), pool, bt[:, :3], [48, 1000], q, "bf16", "bf16", 0.125)
    assert tk.topkv_device_error_flags() == 2 and np.isfinite(lse).sum() >= 1
    tk.check(tk.topkv_reset_device_error_flags())
    out, lse = _run(dev, g, _layout(g), pool, bt, [90, -3], q, "bf16", "bf16", 0.125)
    assert tk.topkv_device_error_flags() == 2 and lse[1, 0] == -np.inf and (out[1] == 0).all()
    tk.check(tk.topkv_reset_device_error_flags())


def test_attend_rows_past_two_gigabytes(dev):
    """Offsets beyond 32 bits: the pages in use lie at the end of a 6 GiB pool."""
    g = _geom(2, 8, 128, 2, 16, 6 * (1 << 30) // 65536)
    pool = torch.zeros(g.pool_bytes(), dtype=torch.uint8, device=dev)
    rng = np.random.default_rng(8)
    sl = [40, 300]
    bt = np.full((2, 20), -1, np.int32)
    bt[0, :3] = [g.num_pages - 1, 5, g.num_pages - 7]
    bt[1, :19] = g.num_pages - 100 + np.arange(19)
    want = {}
    for p in {int(x) for x in bt.reshape(-1) if x >= 0}:
        want[p] = od.encode_elements(rng.normal(size=32768), "bf16")
        pool[p * 65536:(p + 1) * 65536] = torch.from_numpy(want[p]).to(dev)
    small = _geom(2, 8, 128, 2, 16, len(want))
    order = {p: i for i, p in enumerate(want)}
    pool_h = np.concatenate(list(want.values()))
    bt_h = np.array([[order.get(int(x), -1) for x in row] for row in bt], np.int32)
    q = od.decode_elements(od.encode_elements(rng.normal(size=2 * 16 * 128), "bf16"), "bf16").reshape(2, 16, 128)
    got = _run(dev, g, _layout(g), pool, bt, sl, q, "bf16", "bf16", 0.09)
    _check(got, od.attend(small, 0, pool_h, bt_h, sl, q, "bf16", "bf16", 0.09))


def test_attend_in_a_graph_and_on_two_streams(dev):
    """Captured and replayed with other contents; two calls at the same time with a workspace each."""
    rng = np.random.default_rng(11)
    sl = [1500, 40]
    bt, pages = _table(sl, 16, 1, 0, rng)
    g = _geom(2, 2, 64, 2, 16, pages)
    lo = _layout(g)
    pool = torch.zeros(g.pool_bytes(), dtype=torch.uint8, device=dev)
    b = tk.make_batch(torch.from_numpy(bt).to(dev), torch.tensor(sl, dtype=torch.int32, device=dev))
    q = torch.zeros(2, 8, 64, dtype=torch.bfloat16, device=dev)
    outs = [torch.zeros_like(q) for _ in range(2)]
    lses = [torch.zeros(2, 8, device=dev) for _ in range(2)]
    T = tk.TOPKV_TYPE_BF16
    atts = [tk.make_attention(q, o, T, T, 0.125, lse=l) for o, l in zip(outs, lses)]
    n = tk.check(tk.topkv_attend_workspace_bytes(lo, b, atts[0]))
    assert n > 0
    ws = [torch.empty(n, dtype=torch.uint8, device=dev) for _ in range(2)]
    call = lambda i, s: tk.check(tk.topkv_attend_layer(0, pool, lo, b, atts[i], q, outs[i], ws[i], n, s))
    call(0, torch.cuda.current_stream())                      # shared-memory limit raised outside the capture
    torch.cuda.synchronize()
    side = torch.cuda.Stream(dev)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call(0, torch.cuda.current_stream())
    for seed in (1, 2):
        r2 = np.random.default_rng(seed)
        pool_h = _cache(g, bt, sl, "bf16", 0, r2)
        pool.copy_(torch.from_numpy(pool_h))
        q_h = od.decode_elements(od.encode_elements(r2.normal(size=2 * 8 * 64), "bf16"), "bf16").reshape(2, 8, 64)
        q.copy_(torch.from_numpy(q_h).to(torch.bfloat16))
        torch.cuda.synchronize()
        for _ in range(5):
            graph.replay()
            call(1, side)
        torch.cuda.synchronize()
        want = od.attend(g, 0, pool_h, bt, sl, q_h, "bf16", "bf16", 0.125)
        for o, l in zip(outs, lses):
            _check((o.double().cpu().numpy(), l.double().cpu().numpy()), want)


# ------------------------------------------------------------------------- page operators

def _page_case(seed, L=2, F=2, H=2, D=8, E=2, P=4, R=7, style="page", spare=5, maxlen=20):
    rng = np.random.default_rng(seed)
    sl = rng.integers(0, maxlen + 1, size=R).astype(np.int32)
    bt, pages = _table(sl, P, spare, 2, rng)
    g = _geom(F, H, D, E, P, pages, style, L)
    ref = np.zeros(pages, np.int32)
    for p in bt[bt >= 0]:
        ref[p] += 1
    pool = rng.integers(0, 256, g.L * g.S_layer, dtype=np.uint8)
    return rng, g, sl, bt, ref, pool


class _State:
    """Device copies of the tables and the pool, an out set apart or in place."""

    def __init__(self, dev, g, sl, bt, ref, pool, in_place, skew=0):
        self.g, self.lo = g, _layout(g)
        put = lambda x: torch.from_numpy(np.ascontiguousarray(x).copy()).to(dev)
        buf = torch.zeros(len(pool) + skew, dtype=torch.uint8, device=dev)
        self.pool = buf[skew:]
        self.pool.copy_(put(pool))
        self.first = (put(bt), put(sl), put(ref))
        self.out = self.first if in_place else tuple(torch.full_like(x, -77) for x in self.first)
        self.batch = tk.make_batch(self.first[0], self.first[1])
        self.tables = tk.make_page_tables(self.first[2], *self.out)
        self.put = put
        n = tk.check(tk.topkv_page_workspace_bytes(self.lo, self.batch, 64))
        self.ws = torch.full((n,), 0x55, dtype=torch.uint8, device=dev)
        self.n = n

    def check(self, bt, sl, ref, pool, err):
        torch.cuda.synchronize()
        assert tk.topkv_device_error_flags() == err
        tk.check(tk.topkv_reset_device_error_flags())
        for got, want in zip(self.out, (bt, sl, ref)):
            assert np.array_equal(got.cpu().numpy(), want)
        assert np.array_equal(self.pool.cpu().numpy(), pool)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("seed", range(6))
def test_extend(dev, seed, in_place):
    rng, g, sl, bt, ref, pool = _page_case(seed, spare=[5, 0, 3, 40, 6, 2][seed], P=[4, 1, 16, 3, 4, 8][seed])
    s = _State(dev, g, sl, bt, ref, pool, in_place)
    new = rng.integers(0, 6, size=len(sl)).astype(np.int32)
    if seed == 4:
        new[2], new[5] = -1, 1 << 30
    d_new = s.put(new)
    tk.check(tk.topkv_extend_requests(s.lo, s.batch, s.tables, d_new, s.ws, s.n))
    err = od.extend_requests(g.P, bt, sl, ref, new)
    s.check(bt, sl, ref, pool, err)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("seed", range(4))
def test_free(dev, seed, in_place):
    rng, g, sl, bt, ref, pool = _page_case(seed, R=9)
    ref[bt[0, 0]] += 2                                       # a page that others use too
    if seed == 3:
        ref[bt[1, 0]] = 0                                    # a count that is wrong already
        bt[2, 0], sl[2] = len(ref), max(int(sl[2]), 1)
        sl[3] = bt.shape[1] * g.P + 1
    s = _State(dev, g, sl, bt, ref, pool, in_place)
    rows = np.array([3, 0, 3, 1, 2] if seed != 1 else [0, 9, -1, 0], np.int32)
    tk.check(tk.topkv_free_requests(s.lo, s.batch, s.tables, s.put(rows), len(rows)))
    err = od.free_requests(g.P, bt, sl, ref, rows)
    s.check(bt, sl, ref, pool, err)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("style,E,P,skew", [("page", 2, 4, 0), ("padded", 2, 4, 0), ("head", 2, 5, 16), ("plane", 2, 1, 0),
                                            ("page", 2, 200, 16)])
def test_fork(dev, style, E, P, skew, in_place):
    for seed in range(3):
        rng, g, sl, bt, ref, pool = _page_case(seed, E=E, P=P, R=9, style=style, D=64 if P == 200 else 8, maxlen=5 * P,
                                               spare=[4, 2, 0][seed])
        sl[[1, 4, 6]], kept = 0, bt.copy()
        for r in (1, 4, 6):
            for p in kept[r][kept[r] >= 0]:
                ref[p] -= 1
            bt[r] = -1
        ref[bt[0][bt[0] >= 0]] += seed                       # shared already
        s = _State(dev, g, sl, bt, ref, pool, in_place, skew)
        parents = np.array([0, 0, 2, 0, 3, 5, 20], np.int32)
        children = np.array([4, 1, 4, 6, 3, -1, 6], np.int32)  # a row named twice, itself, outside
        if seed == 0:
            parents, children = parents[:2], children[:2]
        tk.check(tk.topkv_fork_requests(s.pool, s.lo, s.batch, s.tables, s.put(parents), s.put(children), len(parents),
                                        s.ws, s.n))
        err = od.fork_requests(g, pool, bt, sl, ref, parents, children)
        s.check(bt, sl, ref, pool, err)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("style,P,skew,pages", [("page", 4, 0, 5), ("padded", 4, 0, 60), ("head", 3, 16, 9), ("plane", 16, 0, 5),
                                                ("page", 1, 0, 9000)])
def test_compact(dev, style, P, skew, pages, in_place):
    for seed in range(3):
        rng, g, sl, bt, ref, pool = _page_case(seed, P=P, R=8, style=style, spare=pages, L=1 if pages > 1000 else 2, maxlen=9 * P)
        ref[bt[3][bt[3] >= 0]] -= 1                          # a request that ended
        bt[3], sl[3] = -1, 0
        ref[rng.integers(0, len(ref), size=3)] += 2          # pages that somebody holds outside the table
        if seed == 2 and sl[5] > 0:
            bt[5, 0] = len(ref) + 3
        s = _State(dev, g, sl, bt, ref, pool, in_place, skew)
        used = torch.full((1,), -5, dtype=torch.int32, device=dev)
        to = torch.full((g.num_pages,), -5, dtype=torch.int32, device=dev)
        tk.check(tk.topkv_compact_pages(s.pool, s.lo, s.batch, s.tables, used, to, s.ws, s.n))
        err, n, want_to = od.compact_pages(g, pool, bt, sl, ref)
        s.check(bt, sl, ref, pool, err)
        assert used.item() == n and np.array_equal(to.cpu().numpy(), want_to)
        ids = np.flatnonzero(ref > 0)
        assert np.array_equal(ids, np.arange(n))


def test_compact_without_requests_and_when_there_is_nothing_to_do(dev):
    _, g, sl, bt, ref, pool = _page_case(3)
    ref[:] = 0
    ref[[2, 3, len(ref) - 1]] = 4
    lo = _layout(g)
    d = torch.from_numpy(pool).to(dev)
    d_ref = torch.from_numpy(ref.copy()).to(dev)
    empty = torch.empty((0, 4), dtype=torch.int32, device=dev)
    none = torch.empty((0,), dtype=torch.int32, device=dev)
    b, t = tk.make_batch(empty, none), tk.make_page_tables(d_ref, empty, none, d_ref)
    n = tk.check(tk.topkv_page_workspace_bytes(lo, b, 0))
    ws, used = torch.empty(n, dtype=torch.uint8, device=dev), torch.zeros(1, dtype=torch.int32, device=dev)
    to = torch.zeros(len(ref), dtype=torch.int32, device=dev)
    bt0, sl0 = np.zeros((0, 4), np.int32), np.zeros(0, np.int32)
    for _ in range(2):                                       # the second time nothing moves
        tk.check(tk.topkv_compact_pages(d, lo, b, t, used, to, ws, n))
        _, want, want_to = od.compact_pages(g, pool, bt0, sl0, ref)
        assert used.item() == want == 3 and np.array_equal(to.cpu().numpy(), want_to)
        assert np.array_equal(d_ref.cpu().numpy(), ref) and np.array_equal(d.cpu().numpy(), pool)


@pytest.mark.parametrize("style,P,D,skew", [("page", 4, 8, 0), ("padded", 4, 8, 16), ("head", 3, 16, 0), ("plane", 1, 64, 0),
                                            ("page", 300, 64, 0), ("padded", 130, 64, 0)])
def test_copy_pages(dev, style, P, D, skew):
    rng, g, sl, bt, ref, pool = _page_case(1, P=P, D=D, L=3, style=style, spare=12)
    ids = rng.permutation(g.num_pages)[:9].astype(np.int32)
    src, dst = ids[:4].copy(), ids[4:8].copy()
    buf = torch.zeros(len(pool) + skew, dtype=torch.uint8, device=dev)
    d = buf[skew:]
    d.copy_(torch.from_numpy(pool))
    lo = _layout(g)
    put = lambda x: torch.from_numpy(x).to(dev)
    tk.check(tk.topkv_copy_pages(1, 2, d, lo, put(src), put(dst), 4))
    od.copy_pages(g, pool, 1, 2, src, dst)
    assert np.array_equal(d.cpu().numpy(), pool)
    # unusable entries are skipped, a page onto itself is left alone
    src = np.array([ids[0], -1, ids[8], ids[1]], np.int32)
    dst = np.array([g.num_pages, ids[2], ids[8], ids[3]], np.int32)
    tk.check(tk.topkv_copy_pages(0, 1, d, lo, put(src), put(dst), 4))
    assert od.copy_pages(g, pool, 0, 1, src, dst) == 2 == tk.topkv_device_error_flags()
    tk.check(tk.topkv_reset_device_error_flags())
    assert np.array_equal(d.cpu().numpy(), pool)


def test_a_random_run_of_page_operators(dev):
    """Thirty calls in a row, in place, against the oracle's loops; then a compaction."""
    rng, g, sl, bt, ref, pool = _page_case(21, R=12, P=4, spare=40, maxlen=16)
    s = _State(dev, g, sl, bt, ref, pool, True)
    err = 0
    for _ in range(30):
        op = rng.integers(0, 3)
        if op == 0:
            new = rng.integers(0, 4, size=12).astype(np.int32)
            new[sl == 0] = 0
            tk.check(tk.topkv_extend_requests(s.lo, s.batch, s.tables, s.put(new), s.ws, s.n))
            err |= od.extend_requests(g.P, bt, sl, ref, new)
        elif op == 1:
            rows = rng.integers(0, 12, size=3).astype(np.int32)
            tk.check(tk.topkv_free_requests(s.lo, s.batch, s.tables, s.put(rows), 3))
            err |= od.free_requests(g.P, bt, sl, ref, rows)
        else:
            parents, children = rng.integers(0, 12, size=4).astype(np.int32), rng.integers(0, 12, size=4).astype(np.int32)
            tk.check(tk.topkv_fork_requests(s.pool, s.lo, s.batch, s.tables, s.put(parents), s.put(children), 4, s.ws, s.n))
            err |= od.fork_requests(g, pool, bt, sl, ref, parents, children)
    used, to = torch.zeros(1, dtype=torch.int32, device=dev), torch.zeros(g.num_pages, dtype=torch.int32, device=dev)
    tk.check(tk.topkv_compact_pages(s.pool, s.lo, s.batch, s.tables, used, to, s.ws, s.n))
    err |= od.compact_pages(g, pool, bt, sl, ref)[0]
    counts = np.zeros_like(ref)
    for r in range(12):
        np.add.at(counts, bt[r, :-(-int(sl[r]) // g.P)], 1)
    assert np.array_equal(counts, ref)                       # the counts are the table's
    s.check(bt, sl, ref, pool, err)


# ------------------------------------------------------------------------- latent rows

@pytest.mark.parametrize("kind", ["bf16", "fp16"])
@pytest.mark.parametrize("Hq", [1, 16, 17, 32, 40, 64, 128])
def test_latent_heads(dev, kind, Hq):
    _case(dev, 1, 1, Hq, 576, 64, [100, 1, 64], kind, Dv=512, seed=Hq)


@pytest.mark.parametrize("D,Dv", [(576, 512), (288, 256), (192, 128), (320, 320), (64, 16), (24, 16), (72, 48), (512, 512), (576, 400)])
def test_latent_dims(dev, D, Dv):
    _case(dev, 1, 1, 20, D, 16, [130, 7, 0], "bf16", Dv=Dv, seed=D)


@pytest.mark.parametrize("P,style", [(1, "page"), (3, "padded"), (16, "padded"), (64, "page"), (100, "page"), (512, "padded")])
def test_latent_pages(dev, P, style):
    _case(dev, 1, 1, 8, 192, P, [300, 65, 1, 64], "fp16", Dv=128, style=style, seed=P, layer=1, L=2)


@pytest.mark.parametrize("sl", [[1], [0, 0], [0, 257, 1, 0, 900, 64], [4000], [700, 3000, 63]])
def test_latent_lengths(dev, sl):
    for Hq in (3, 70):
        _case(dev, 1, 1, Hq, 128, 16, sl, "bf16", Dv=64, seed=sum(sl))


@pytest.mark.parametrize("window,sinks", [(1, 0), (64, 4), (100, 0), (700, 65)])
def test_latent_window_and_sinks(dev, window, sinks):
    _case(dev, 1, 1, 16, 128, 16, [1, 64, 257, 1400, 0], "fp16", Dv=128, window=window, sinks=sinks, seed=window)


def test_latent_growing_scores(dev):
    """Each tile's scores lie far above the ones before: the running maximum moves every time, by
    little and by much, up to weights that vanish."""
    for step in (0.5, 3.0, 9.0, 40.0):
        for kind in ("bf16", "fp16"):
            rng = np.random.default_rng(17)
            sl = [900]
            bt, pages = _table(sl, 64, 1, 0, rng)
            g = _geom(1, 1, 64, 2, 64, pages)
            pool = np.zeros(g.pool_bytes(), np.uint8)
            for i in range(900):
                row = rng.normal(size=64)
                row[0] = (i // 64) * step if i % 3 else -(i // 64) * step
                a = od.row_offset(g, 0, int(bt[0, i // 64]), 0, i % 64, 0)
                pool[a:a + 128] = od.encode_elements(row, kind)
            q = np.zeros((1, 18, 64))
            q[0, :, 0] = np.linspace(-2, 2, 18)
            q[0, :, 1:] = 0.1 * rng.normal(size=(18, 63))
            q = od.decode_elements(od.encode_elements(q.reshape(-1), kind), kind).reshape(q.shape)
            got = _run(dev, g, _layout(g), torch.from_numpy(pool).to(dev), bt, sl, q, kind, kind, 1.0, 64)
            _check(got, od.attend(g, 0, pool, bt, sl, q, kind, kind, 1.0, 64))


def test_latent_same_bits_graph_and_unusable_tables(dev):
    rng = np.random.default_rng(12)
    sl = [1500, 40, 700]
    a = _case(dev, 1, 1, 33, 192, 16, sl, "bf16", Dv=128, seed=2)
    b = _case(dev, 1, 1, 33, 192, 16, sl, "bf16", Dv=128, seed=2, T=2240, flags=tk.TOPKV_FLAG_TABLES_SETTLED, out_order="hr")
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])
    bt, pages = _table(sl, 16, 1, 0, rng)
    g = _geom(1, 1, 192, 2, 16, pages)
    pool_h = _cache(g, bt, sl, "bf16", 0, rng)
    q = od.decode_elements(od.encode_elements(rng.normal(size=3 * 4 * 192), "bf16"), "bf16").reshape(3, 4, 192)
    broken = bt.copy()
    broken[1, :] = -1
    broken[2, 1] = 1 << 29
    out, lse = _run(dev, g, _layout(g), torch.from_numpy(pool_h).to(dev), broken, sl, q, "bf16", "bf16", 0.07, 128)
    assert tk.topkv_device_error_flags() == 2
    tk.check(tk.topkv_reset_device_error_flags())
    want = od.attend(g, 0, pool_h, bt, sl, q, "bf16", "bf16", 0.07, 128)
    assert (np.abs(out[0] - want[0][0]) <= want[2][0]).all()
    assert np.isfinite(out[2]).all() and (lse[1] == -np.inf).all()


# ------------------------------------------------------------------------- all of it together

@pytest.mark.parametrize("F,H,G,D,Dv", [(2, 2, 4, 64, 0), (1, 1, 24, 192, 128)])
def test_received_cache_is_decoded(dev, F, H, G, D, Dv):
    """A transfer through pinned host memory, then a decode worker's life on the cache it received:
    tokens appended and attended to, a request forked, another one freed, the pool compacted."""
    from paper_2607_28633_b200 import harness, session, workloads as wl
    spec = wl.WorkloadSpec("decode", L=2, F=F, H=H, D=D, E=2, P=8, R=3, lengths=("fixed", (16, 33, 290)), pool_factor=2.0, seed=40)
    w = harness.setup(spec, dev, need_wire=False)
    tx = session.TransferSender(w.src_pool, w.layout, w.src_bt, w.seq_lens, w.batch.total_tokens)
    rx = session.TransferReceiver(w.dst_pool, w.layout, w.dst_bt, w.seq_lens, w.batch.total_tokens)
    h_wire = torch.zeros(spec.L * w.n_layer, dtype=torch.uint8).pin_memory()
    _, status = session.transfer(tx, rx, h_wire, [1, 2, 3], 7, w.batch.seq_lens)
    assert status == [tk.TOPKV_OK] * 3
    g = Geom(L=2, F=F, h_kv=H, d_h=D, b_p=2, P=8, num_pages=w.batch.num_pool_pages)
    cache = session.DecodeCache(w.dst_pool, w.layout, w.dst_bt, w.seq_lens, rows=5, max_pages=w.dst_bt.shape[1] + 2)
    # the oracle's copies
    pool = w.dst_pool.cpu().numpy()
    bt, sl, ref = (x.cpu().numpy().copy() for x in (cache.block_table, cache.seq_lens, cache.ref_counts))
    rng = np.random.default_rng(3)
    s = torch.cuda.Stream(dev)
    put = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)
    keep = []

    def step(live):
        new = np.array([1 if r in live else 0 for r in range(5)], np.int32)
        d_new = put(new)
        s.wait_stream(torch.cuda.current_stream(dev))
        cache.extend(d_new, s)
        assert od.extend_requests(g.P, bt, sl, ref, new) == 0
        for layer in range(2):
            rows = od.encode_elements(rng.normal(size=len(live) * F * H * D), "bf16")
            kv = torch.from_numpy(rows).to(dev)
            q = torch.from_numpy(rng.normal(size=(5, H * G, D))).to(dev).to(torch.bfloat16)
            out = torch.zeros((5, H * G, Dv or D), dtype=torch.bfloat16, device=dev)
            s.wait_stream(torch.cuda.current_stream(dev))
            cache.append(layer, kv, s)
            keep.append((kv, q, out, d_new))
            rows = rows.reshape(len(live), F, H, D * 2)
            for k, r in enumerate(live):
                i = int(sl[r]) - 1
                for c in range(F):
                    for h in range(H):
                        a = od.row_offset(g, layer, int(bt[r, i // g.P]), c, i % g.P, h)
                        pool[a:a + 2 * D] = rows[k, c, h]
            cache.attend(layer, q, out, D ** -0.5, s, value_dim=Dv)
            s.synchronize()
            want, _, tol, _ = od.attend(g, layer, pool, bt, sl, q.double().cpu().numpy(), "bf16", "bf16", D ** -0.5, Dv)
            assert (np.abs(out.double().cpu().numpy() - want) <= tol).all()

    step([0, 1, 2])
    parents, children = put([2, 1]), put([3, 4])
    s.wait_stream(torch.cuda.current_stream(dev))
    cache.fork(parents, children, s)
    assert od.fork_requests(g, pool, bt, sl, ref, [2, 1], [3, 4]) == 0
    step([0, 1, 2, 3, 4])
    ended = put([2, 0])
    s.wait_stream(torch.cuda.current_stream(dev))
    cache.free(ended, s)
    assert od.free_requests(g.P, bt, sl, ref, [2, 0]) == 0
    step([1, 3, 4])
    cache.compact(s)
    err, n, to = od.compact_pages(g, pool, bt, sl, ref)
    step([1, 3, 4])
    s.synchronize()
    assert err == 0 and cache.num_used.item() == n
    for got, want in ((cache.block_table, bt), (cache.seq_lens, sl), (cache.ref_counts, ref), (w.dst_pool, pool)):
        assert np.array_equal(got.cpu().numpy(), want)


# ------------------------------------------------------------------------- calls at the edges

@pytest.mark.parametrize("D,kind", [(8, "bf16"), (24, "fp16"), (248, "bf16"), (48, "e4m3"), (144, "e4m3")])
def test_attend_odd_head_dims(dev, D, kind):
    _case(dev, 2, 3, 2, D, 16, [33, 600, 1], kind, seed=D)


@pytest.mark.parametrize("F", [1, 2])
def test_attend_broadcast_queries(dev, F):
    """One query for all requests, and one for all heads (strides of 0)."""
    rng = np.random.default_rng(2)
    sl, D, Dv, Hq = [400, 20, 1500], 64, 48 if F == 1 else 0, 6
    bt, pages = _table(sl, 16, 1, 0, rng)
    g = _geom(F, 1, D, 2, 16, pages)
    pool_h = _cache(g, bt, sl, "bf16", 0, rng)
    pool, lo = torch.from_numpy(pool_h).to(dev), _layout(g)
    b = tk.make_batch(torch.from_numpy(bt).to(dev), torch.tensor(sl, dtype=torch.int32, device=dev))
    base = torch.from_numpy(rng.normal(size=(3, Hq, D))).to(dev).to(torch.bfloat16)
    for q in (base[:1].expand(3, Hq, D), base[:, :1].expand(3, Hq, D), base[:1, :1].expand(3, Hq, D)):
        out = torch.zeros(3, Hq, Dv or D, dtype=torch.bfloat16, device=dev)
        lse = torch.zeros(3, Hq, device=dev)
        att = tk.make_attention(q, out, 1, 1, 0.125, value_dim=Dv, lse=lse)
        n = tk.check(tk.topkv_attend_workspace_bytes(lo, b, att))
        ws = torch.empty(n, dtype=torch.uint8, device=dev)
        tk.check(tk.topkv_attend_layer(0, pool, lo, b, att, q, out, ws, n))
        torch.cuda.synchronize()
        _check((out.double().cpu().numpy(), lse.double().cpu().numpy()),
               od.attend(g, 0, pool_h, bt, sl, q.double().cpu().numpy(), "bf16", "bf16", 0.125, Dv))


@pytest.mark.parametrize("F,Hq,Dv", [(2, 2, 0), (1, 5, 16)])
def test_attend_mostly_empty_batches(dev, F, Hq, Dv):
    """A padded batch: far more rows than CTAs, nearly all of them empty, lengths of 0 at both ends."""
    sl = np.zeros(3000, np.int64)
    sl[[5, 1234, 2998]] = [700, 1, 330]
    _case(dev, F, 1, Hq, 32, 16, sl, "bf16", Dv=Dv)
    _case(dev, F, 1, Hq, 32, 16, np.minimum(sl, 200), "bf16", Dv=Dv)
    _case(dev, F, 1, Hq, 32, 16, np.zeros(2000, np.int64), "bf16", Dv=Dv, extra_cols=100)


@pytest.mark.parametrize("P", [8, 24, 40, 64, 192])
def test_latent_tensor_copies_with_a_bad_page(dev, P):
    """Pages of several pieces and of odd multiples of 8; the tile with the bad page comes row by row."""
    rng = np.random.default_rng(P)
    sl = [1000, 129]
    bt, pages = _table(sl, P, 2, 1, rng)
    g = _geom(1, 1, 128, 2, P, pages)
    pool_h = _cache(g, bt, sl, "bf16", 0, rng)
    pool = torch.from_numpy(pool_h).to(dev)
    q = od.decode_elements(od.encode_elements(rng.normal(size=2 * 17 * 128), "bf16"), "bf16").reshape(2, 17, 128)
    got = _run(dev, g, _layout(g), pool, bt, sl, q, "bf16", "bf16", 0.09, 64)
    _check(got, od.attend(g, 0, pool_h, bt, sl, q, "bf16", "bf16", 0.09, 64))
    broken = bt.copy()
    broken[0, 3] = pages + 7
    out, lse = _run(dev, g, _layout(g), pool, broken, sl, q, "bf16", "bf16", 0.09, 64)
    assert tk.topkv_device_error_flags() == 2
    tk.check(tk.topkv_reset_device_error_flags())
    rows = np.array([i for i in range(1000) if i // P != 3])
    k = od.rows_of(g, 0, pool_h, bt[0], rows, 0, 0, "bf16")
    for a in range(17):
        w = np.exp(0.09 * k @ q[0, a])
        assert np.abs(out[0, a] - w @ k[:, :64] / w.sum()).max() < 2.0 ** -6 and abs(lse[0, a] - np.log(w.sum())) < 1e-4
    _, want_lse, _, _ = od.attend(g, 0, pool_h, bt, sl, q, "bf16", "bf16", 0.09, 64)
    assert np.abs(lse[1] - want_lse[1]).max() < 1e-4


def test_latent_rows_past_two_gigabytes_and_graphs_on_two_streams(dev):
    g = _geom(1, 1, 576, 2, 64, 6 * (1 << 30) // 73728)
    pool = torch.zeros(g.pool_bytes(), dtype=torch.uint8, device=dev)
    rng = np.random.default_rng(8)
    sl = [100, 700]
    bt = np.full((2, 12), -1, np.int32)
    bt[0, :2] = [g.num_pages - 1, 5]
    bt[1, :11] = g.num_pages - 100 + np.arange(11)
    want = {int(p): od.encode_elements(rng.normal(size=36864), "bf16") for p in bt.reshape(-1) if p >= 0}
    for p, raw in want.items():
        pool[p * 73728:(p + 1) * 73728] = torch.from_numpy(raw).to(dev)
    small = _geom(1, 1, 576, 2, 64, len(want))
    order = {p: i for i, p in enumerate(want)}
    pool_h = np.concatenate(list(want.values()))
    bt_h = np.array([[order.get(int(x), -1) for x in row] for row in bt], np.int32)
    lo = _layout(g)
    b = tk.make_batch(torch.from_numpy(bt).to(dev), torch.tensor(sl, dtype=torch.int32, device=dev))
    q = torch.zeros(2, 70, 576, dtype=torch.bfloat16, device=dev)
    outs = [torch.zeros(2, 70, 512, dtype=torch.bfloat16, device=dev) for _ in range(2)]
    lses = [torch.zeros(2, 70, device=dev) for _ in range(2)]
    atts = [tk.make_attention(q, o, 1, 1, 0.04, value_dim=512, lse=l) for o, l in zip(outs, lses)]
    n = tk.check(tk.topkv_attend_workspace_bytes(lo, b, atts[0]))
    ws = [torch.empty(n, dtype=torch.uint8, device=dev) for _ in range(2)]
    call = lambda i, s: tk.check(tk.topkv_attend_layer(0, pool, lo, b, atts[i], q, outs[i], ws[i], n, s))
    call(0, torch.cuda.current_stream())
    torch.cuda.synchronize()
    side = torch.cuda.Stream(dev)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call(0, torch.cuda.current_stream())
    for seed in (1, 2):
        q_h = od.decode_elements(od.encode_elements(np.random.default_rng(seed).normal(size=2 * 70 * 576), "bf16"), "bf16").reshape(2, 70, 576)
        q.copy_(torch.from_numpy(q_h).to(torch.bfloat16))
        torch.cuda.synchronize()
        for _ in range(5):
            graph.replay()
            call(1, side)
        torch.cuda.synchronize()
        exact = od.attend(small, 0, pool_h, bt_h, sl, q_h, "bf16", "bf16", 0.04, 512)
        for o, l in zip(outs, lses):
            _check((o.double().cpu().numpy(), l.double().cpu().numpy()), exact)


def test_page_operators_in_a_graph(dev):
    """A captured turn (free, fork, extend) replayed from restored tables gives the same tables."""
    rng, g, sl, bt, ref, pool = _page_case(5, R=8, P=4, spare=20, maxlen=14)
    sl[1] = max(int(sl[1]), 1)
    s = _State(dev, g, sl, bt, ref, pool, False)
    in_place = tk.make_page_tables(s.out[2], *s.out)
    b2 = tk.make_batch(s.out[0], s.out[1])
    rows, parents, children = s.put(np.array([0, 3], np.int32)), s.put(np.array([1, 1], np.int32)), s.put(np.array([0, 3], np.int32))
    new = s.put(np.ones(8, np.int32))

    def turn(st):
        tk.check(tk.topkv_free_requests(s.lo, s.batch, s.tables, rows, 2, st))
        tk.check(tk.topkv_fork_requests(s.pool, s.lo, b2, in_place, parents, children, 2, s.ws, s.n, st))
        tk.check(tk.topkv_extend_requests(s.lo, b2, in_place, new, s.ws, s.n, st))
    side = torch.cuda.Stream(dev)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        turn(torch.cuda.current_stream())
    err = od.free_requests(g.P, bt, sl, ref, [0, 3])
    err |= od.fork_requests(g, pool, bt, sl, ref, [1, 1], [0, 3])
    err |= od.extend_requests(g.P, bt, sl, ref, [1] * 8)
    for _ in range(3):
        graph.replay()
    s.check(bt, sl, ref, pool, err)


def test_page_operators_on_large_tables(dev):
    """Tables that are copied by a launch of their own, and more rows than one CTA takes."""
    rng, g, sl, bt, ref, pool = _page_case(2, L=1, F=1, H=1, P=1, R=400, spare=40000, maxlen=30)
    s = _State(dev, g, sl, bt, ref, pool, False)
    rows = rng.permutation(400)[:150].astype(np.int32)
    tk.check(tk.topkv_free_requests(s.lo, s.batch, s.tables, s.put(rows), len(rows)))
    err = od.free_requests(g.P, bt, sl, ref, rows)
    s.check(bt, sl, ref, pool, err)
    s = _State(dev, g, sl, bt, ref, pool, False)
    new = rng.integers(0, 3, size=400).astype(np.int32)
    new[sl + new > bt.shape[1]] = 0
    tk.check(tk.topkv_extend_requests(s.lo, s.batch, s.tables, s.put(new), s.ws, s.n))
    err = od.extend_requests(g.P, bt, sl, ref, new)
    s.check(bt, sl, ref, pool, err)
    s = _State(dev, g, sl, bt, ref, pool, True)
    tk.check(tk.topkv_free_requests(s.lo, s.batch, s.tables, s.put(np.arange(400, dtype=np.int32)), 400))
    err = od.free_requests(g.P, bt, sl, ref, range(400))
    s.check(bt, sl, ref, pool, err)
    assert (ref == 0).all()


@pytest.mark.parametrize("seed", range(30))
def test_attend_random_cases(dev, seed):
    """Drawn shapes, types, pools, windows and lengths of both kinds of cache."""
    rng = np.random.default_rng(1000 + seed)
    pick = lambda xs: xs[int(rng.integers(0, len(xs)))]
    R = pick([1, 2, 5, 9])
    sl = rng.integers(0, pick([3, 70, 300, 900]) + 1, size=R)
    window, sinks = (pick([1, 33, 64, 200]), pick([0, 3, 70])) if rng.random() < 0.3 else (0, 0)
    P, style = pick([1, 2, 7, 16, 32, 64, 130]), pick(["page", "padded"])
    if seed % 3 == 2:
        D = pick([64, 192, 200, 320])
        _case(dev, 1, 1, pick([1, 9, 16, 30, 65]), D, P, sl, pick(["bf16", "fp16"]), Dv=pick([16, 64]), window=window, sinks=sinks,
              style=style, seed=seed, extra_cols=pick([0, 3]))
    else:
        kind = pick(["bf16", "fp16", "e4m3"])
        _case(dev, 2, pick([1, 2, 3]), pick([1, 2, 5, 18]), pick([16, 64, 96, 160]), P, sl, kind, pick(["bf16", "fp16"]) if kind == "e4m3" else kind,
              window=window, sinks=sinks, style=pick([style, "head", "plane"]), seed=seed, extra_cols=pick([0, 3]),
              out_order=pick(["rh", "hr"]), T=pick([-1, int(sl.sum())]) if window == 0 else -1)


def test_attend_negative_and_zero_scale(dev):
    rng = np.random.default_rng(4)
    sl = [300, 17]
    for F, Dv in ((2, 0), (1, 32)):
        bt, pages = _table(sl, 16, 1, 0, rng)
        g = _geom(F, 1, 64, 2, 16, pages)
        pool_h = _cache(g, bt, sl, "fp16", 0, rng)
        q = od.decode_elements(od.encode_elements(rng.normal(size=2 * 5 * 64), "fp16"), "fp16").reshape(2, 5, 64)
        for scale in (-0.3, 0.0):
            got = _run(dev, g, _layout(g), torch.from_numpy(pool_h).to(dev), bt, sl, q, "fp16", "fp16", scale, Dv)
            _check(got, od.attend(g, 0, pool_h, bt, sl, q, "fp16", "fp16", scale, Dv))


@pytest.mark.parametrize("kind,D,H,R,window,sinks", [("fp16", 64, 3, 207, 20, 3), ("e4m3", 128, 2, 230, 0, 0), ("fp16", 64, 9, 203, 60, 30), ("bf16", 256, 1, 600, 0, 0),
                                                     ("bf16", 80, 5, 301, 100, 40), ("fp16", 128, 8, 70, 1, 0)])
def test_attend_many_short_requests(dev, kind, D, H, R, window, sinks):
    """More short requests than CTAs at a time: a warp each, some of them empty, a last CTA that is not full."""
    rng = np.random.default_rng(R)
    sl = rng.integers(0, 41 if window == 0 else 300, size=R)
    sl[rng.integers(0, R, size=R // 10)] = 0
    _case(dev, 2, H, 2, D, 16, sl, kind, window=window, sinks=sinks, seed=R, extra_cols=0, ks=0.5 if kind == "e4m3" else 1.0)


# ------------------------------------------------------------------------- requests all of whose pages are unusable

@pytest.mark.parametrize("F,kind,H,G,D,Dv,sl", [
    (2, "bf16", 2, 3, 64, 0, [60, 130, 0]),          # finished by one CTA
    (2, "e4m3", 2, 3, 80, 0, [60, 130, 0]),
    (2, "bf16", 1, 2, 64, 0, [900, 4000, 70]),       # cut between CTAs and joined
    (2, "fp16", 2, 18, 256, 0, [900, 4000, 70]),
    (2, "e4m3", 1, 2, 128, 0, [900, 4000, 70]),
    (2, "fp16", 2, 2, 16, 0, [40] * 700),            # a warp each
    (2, "e4m3", 2, 2, 64, 0, [40] * 700),
    (1, "bf16", 1, 20, 192, 128, [60, 130, 0]),
    (1, "fp16", 1, 70, 128, 128, [900, 4000, 70]),
    (1, "bf16", 1, 16, 576, 512, [900, 4000, 70]),
])
def test_attend_requests_without_a_usable_page(dev, F, kind, H, G, D, Dv, sl):
    """A page outside the pool counts as not visible; a request that has no other sees nothing, which is
    zeros and a log-sum-exp of minus infinity. The others are not touched by it."""
    rng = np.random.default_rng(31)
    io = "bf16" if kind == "e4m3" else kind
    bt, pages = _table(sl, 16, 1, 0, rng)
    g = _geom(F, H, D, 1 if kind == "e4m3" else 2, 16, pages)
    pool_h = _cache(g, bt, sl, kind, 0, rng)
    q = od.decode_elements(od.encode_elements(rng.normal(size=len(sl) * H * G * D), io), io).reshape(len(sl), H * G, D)
    want = od.attend(g, 0, pool_h, bt, sl, q, kind, io, 0.1, Dv)
    bad = [1] if len(sl) < 10 else list(range(3, len(sl), 7))
    broken = bt.copy()
    broken[bad] = pages + 1
    out, lse = _run(dev, g, _layout(g), torch.from_numpy(pool_h).to(dev), broken, sl, q, kind, io, 0.1, Dv)
    assert tk.topkv_device_error_flags() == 2
    tk.check(tk.topkv_reset_device_error_flags())
    assert (out[bad] == 0).all() and (lse[bad] == -np.inf).all()
    good = [r for r in range(len(sl)) if r not in bad]
    _check((out[good], lse[good]), tuple(x[good] for x in want))


@pytest.mark.parametrize("sl", [[70, 40], [3000, 40]])
def test_attend_infinite_keys_beside_unusable_pages(dev, sl):
    """Scores of minus infinity are scores: a request that sees nothing else has no finite result, also where
    some of its pages are unusable, whole or cut between CTAs."""
    rng = np.random.default_rng(32)
    for F, Dv in ((2, 0), (1, 16)):
        bt, pages = _table(sl, 16, 1, 0, rng)
        g = _geom(F, 1, 16, 2, 16, pages)
        pool = np.zeros(g.pool_bytes(), np.uint8)
        ones = od.encode_elements(np.ones(16), "fp16")
        for p in range(pages):
            for c in range(F):
                for t in range(16):
                    a = od.row_offset(g, 0, p, c, t, 0)
                    pool[a:a + 32] = ones
                    if c == 0:
                        pool[a:a + 2] = od.encode_elements(np.array([-np.inf]), "fp16")
        broken = bt.copy()
        broken[0, 1:] = -1                                   # request 0 keeps its first page only
        out, lse = _run(dev, g, _layout(g), torch.from_numpy(pool).to(dev), broken, sl, np.ones((2, 3, 16)), "fp16", "fp16", 1.0, Dv)
        assert tk.topkv_device_error_flags() == 2
        tk.check(tk.topkv_reset_device_error_flags())
        assert np.isnan(out[..., 0]).all() and (lse == -np.inf).all()


# ------------------------------------------------------------------------- appends behind refusals

def _append_oracle(g, pool, bt, before, after, new, layer, rows):
    """One new token per request that asked for one, `rows` in request order; refused ones are skipped."""
    at, row = 0, rows.reshape(-1, g.F, g.h_kv, g.d_h * g.b_p)
    for r in range(len(after)):
        wanted = int(before[r]) + int(new[r])
        if wanted > 0:
            if new[r] and after[r] == wanted:
                i = wanted - 1
                for c in range(g.F):
                    for h in range(g.h_kv):
                        a = od.row_offset(g, layer, int(bt[r, i // g.P]), c, i % g.P, h)
                        pool[a:a + g.d_h * g.b_p] = row[at, c, h]
            at += 1


@pytest.mark.parametrize("held", [0, 2])   # pages that somebody else has: without them there are enough
@pytest.mark.parametrize("captured", [False, True])
def test_decode_cache_with_too_few_pages(dev, captured, held):
    """Turns in a pool that runs out of pages: requests are refused, freed and extended again, on a side
    stream, call by call or as a graph that holds the extension and the appends of a turn."""
    from paper_2607_28633_b200 import session
    rng = np.random.default_rng(5)
    g = _geom(2, 2, 64, 2, 4, 9, L=2)
    bt = np.full((6, 6), -1, np.int32)
    sl = np.array([4, 8, 3, 6, 0, 0], np.int32)
    bt[0, 0], bt[1, :2], bt[2, 0], bt[3, :2] = 7, (2, 5), 0, (8, 1)
    lo = tk.make_layout(2, 2, 2, 64, 2, 4, 9, wire_layer_stride=6 * 512)
    pool_h = rng.integers(0, 256, g.pool_bytes(), dtype=np.uint8)
    pool = torch.from_numpy(pool_h).to(dev)
    cache = session.DecodeCache(pool, lo, torch.from_numpy(bt).to(dev), torch.from_numpy(sl).to(dev))
    cache.ref_counts[3:3 + held] += 1
    ref = cache.ref_counts.cpu().numpy().copy()
    s = torch.cuda.Stream(dev)
    d_new = torch.zeros(6, dtype=torch.int32, device=dev)
    d_kv = [torch.zeros(6 * 512, dtype=torch.uint8, device=dev) for _ in range(2)]
    rows = torch.zeros(1, dtype=torch.int32, device=dev)

    def turn(stream):
        cache.extend(d_new, stream)
        for layer in range(2):
            cache.append(layer, d_kv[layer], stream)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    err = 0
    for n, (new, ended) in enumerate([([1, 1, 1, 1, 0, 0], 1), ([0, 0, 1, 1, 0, 0], 4), ([1, 0, 1, 2, 1, 0], 3), ([1, 1, 1, 0, 1, 1], 5),
                                      ([3, 0, 2, 0, 1, 1], 0), ([4, 4, 1, 0, 1, 1], 2), ([1, 1, 1, 1, 1, 1], 5)]):
        new = np.array(new, np.int32)
        d_new.copy_(torch.from_numpy(new))
        kv = [rng.integers(0, 256, 6 * 512, dtype=np.uint8) for _ in range(2)]
        for d, h in zip(d_kv, kv):
            d.copy_(torch.from_numpy(h))
        rows.fill_(ended)
        torch.cuda.synchronize()
        if captured and n == 1:
            with torch.cuda.graph(graph, stream=s):
                turn(torch.cuda.current_stream())
        if captured and n >= 1:
            graph.replay()
        else:
            turn(s)
        torch.cuda.synchronize()
        before = sl.copy()
        err |= od.extend_requests(4, bt, sl, ref, new)
        for layer in range(2):
            _append_oracle(g, pool_h, bt, before, sl, new, layer, kv[layer])
        for got, want in ((cache.block_table, bt), (cache.seq_lens, sl), (cache.ref_counts, ref), (pool, pool_h)):
            assert np.array_equal(got.cpu().numpy(), want), n
        cache.free(rows, s)
        err |= od.free_requests(4, bt, sl, ref, [ended])
    torch.cuda.synchronize()
    assert err == tk.topkv_device_error_flags() == (8 if held else 0)
    tk.check(tk.topkv_reset_device_error_flags())


def test_decode_cache_frees_and_forks_between_extend_and_append(dev):
    """A refused request is freed or forked before the appends: places in the slab and tokens stay right."""
    from paper_2607_28633_b200 import session
    g = _geom(2, 1, 8, 2, 4, 4)
    lo = tk.make_layout(1, 2, 1, 8, 2, 4, 4)
    mark = lambda cache, r, i: {int(x) for c in range(2) for x in cache.pool.cpu().numpy()[
        od.row_offset(g, 0, int(cache.block_table[r, i // 4]), c, i % 4, 0):][:16]}
    put = lambda *x: torch.tensor(x, dtype=torch.int32, device=dev)
    slab = lambda *m: torch.tensor(m, dtype=torch.uint8, device=dev)[:, None].expand(len(m), 32).contiguous()

    def start():
        cache = session.DecodeCache(torch.full((g.pool_bytes(),), 9, dtype=torch.uint8, device=dev), lo,
                                    put(0, -1, 1, -1, 2, -1, -1, -1).view(4, 2), put(4, 3, 4, 0))
        cache.extend(put(1, 1, 1, 0), None)                  # row 2 is refused
        return cache
    cache = start()
    cache.free(put(0, -3, 77), None)
    cache.append(0, slab(21, 22), None)
    torch.cuda.synchronize()
    assert cache.seq_lens.tolist() == [0, 4, 4, 0] and mark(cache, 1, 3) == {21} and mark(cache, 2, 3) == {9}
    cache = start()
    cache.fork(put(2, 1, 2), put(3, 3, 0), None)             # the refused parent's child is refused as well
    cache.append(0, slab(31, 32, 33, 34), None)
    torch.cuda.synchronize()
    assert cache.seq_lens.tolist() == [5, 4, 4, 4]
    assert [mark(cache, r, i) for r, i in ((0, 4), (0, 3), (1, 3), (2, 3), (3, 3))] == [{31}, {9}, {32}, {9}, {9}]
    torch.cuda.synchronize()
    assert tk.topkv_device_error_flags() == 8 | 2            # pages; rows outside the table, a row named twice
    tk.check(tk.topkv_reset_device_error_flags())


def test_decode_cache_of_more_rows_than_a_copy_counts_itself(dev):
    from paper_2607_28633_b200 import session
    g = _geom(1, 1, 16, 2, 4, 6)
    bt, sl = torch.full((1100, 2), -1, dtype=torch.int32, device=dev), torch.zeros(1100, dtype=torch.int32, device=dev)
    bt[3, 0], bt[1090, 0], sl[3], sl[1090] = 4, 2, 2, 3
    lo = tk.make_layout(1, 1, 1, 16, 2, 4, 6)
    cache = session.DecodeCache(torch.zeros(g.pool_bytes(), dtype=torch.uint8, device=dev), lo, bt, sl)
    slab = lambda *m: torch.tensor(m, dtype=torch.uint8, device=dev)[:, None].expand(len(m), 32).contiguous()
    at = lambda page, t: cache.pool.view(6, 4, 32)[page, t].unique().tolist()
    s = torch.cuda.Stream(dev)
    kv = slab(1, 2), slab(3, 4, 5), slab(6, 7)
    new = torch.zeros(1100, dtype=torch.int32, device=dev)
    new[1090] = new[1050] = 1
    torch.cuda.synchronize()
    cache.append(0, kv[0], s)
    torch.cuda.synchronize()
    assert at(4, 1) == [1] and at(2, 2) == [2] and at(4, 0) == [0]
    cache.extend(new, s)                                     # row 1050 takes page 0
    cache.append(0, kv[1], s)
    torch.cuda.synchronize()
    assert [at(4, 1), at(0, 0), at(2, 2), at(2, 3)] == [[1], [4], [2], [5]]
    cache.free(torch.tensor([3], dtype=torch.int32, device=dev), s)
    cache.append(0, kv[2], s)
    torch.cuda.synchronize()
    assert at(0, 0) == [6] and at(2, 3) == [7]


def test_decode_cache_attends_in_a_graph_beside_larger_calls(dev):
    """A graph that holds an attention is replayed after a call of another kind has asked for a larger
    workspace and the memory around has been handed out; streams by handle, and none."""
    from paper_2607_28633_b200 import session
    rng = np.random.default_rng(14)
    sl = [900, 40, 2000]
    bt, pages = _table(sl, 16, 1, 0, rng)
    g = _geom(2, 2, 64, 2, 16, pages)
    pool_h = _cache(g, bt, sl, "bf16", 0, rng)
    cache = session.DecodeCache(torch.from_numpy(pool_h).to(dev), _layout(g), torch.from_numpy(bt).to(dev),
                                torch.tensor(sl, dtype=torch.int32, device=dev))
    q = torch.zeros(3, 4, 64, dtype=torch.bfloat16, device=dev)
    wide = torch.randn(3, 32, 64, device=dev).to(torch.bfloat16)
    out, wide_out, lse = torch.zeros_like(q), torch.zeros_like(wide), torch.zeros(3, 4, device=dev)
    torch.cuda.synchronize()
    cache.attend(0, q, out, 0.125, None, lse=lse)
    side = torch.cuda.Stream(dev)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        cache.attend(0, q, out, 0.125, torch.cuda.current_stream(), lse=lse)
    cache.attend(0, wide, wide_out, 0.125, side.cuda_stream)
    torch.cuda.synchronize()
    others = [torch.full((1 << 18,), 3, dtype=torch.uint8, device=dev) for _ in range(64)]
    q_h = od.decode_elements(od.encode_elements(rng.normal(size=3 * 4 * 64), "bf16"), "bf16").reshape(3, 4, 64)
    q.copy_(torch.from_numpy(q_h).to(torch.bfloat16))
    torch.cuda.synchronize()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    _check((out.double().cpu().numpy(), lse.double().cpu().numpy()), od.attend(g, 0, pool_h, bt, sl, q_h, "bf16", "bf16", 0.125))
    assert all((x == 3).all() for x in others)


@pytest.mark.parametrize("D,long", [(64, 0), (128, 0), (128, 3000)])
def test_attend_bf16_weights_keep_sixteen_bits(dev, D, long):
    """Two values that nearly cancel: half a step of an 8-bit weight would be far more than the result's
    rounding. A weight is split into two bf16 values, the second of what the first leaves: 2^-8 of 2^-8."""
    heads = 16
    n = 2 + long                                             # further tokens weigh nothing
    bt, pages = _table([n], 16, 1, 0, np.random.default_rng(0))
    g = _geom(2, 1, D, 2, 16, pages)
    pool = np.zeros(g.pool_bytes(), np.uint8)
    q = np.zeros((1, heads, D))
    q[0, :, 0], q[0, :, 1] = -np.arange(1, heads + 1) / 8, 1.0
    w = np.exp(q[0, :, 0])
    k, v = np.zeros((n, D)), np.zeros((n, D))
    k[1, 0], k[2:, 1] = 1.0, -200.0
    v[0, :heads], v[1, :heads] = od.decode_elements(od.encode_elements(w, "bf16"), "bf16"), -1.0
    for i in range(n):
        for c, x in ((0, k), (1, v)):
            a = od.row_offset(g, 0, int(bt[0, i // 16]), c, i % 16, 0)
            pool[a:a + 2 * D] = od.encode_elements(x[i], "bf16")
    got = _run(dev, g, _layout(g), torch.from_numpy(pool).to(dev), bt, [n], q, "bf16", "bf16", 1.0)
    want = od.attend(g, 0, pool, bt, [n], q, "bf16", "bf16", 1.0, weight_step=2.0 ** -16)
    coarse = od.attend(g, 0, pool, bt, [n], q, "bf16", "bf16", 1.0)
    _check(got, want)
    own = np.arange(heads)
    if not long:  # the bound would not let 8 bits through (scores of -200 alone allow 2 * 136 * 2^-23 * 200 = 0.0065)
        assert (want[2][0, own, own] < coarse[2][0, own, own] / 4).all()


@pytest.mark.parametrize("kind,window,sinks,rows", [("e4m3", 0, 0, 4), ("e4m3", 33, 5, 4), ("fp16", 64, 4, 6), ("bf16", 1, 0, 4)])
def test_decode_cache_attends_with_windows_and_eight_bits(dev, kind, window, sinks, rows):
    """One object for layers of both kinds: all tokens, and a window with first tokens; rows to spare."""
    from paper_2607_28633_b200 import session
    rng = np.random.default_rng(window + rows)
    sl = [700, 40, 0, 1300]
    io = "bf16" if kind == "e4m3" else kind
    bt, pages = _table(sl, 16, 1, 0, rng)
    g = _geom(2, 2, 64, 1 if kind == "e4m3" else 2, 16, pages)
    pool_h = _cache(g, bt, sl, kind, 0, rng)
    s = torch.cuda.Stream(dev)
    cache = session.DecodeCache(torch.from_numpy(pool_h).to(dev), _layout(g), torch.from_numpy(bt).to(dev),
                                torch.tensor(sl, dtype=torch.int32, device=dev), rows=rows)
    sl, bt = sl + [0] * (rows - 4), np.concatenate([bt, np.full((rows - 4, bt.shape[1]), -1, np.int32)])
    q_h = od.decode_elements(od.encode_elements(rng.normal(size=rows * 6 * 64), io), io).reshape(rows, 6, 64)
    q = torch.from_numpy(q_h).to(dev).to(TORCH[io])
    ks, vs = (0.5, 2.0) if kind == "e4m3" else (1.0, 1.0)
    for w, n in ((0, 0), (window, sinks)):
        out, lse = torch.full_like(q, 7), torch.zeros(rows, 6, device=dev)
        torch.cuda.synchronize()
        cache.attend(0, q, out, 0.125, s, cache_type=TYPE[kind], window_tokens=w, sink_tokens=n, k_scale=ks, v_scale=vs, lse=lse)
        torch.cuda.synchronize()
        g.window = w
        _check((out.double().cpu().numpy(), lse.double().cpu().numpy()), od.attend(g, 0, pool_h, bt, sl, q_h, kind, io, 0.125, 0, n, ks, vs))

"""CPU checks of the decode side's entry points (attention over the paged cache, page operators):
refusals, workspace sizes, and the oracle's own definitions against hand-derived values. Nothing
is launched: what is acceptable ends in TOPKV_ERR_CUDA on a box without a GPU."""
import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import __graft_entry__ as entry
from oracle import Geom, decode as od
from paper_2607_28633_b200 import binding as tk

INVALID, LAYER, ALIGN, CAP, LAYOUT, CUDA = (tk.TOPKV_ERR_INVALID_ARG, tk.TOPKV_ERR_LAYER_RANGE,
                                            tk.TOPKV_ERR_ALIGNMENT, tk.TOPKV_ERR_CAPACITY,
                                            tk.TOPKV_ERR_UNSUPPORTED_LAYOUT, tk.TOPKV_ERR_CUDA)


class _Fake:
    def __init__(self, addr, shape):
        self._a, self.shape, self.ndim = addr, shape, len(shape)

    def data_ptr(self):
        return self._a


@pytest.fixture(scope="module", autouse=True)
def _built():
    entry.build()
    if torch.cuda.is_available():
        pytest.skip("fake addresses must never reach a real device")


def _batch(R=4, maxp=64, T=-1, **kw):
    return tk.make_batch(_Fake(0x10000, (R, maxp)), _Fake(0x20000, (R,)), T, **kw)


def _attention(Hq=64, D=128, cache=None, io=None, Dv=0, R=4, **kw):
    a = tk.topkv_attention()
    a.struct_size = ctypes.sizeof(a)
    a.cache_type = tk.TOPKV_TYPE_BF16 if cache is None else cache
    a.io_type = tk.TOPKV_TYPE_BF16 if io is None else io
    a.num_q_heads, a.value_dim, a.scale, a.k_scale, a.v_scale = Hq, Dv, 0.1, 1.0, 1.0
    a.q_head_stride, a.out_head_stride = 2 * D, 2 * (Dv or D)
    a.q_request_stride, a.out_request_stride = Hq * a.q_head_stride, Hq * a.out_head_stride
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _gqa(H=8, D=128, E=2, P=16, L=2, N=100):
    return tk.make_layout(L, 2, H, D, E, P, N)


def _attend(lo, b, a, layer=0, pool=0x7000000, q=0x8000000, out=0x9000000, ws=0xA000000, n=1 << 40):
    return tk.topkv_attend_layer(layer, pool, lo, b, a, q, out, ws, n)


def test_struct_sizes():
    assert ctypes.sizeof(tk.topkv_attention) == 80
    assert ctypes.sizeof(tk.topkv_page_tables) == 40


def test_attend_accepts_what_the_header_allows():
    e4 = tk.TOPKV_TYPE_E4M3
    for lo, b, a in [
        (_gqa(), _batch(), _attention()),
        (_gqa(), _batch(R=3000), _attention()),                                # no cu_seq_lens needed
        (_gqa(H=1, D=64), _batch(), _attention(Hq=1, D=64)),
        (_gqa(H=5, D=256), _batch(), _attention(Hq=35, D=256)),
        (_gqa(E=1), _batch(), _attention(cache=e4, k_scale=0.5, v_scale=3.0)),
        (_gqa(E=1), _batch(), _attention(cache=e4, io=tk.TOPKV_TYPE_FP16)),
        (_gqa(), _batch(window_tokens=128), _attention(sink_tokens=4)),
        (_gqa(), _batch(flags=3), _attention()),
        (_gqa(), _batch(), _attention(q_request_stride=0)),                    # one query for all requests
        (_gqa(), _batch(), _attention(out_request_stride=256, out_head_stride=4 * 256)),   # [heads][requests]
    ]:
        assert _attend(lo, b, a) == CUDA
    empty = _batch(R=0)
    assert _attend(_gqa(), empty, _attention()) == tk.TOPKV_OK


def test_attend_refusals():
    lo, b = _gqa(), _batch()
    for status, change in [
        (INVALID, dict(struct_size=8)), (INVALID, dict(reserved=1)), (INVALID, dict(cache_type=0)),
        (INVALID, dict(cache_type=4)), (INVALID, dict(io_type=3)), (INVALID, dict(io_type=tk.TOPKV_TYPE_FP16)),
        (INVALID, dict(num_q_heads=0)), (INVALID, dict(num_q_heads=63)), (INVALID, dict(value_dim=64)),
        (INVALID, dict(scale=float("nan"))), (INVALID, dict(scale=float("inf"))), (INVALID, dict(k_scale=2.0)),
        (INVALID, dict(v_scale=0.5)), (INVALID, dict(sink_tokens=1 << 31)), (INVALID, dict(q_head_stride=-16)),
        (ALIGN, dict(q_head_stride=264)), (ALIGN, dict(out_request_stride=64 * 256 + 8)), (ALIGN, dict(lse=2)),
        (INVALID, dict(out_head_stride=128)), (INVALID, dict(out_request_stride=0)),
        (INVALID, dict(out_request_stride=63 * 256)), (INVALID, dict(q_request_stride=1 << 41)),
    ]:
        assert _attend(lo, b, _attention(**change)) == status, change
    a = _attention()
    assert _attend(lo, b, a, layer=2) == LAYER and _attend(lo, b, a, layer=-1) == LAYER
    for name in ("pool", "q", "out"):
        assert _attend(lo, b, a, **{name: None}) == INVALID
        assert _attend(lo, b, a, **{name: 0x7000008}) == ALIGN
    assert _attend(lo, b, a, ws=None) == INVALID and _attend(lo, b, a, ws=0xA000008) == ALIGN
    need = tk.topkv_attend_workspace_bytes(lo, b, a)
    assert need > 0 and _attend(lo, b, a, n=need - 1) == CAP and _attend(lo, b, a, n=need) == CUDA
    short = _batch(maxp=16)                              # 256 tokens: never split, no workspace
    assert tk.topkv_attend_workspace_bytes(lo, short, a) == 0 and _attend(lo, short, a, ws=None, n=0) == CUDA
    assert _attend(_gqa(E=1), b, a) == LAYOUT and _attend(lo, b, _attention(cache=tk.TOPKV_TYPE_E4M3)) == LAYOUT
    assert _attend(_gqa(D=264), b, _attention(D=264)) == LAYOUT
    assert _attend(_gqa(H=2, D=24, E=1), b, _attention(D=24, cache=tk.TOPKV_TYPE_E4M3)) == LAYOUT
    # one plane, several heads: neither grouped heads nor a latent row
    assert _attend(tk.make_layout(1, 1, 2, 128, 2, 16, 9), b, _attention(Dv=64)) == LAYOUT
    bad = _batch(); bad.flags = 4
    assert _attend(lo, bad, a) == INVALID
    bad = _batch(); bad.seq_lens = None
    assert _attend(lo, bad, a) == INVALID
    bad = _batch(); bad.block_table = None
    assert _attend(lo, bad, a) == INVALID
    bad = _batch(maxp=1 << 28)
    assert _attend(lo, bad, a) == INVALID
    bad = _batch(); bad.seq_lens = 0x20002
    assert _attend(lo, bad, a) == ALIGN
    assert tk.topkv_attend_workspace_bytes(lo, bad, a) == ALIGN


def test_make_attention_checks_shapes():
    q = torch.zeros(3, 8, 64, dtype=torch.bfloat16)
    out = torch.zeros(3, 8, 64, dtype=torch.bfloat16)
    T = tk.TOPKV_TYPE_BF16
    a = tk.make_attention(q, out, T, T, 0.125, lse=torch.zeros(3, 8))
    assert (a.q_request_stride, a.q_head_stride, a.num_q_heads) == (1024, 128, 8)
    for bad in (dict(q=q.float()), dict(q=q.transpose(1, 2)), dict(out=out[:2]), dict(lse=torch.zeros(8, 3)),
                dict(lse=torch.zeros(3, 8, dtype=torch.float64)), dict(q=q[0])):
        with pytest.raises(ValueError):
            tk.make_attention(**{**dict(q=q, out=out, cache_type=T, io_type=T, scale=1.0), **bad})


def _tables(**kw):
    t = tk.make_page_tables(0x30000, 0x40000, 0x50000, 0x60000)
    for k, v in kw.items():
        setattr(t, k, v)
    return t


def test_page_operator_refusals():
    lo, b, t, ws, n = _gqa(), _batch(), _tables(), 0xA000000, 1 << 30
    pool = 0x7000000
    calls = {
        "extend": lambda lo=lo, b=b, t=t, x=0x70000, ws=ws, n=n: tk.topkv_extend_requests(lo, b, t, x, ws, n),
        "fork": lambda lo=lo, b=b, t=t, x=0x70000, ws=ws, n=n: tk.topkv_fork_requests(pool, lo, b, t, x, 0x80000, 3, ws, n),
        "free": lambda lo=lo, b=b, t=t, x=0x70000, ws=ws, n=n: tk.topkv_free_requests(lo, b, t, x, 3),
        "compact": lambda lo=lo, b=b, t=t, x=0x70000, ws=ws, n=n: tk.topkv_compact_pages(pool, lo, b, t, x, 0x80000, ws, n),
    }
    for name, call in calls.items():
        assert call() == CUDA, name
        assert call(x=None) == INVALID and call(x=0x70002) == ALIGN, name
        assert call(t=_tables(struct_size=8)) == INVALID and call(t=_tables(reserved=1)) == INVALID, name
        for field in ("ref_counts", "block_table_out", "seq_lens_out", "ref_counts_out"):
            assert call(t=_tables(**{field: None})) == INVALID and call(t=_tables(**{field: 0x40002})) == ALIGN, (name, field)
        assert call(b=_batch(window_tokens=16)) == INVALID, name
        if name != "free":
            assert call(ws=None) == INVALID and call(ws=0xA000004) == ALIGN, name
            assert call(n=15) == CAP, name
        big = _gqa(N=1 << 31)
        assert call(lo=big) == LAYOUT, name
        if name != "compact":
            assert call(b=_batch(R=0)) == tk.TOPKV_OK and call(b=_batch(maxp=0)) == tk.TOPKV_OK, name
    fork = lambda n, k: tk.topkv_fork_requests(pool, lo, b, t, 0x70000, 0x80000, n, ws, k)
    need = tk.topkv_page_workspace_bytes(lo, b, 1000)
    assert need >= 4 * (5 * 1000 + 4) and fork(1000, need) == CUDA and fork(1000, need - 4) == CAP
    assert fork(-1, need) == INVALID
    assert tk.topkv_page_workspace_bytes(lo, b, -1) == INVALID
    assert tk.topkv_free_requests(lo, b, t, 0x70000, -1) == INVALID
    deep = _gqa(L=70000)
    assert tk.topkv_fork_requests(pool, deep, b, t, 0x70000, 0x80000, 1, ws, n) == LAYOUT
    cp = tk.topkv_copy_pages
    assert cp(0, 2, pool, lo, 0x70000, 0x80000, 5) == CUDA and cp(0, 0, pool, lo, 0x70000, 0x80000, 5) == tk.TOPKV_OK
    assert cp(0, 2, pool, lo, None, None, 0) == tk.TOPKV_OK
    for st, args in [(LAYER, (0, 3, pool, lo, 1 << 16, 1 << 17, 5)), (LAYER, (-1, 1, pool, lo, 1 << 16, 1 << 17, 5)),
                     (INVALID, (0, 2, None, lo, 1 << 16, 1 << 17, 5)), (INVALID, (0, 2, pool, lo, None, 1 << 17, 5)),
                     (INVALID, (0, 2, pool, lo, 1 << 16, 1 << 17, -1)), (ALIGN, (0, 2, pool, lo, 1 << 16, 6, 5)),
                     (ALIGN, (0, 2, pool + 8, lo, 1 << 16, 1 << 17, 5))]:
        assert cp(*args) == st, args


def test_nothing_is_launched_here():
    before = tk.topkv_kernel_launch_count()
    assert _attend(_gqa(), _batch(), _attention()) == CUDA
    assert tk.topkv_kernel_launch_count() == before


# ---- the oracle's definitions ------------------------------------------------------------------------

def test_oracle_element_types():
    assert od.E4M3[0x38] == 1.0 and od.E4M3[0x7E] == 448.0 and od.E4M3[1] == 2.0 ** -9 and np.isnan(od.E4M3[0xFF])
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(t, od.E4M3, equal_nan=True)
    x = np.random.default_rng(0).normal(size=4000) * np.exp2(np.random.default_rng(1).integers(-12, 9, size=4000))
    for kind, dt in (("bf16", torch.bfloat16), ("fp16", torch.float16), ("e4m3", torch.float8_e4m3fn)):
        y = x.clip(-440, 440) if kind == "e4m3" else x
        f32 = torch.from_numpy(y).float()
        assert np.array_equal(od.encode_elements(f32.double().numpy(), kind), f32.to(dt).view(torch.uint8).numpy())


def test_oracle_attention_by_hand():
    """Two tokens, one head: scores 0 and ln 3 give the weights 1/4 and 3/4."""
    g = Geom(L=1, F=2, h_kv=1, d_h=8, b_p=2, P=1, num_pages=4)
    pool = np.zeros(g.pool_bytes(), dtype=np.uint8)
    def put(page, plane, row):
        a = od.row_offset(g, 0, page, plane, 0, 0)
        pool[a:a + 16] = od.encode_elements(np.array(row, dtype=np.float64), "fp16")
    put(3, 0, [0] * 8); put(1, 0, [1] + [0] * 7)
    put(3, 1, [4] * 8); put(1, 1, [8] * 8)
    q = np.zeros((1, 1, 8)); q[0, 0, 0] = np.log(3.0)
    out, lse, _, _ = od.attend(g, 0, pool, [[3, 1]], [2], q, "fp16", "fp16", 1.0)
    assert np.allclose(out, 7.0) and np.allclose(lse, np.log(4.0))
    out, lse, _, _ = od.attend(g, 0, pool, [[3, 1]], [0], q, "fp16", "fp16", 1.0)
    assert (out == 0).all() and (lse == -np.inf).all()
    assert od.visible(10, 3, 2).tolist() == [0, 1, 7, 8, 9] and od.visible(4, 3, 2).tolist() == [0, 1, 2, 3]
    assert od.visible(2, 3, 2).tolist() == [0, 1] and od.visible(5, 0, 2).tolist() == [0, 1, 2, 3, 4]


def test_oracle_page_operators_by_hand():
    g = Geom(L=1, F=1, h_kv=1, d_h=8, b_p=2, P=2, num_pages=8)
    pool = np.arange(g.pool_bytes(), dtype=np.uint8)
    bt = np.array([[5, 2, -1], [7, -1, -1], [-1, -1, -1]], np.int32)
    sl = np.array([3, 2, 0], np.int32)
    ref = np.array([0, 0, 1, 0, 0, 1, 0, 1], np.int32)
    assert od.fork_requests(g, pool, bt, sl, ref, [0], [2]) == 0
    assert bt[2].tolist() == [5, 0, -1] and sl[2] == 3 and ref.tolist() == [1, 0, 1, 0, 0, 2, 0, 1]
    assert np.array_equal(pool[:16], np.arange(64, 80)) and np.array_equal(pool[16:32], np.arange(16, 32))
    assert od.extend_requests(2, bt, sl, ref, [2, 0, 1]) == 0
    assert bt.tolist() == [[5, 2, 1], [7, -1, -1], [5, 0, -1]] and sl.tolist() == [5, 2, 4]
    assert od.free_requests(2, bt, sl, ref, [0, 0]) == 0
    assert ref.tolist() == [1, 0, 0, 0, 0, 1, 0, 1] and bt[0].tolist() == [-1] * 3 and sl[0] == 0
    err, n, to = od.compact_pages(g, pool, bt, sl, ref)
    assert (err, n) == (0, 3) and to.tolist() == [0, -1, -1, -1, -1, 1, -1, 2]
    assert bt.tolist() == [[-1] * 3, [2, -1, -1], [1, 0, -1]] and ref.tolist() == [1, 1, 1, 0, 0, 0, 0, 0]
    assert np.array_equal(pool[32:64], np.arange(5 * 32, 6 * 32)) and np.array_equal(pool[64:96], np.arange(7 * 32, 8 * 32) % 256)
    # eight pages, three in use: 3 + 1 + 1 more fit exactly, then nothing is left
    assert od.extend_requests(2, bt, sl, ref, [6, 2, 2]) == 0
    assert bt.tolist() == [[3, 4, 5], [2, 6, -1], [1, 0, 7]] and ref.tolist() == [1] * 8 and sl.tolist() == [6, 4, 6]
    assert od.extend_requests(2, bt, sl, ref, [0, 2, 0]) == od.ERR_PAGES
    assert bt[1].tolist() == [2, 6, -1] and sl.tolist() == [6, 4, 6]
    assert od.extend_requests(2, bt, sl, ref, [0, 3, 0]) == od.ERR_TABLE       # longer than its row


@pytest.mark.parametrize("seed", range(3))
def test_entry_points_survive_random_descriptors(seed):
    """Random, mostly malformed descriptors with fake addresses: a status from the documented set every
    time, and nothing launched."""
    rng = np.random.default_rng(seed)
    known = {tk.TOPKV_OK, INVALID, LAYER, ALIGN, CAP, LAYOUT, CUDA}
    pick = lambda xs: xs[int(rng.integers(0, len(xs)))]
    before = tk.topkv_kernel_launch_count()
    seen = set()
    for _ in range(100):
        F, H, D, E = pick([(2, 8, 128, 2), (2, 1, 64, 1), (1, 1, 576, 2), (2, 3, 256, 2), (1, 2, 64, 2), (2, 2, 24, 1)])
        lo = tk.topkv_layout()
        try:
            lo = tk.make_layout(pick([1, 5, 80]), F, H, D, E, pick([1, 16, 64, 1000]), pick([1, 100, 1 << 20]))
        except tk.TopkvError:
            pass
        b = _batch(R=pick([0, 1, 16, 5000]), maxp=pick([0, 1, 64, 5000]), T=pick([-1, 0, 100, 1 << 40]))
        b.window_tokens = pick([0, 0, 1, 128, -1])
        narrow = E == 1
        a = _attention(Hq=H * pick([1, 8, 17]), D=D, cache=3 if narrow else pick([1, 2]), Dv=pick([0, 0, 512, 16, D]),
                       sink_tokens=pick([0, 4, 0x7fffffff]))
        a.io_type = a.cache_type if not narrow else pick([1, 2])
        t = _tables()
        for _ in range(pick([0, 1, 2])):
            k = pick(range(10))
            if k == 0: lo.pool_page_stride += pick([8, 16, -16])
            elif k == 1: lo.page_tokens = pick([0, 0xffffffff, 7])
            elif k == 2: lo.num_pool_pages = pick([0, -1, 1 << 33])
            elif k == 3: a.num_q_heads = pick([0, 7, 65535, 1 << 31])
            elif k == 4: a.out_head_stride = pick([0, 16, 1 << 50, -16])
            elif k == 5: a.scale = pick([0.0, -1.0, float("nan")])
            elif k == 6: b.num_requests = pick([-1, 1 << 30])
            elif k == 7: b.max_pages_per_req = pick([-1, 1 << 30])
            elif k == 8: t.ref_counts = pick([None, 3])
            elif k == 9: lo.head_dim = pick([0, 7, 1 << 20])
        n, off = pick([0, 1 << 12, 1 << 40]), pick([0, 0, 8])
        for st in (_attend(lo, b, a, layer=pick([0, 0, 7]), pool=0x7000000 + off, n=n),
                   min(0, tk.topkv_attend_workspace_bytes(lo, b, a)), min(0, tk.topkv_page_workspace_bytes(lo, b, pick([0, 9, -1]))),
                   tk.topkv_extend_requests(lo, b, t, 0x70000, 0xA000000 + off, n),
                   tk.topkv_fork_requests(0x7000000, lo, b, t, 0x70000, 0x80000, pick([0, 5, -1]), 0xA000000, n),
                   tk.topkv_free_requests(lo, b, t, 0x70000, pick([0, 5, -1])),
                   tk.topkv_compact_pages(0x7000000, lo, b, t, 0x70000, 0x80000, 0xA000000, n),
                   tk.topkv_copy_pages(0, 1, 0x7000000 + off, lo, 0x70000, 0x80000, 3)):
            assert st in known, st
            seen.add(st)
    assert tk.topkv_kernel_launch_count() == before
    assert {INVALID, CAP, LAYOUT, CUDA} <= seen


def test_version_tells_the_decode_side_apart():
    """120 was the library without attention and page operators."""
    assert tk.topkv_version() >= 130

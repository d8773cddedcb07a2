"""GPU tests of new tokens on their way into the paged cache: rotation, conversion, places, against the
definition in 64 bits (tolerances derived in oracle.tokens.append); what is skipped stays as it was."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import decode as od, tokens as ot
from paper_2607_28633_b200 import binding as tk
from test_gpu_decode import NAN, TORCH, TYPE, _geom, _layout, _table

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
    yield
    assert tk.topkv_device_error_flags() == 0


def _values(rng, shape, io):
    return od.decode_elements(od.encode_elements(rng.normal(size=int(np.prod(shape))), io), io).reshape(shape)


def _case(dev, R=3, H=2, G=2, D=64, P=16, F=2, kind="bf16", io=None, style="page", new=None, sl=None, count=None, first=0, pairs=False,
          scale=1.0, far=None, base=10000.0, in_place=False, queries=True, spare=0, seed=0, L=1, layer=0, scales=None, error=0, bad_page=None,
          stream=None, graph=False, fused=True):
    rng = np.random.default_rng(seed)
    io = io or (kind if kind != "e4m3" else "bf16")
    one = new is None
    new = np.ones(R, np.int64) if one else np.asarray(new)
    sl = np.array([17, 64, 40][:R] if sl is None else sl)
    bt, pages = _table(np.maximum(sl, 0), P, 2, 1, rng)
    if bad_page is not None:
        bt[bad_page] = pages + 5
    g = _geom(F, H, D, 1 if kind == "e4m3" else 2, P, pages, style, L)
    cu = None if one else np.concatenate([[0], np.cumsum(new)])
    rows = int(new.sum()) + spare
    x = _values(rng, (max(rows, 1), H * G + F * H, D), io)[:rows]
    d_x = torch.from_numpy(x).to(dev).to(TORCH[io])
    if not fused:  # every tensor with padding of its own between rows
        d_x = torch.nn.functional.pad(d_x, (0, 8, 0, 1))[:, :-1, :D]
    Hq = H * G
    q, k, v = d_x[:, :Hq], d_x[:, Hq:Hq + H], d_x[:, Hq + H:] if F == 2 else None
    q_out = q if in_place else torch.full((rows, Hq, D), 7.0, dtype=d_x.dtype, device=dev)
    count = D if count is None else count
    freq = ot.frequencies(count, base)
    positions = None if far is None else rng.integers(0, far, size=rows)
    scales = scales or ((0.5, 3.0) if kind == "e4m3" else (1.0, 1.0))
    rotary = None
    if count:
        rotary = tk.make_rotary(torch.from_numpy(tk.topkv_rotary_turns(freq).view(np.int64)).to(dev),
                                tk.TOPKV_ROTARY_PAIRS if pairs else tk.TOPKV_ROTARY_HALVES, first, scale)
    pool_h = np.empty(g.L * g.S_layer, np.uint8)
    pool_h[0::2], pool_h[1::2] = NAN[kind]
    pool = torch.from_numpy(pool_h).to(dev)
    put = lambda a, t: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).to(dev).to(t)
    b = tk.make_batch(put(bt, torch.int32), put(sl, torch.int32))
    n = tk.make_new_tokens(k, v, TYPE[kind], TYPE[io], q=q if queries else None, q_out=q_out if queries else None, rotary=rotary,
                           cu_tokens=put(cu, torch.int64), positions=put(positions, torch.int32), k_scale=scales[0], v_scale=scales[1])
    call = lambda s: tk.check(tk.topkv_append_layer(layer, pool, _layout(g), b, n, k, v, q if queries else None, q_out if queries else None, s))
    torch.cuda.synchronize()
    if graph:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            call(torch.cuda.current_stream())
        assert np.array_equal(pool.cpu().numpy(), pool_h)
        gr.replay()
    else:
        call(stream)
    torch.cuda.synchronize()
    assert tk.topkv_device_error_flags() == error
    if error:
        tk.check(tk.topkv_reset_device_error_flags())
    found, err = ot.append(g, layer, bt, sl, cu, x[:, Hq:Hq + H], x[:, Hq + H:] if F == 2 else None, x[:, :Hq] if queries else None, positions,
                           freq, first, pairs, scale, *scales, kind, io)
    assert err == error
    got_pool, got_q = pool.cpu().numpy(), q_out.double().cpu().numpy()
    untouched, bytes_ = np.ones(len(pool_h), bool), D * g.b_p
    seen = np.zeros(rows, bool)
    for off, t, h, want, tol in found:
        if off is None:
            have = got_q[t, h]
            seen[t] = True
        else:
            assert untouched[off:off + bytes_].all()
            untouched[off:off + bytes_] = False
            have = od.decode_elements(got_pool[off:off + bytes_].copy(), kind)
        bad = ~(np.abs(have - want) <= tol)
        assert not bad.any(), (off, t, h, np.argwhere(bad)[:4], have[bad][:4], want[bad][:4], tol[bad][:4])
    assert np.array_equal(got_pool[untouched], pool_h[untouched])
    if queries:
        assert np.array_equal(got_q[~seen], x[~seen, :Hq] if in_place else np.full((int((~seen).sum()), Hq, D), 7.0))


@pytest.mark.parametrize("kw", [
    dict(),
    dict(io="fp16", kind="fp16", style="head", pairs=True),
    dict(kind="e4m3", io="fp16", style="padded"),
    dict(kind="e4m3", D=128, G=3, scale=1.25),
    dict(D=72, count=72, H=1),                              # halves of 36: no whole chunks
    dict(D=80, count=80, G=7),
    dict(D=80, count=40, first=40, pairs=True),
    dict(D=64, count=6, first=2), dict(D=64, count=6, first=58, pairs=True),
    dict(D=64, count=2), dict(D=24, H=5, count=16, first=8), dict(D=8, H=3, P=1, style="head"),
    dict(D=256, count=0), dict(D=128, count=64, first=64, style="plane"),
    dict(F=1, H=1, G=5, D=576, count=64, first=512, pairs=True, P=64),
    dict(F=1, H=1, G=1, D=576, count=64, first=512, kind="fp16"),
    dict(queries=False), dict(in_place=True), dict(in_place=True, D=72, H=2, count=18, first=3), dict(fused=False),
    dict(L=3, layer=2, style="padded"),
    dict(far=2 ** 31 - 1, base=500000.0), dict(far=10 ** 6, pairs=True),
    dict(D=2048, H=1, G=1, count=2048, P=4, sl=[3, 4, 5]),
])
def test_one_token_each(dev, kw):
    _case(dev, **kw)


@pytest.mark.parametrize("kw", [
    dict(new=[17, 1, 40], sl=[17, 64, 40]),
    dict(new=[5, 0, 33], spare=3), dict(new=[0, 0, 0], spare=2), dict(new=[0, 0, 0]),
    dict(new=[5, 9, 33], sl=[17, 0, 40], in_place=True),    # the middle one is left out
    dict(new=[300, 1, 700], sl=[400, 1, 700], P=24, kind="e4m3"),
    dict(new=[300, 20, 100], sl=[400, 20, 700], P=1, D=96, count=32, first=64),
    dict(R=1500, new=np.arange(1500) % 3, sl=2 + np.arange(1500) % 40, H=1, D=16, G=1),
    dict(R=1500, sl=np.arange(1500) % 40, H=1, D=16, G=1),
    dict(R=1, new=[2500], sl=[2500], H=1, G=1, D=64, far=10 ** 8),
])
def test_many_tokens(dev, kw):
    _case(dev, **kw)


@pytest.mark.parametrize("kw", [
    dict(new=[20, 1, 2], sl=[17, 64, 40]),                  # more tokens than the request has
    dict(new=[3, 1, 2], sl=[-4, 64, 40]),
    dict(sl=[17, 64, 40], bad_page=(1, 3)),
    dict(new=[4, 30, 4], sl=[17, 64, 40], bad_page=(1, 2)),
])
def test_unusable_tables_are_reported_and_skipped(dev, kw):
    _case(dev, error=2, **kw)


def test_another_stream_and_a_graph(dev):
    _case(dev, stream=torch.cuda.Stream(dev))
    _case(dev, graph=True)


def test_values_beyond_the_range_of_8_bits(dev):
    _case(dev, kind="e4m3", scales=(1e-3, -2e-3))


def test_nan_and_infinity_pass(dev):
    lo = tk.make_layout(1, 2, 1, 16, 1, 4, 2)
    k = torch.tensor([[[float("nan"), float("inf"), -float("inf"), 500.0] + [0.0] * 12]], device=dev, dtype=torch.bfloat16)
    pool = torch.zeros(2 * 4 * 2 * 16, dtype=torch.uint8, device=dev)
    bt, sl = torch.zeros((1, 1), dtype=torch.int32, device=dev), torch.ones(1, dtype=torch.int32, device=dev)
    n = tk.make_new_tokens(k, k, TYPE["e4m3"], TYPE["bf16"])
    tk.check(tk.topkv_append_layer(0, pool, lo, tk.make_batch(bt, sl), n, k, k, None, None))
    torch.cuda.synchronize()
    got = pool.view(torch.float8_e4m3fn).float()[:4]
    assert torch.isnan(got[0]) and got[1:].tolist() == [448.0, -448.0, 448.0]


def test_gradient_free_inverse(dev):
    """A rotation by minus the position, i.e. with frequencies negated, brings fp16 values back."""
    D, freq = 64, ot.frequencies(64, 10000.0)
    x = torch.randn(1, 1, D, device=dev, dtype=torch.float16)
    lo = tk.make_layout(1, 1, 1, D, 2, 8, 4)
    pool = torch.zeros(4 * 8 * D, dtype=torch.float16, device=dev)
    bt, sl = torch.tensor([[2]], dtype=torch.int32, device=dev), torch.tensor([6], dtype=torch.int32, device=dev)
    there, back = torch.empty_like(x), torch.empty_like(x)
    for src, dst, f in ((x, there, freq), (there, back, -freq)):
        turns = torch.from_numpy(tk.topkv_rotary_turns(f).view(np.int64)).to(dev)
        n = tk.make_new_tokens(src, None, TYPE["fp16"], TYPE["fp16"], q=src, q_out=dst, rotary=tk.make_rotary(turns))
        tk.check(tk.topkv_append_layer(0, pool, lo, tk.make_batch(bt, sl), n, src, None, src, dst))
    torch.cuda.synchronize()
    pair = (x[..., :D // 2].abs() + x[..., D // 2:].abs()).repeat(1, 1, 2).float()
    # two roundings to fp16, each half a step of at most the pair's size
    assert ((back - x).float().abs() <= pair * 2 * 2.0 ** -11 * 1.01).all()
    assert not torch.equal(there, x) and torch.equal(pool.view(4, 8, D)[2, 5], back[0, 0])


@pytest.mark.parametrize("kind, count", [("bf16", 64), ("e4m3", 64), ("bf16", 6)])
def test_offsets_beyond_32_bits(dev, kind, count):
    """Pages far apart get the bits that the same pages get side by side, and nothing around them."""
    rng = np.random.default_rng(3)
    sl, H, D, P = np.array([17, 64, 40]), 2, 64, 16
    bt, pages = _table(sl, P, 2, 1, rng)
    g = _geom(2, H, D, 1 if kind == "e4m3" else 2, P, pages)
    lo = _layout(g)
    k, v = (torch.from_numpy(_values(rng, (3, H, D), "bf16")).to(dev).to(torch.bfloat16) for _ in range(2))
    turns = torch.from_numpy(tk.topkv_rotary_turns(ot.frequencies(count, 10000.0)).view(np.int64)).to(dev)
    n = tk.make_new_tokens(k, v, TYPE[kind], TYPE["bf16"], rotary=tk.make_rotary(turns, tk.TOPKV_ROTARY_HALVES, 0, 1.0))
    b = tk.make_batch(torch.from_numpy(bt).to(dev), torch.from_numpy(sl.astype(np.int32)).to(dev))
    near = torch.zeros(pages * g.S_page, dtype=torch.uint8, device=dev)
    tk.check(tk.topkv_append_layer(0, near, lo, b, n, k, v, None, None))
    far = 700_000_000
    big = torch.zeros(pages * far, dtype=torch.uint8, device=dev)
    lo.pool_page_stride, lo.pool_layer_stride = far, pages * far
    tk.check(tk.topkv_append_layer(0, big, lo, b, n, k, v, None, None))
    torch.cuda.synchronize()
    assert torch.equal(big.view(pages, far)[:, :g.S_page], near.view(pages, g.S_page)) and near.any() and pages * far > 1 << 32
    for page in big.view(pages, far):
        assert not page[g.S_page:].any()


@pytest.mark.parametrize("io", ["bf16", "fp16"])
@pytest.mark.parametrize("count, pairs", [(0, False), (64, False), (64, True), (6, False)])
@pytest.mark.parametrize("scale", [7 / 1024, 0.3, 0.9, -1.1, 3.0, 0.5, 2.0 ** -126, 1e-38, 3e38])
def test_stored_elements_are_quotients(dev, io, count, pairs, scale):
    """Every value of 16 bits as an element of V, and of the part of K that does not turn: divided in 32 bits and
    rounded once, bit for bit (a quotient between two 8-bit values goes to the even one)."""
    D, rows = 256, 256
    bits = torch.arange(-32768, 32768, dtype=torch.int32).to(torch.int16).view(rows, 1, D)
    x = bits.view(TORCH[io]).to(dev)
    lo = tk.make_layout(1, 2, 1, D, 1, 1, rows)
    pool = torch.zeros(rows * 2 * D, dtype=torch.uint8, device=dev)
    bt, sl = torch.arange(rows, dtype=torch.int32, device=dev).view(rows, 1), torch.ones(rows, dtype=torch.int32, device=dev)
    rotary = None
    if count:
        turns = torch.from_numpy(tk.topkv_rotary_turns(ot.frequencies(count, 10000.0)).view(np.int64)).to(dev)
        rotary = tk.make_rotary(turns, tk.TOPKV_ROTARY_PAIRS if pairs else tk.TOPKV_ROTARY_HALVES, D - count)
    n = tk.make_new_tokens(x, x, TYPE["e4m3"], TYPE[io], rotary=rotary, k_scale=scale, v_scale=scale)
    tk.check(tk.topkv_append_layer(0, pool, lo, tk.make_batch(bt, sl), n, x, x, None, None))
    torch.cuda.synchronize()
    got = pool.cpu().numpy().reshape(rows, 2, D)
    with np.errstate(over="ignore"):
        quotient = x.float().cpu().numpy()[:, 0] / np.float32(scale)  # one operation in 32 bits
    nan = np.isnan(quotient)
    want = od.encode_elements(np.where(nan, 0, quotient).astype(np.float64).clip(-448, 448).reshape(-1), "e4m3").reshape(rows, D)
    for plane, columns in ((0, D - count), (1, D)):
        have, same = got[:, plane, :columns], np.where(nan, 0x7F, want)[:, :columns]
        bad = np.where(nan[:, :columns], have & 0x7F, have) != same
        assert not bad.any(), (plane, np.argwhere(bad)[:4], quotient[:, :columns][bad][:4], have[bad][:4], same[bad][:4])

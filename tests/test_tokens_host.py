"""CPU checks of the calls around the decode side's attention (rotated new tokens, shared prefixes, chosen
pages): refusals, workspace sizes, rotary tables, the class on top of them, and the oracle's own definitions
against hand-derived values. Nothing is launched: what is acceptable ends in TOPKV_ERR_CUDA without a GPU."""
import ctypes
from fractions import Fraction

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import __graft_entry__ as entry
from oracle import Geom, tokens as ot
from paper_2607_28633_b200 import binding as tk
from paper_2607_28633_b200 import session
from test_decode_host import ALIGN, CAP, CUDA, INVALID, LAYER, LAYOUT, _attention, _batch, _Fake, _gqa

BF16, FP16, E4M3 = tk.TOPKV_TYPE_BF16, tk.TOPKV_TYPE_FP16, tk.TOPKV_TYPE_E4M3


@pytest.fixture(scope="module", autouse=True)
def _built():
    entry.build()
    if torch.cuda.is_available():
        pytest.skip("fake addresses must never reach a real device")


def test_struct_sizes():
    assert ctypes.sizeof(tk.topkv_rotary) == 32 and ctypes.sizeof(tk.topkv_new_tokens) == 120
    assert ctypes.sizeof(tk.topkv_rotary_stretch) == 48 and ctypes.sizeof(tk.topkv_page_choice) == 40


# ---- rotary tables ----------------------------------------------------------------------------------

def _frequencies(count, stretch):
    f = np.full(count // 2, 7.0)
    return tk.lib().topkv_rotary_frequencies(ctypes.byref(stretch), count, f.ctypes.data), f


def _stretch(kind=0, base=10000.0, factor=1.0, original=0.0, slow=0.0, fast=0.0):
    s = tk.topkv_rotary_stretch()
    s.struct_size, s.kind, s.base, s.factor, s.original_tokens, s.slow, s.fast = ctypes.sizeof(s), kind, base, factor, original, slow, fast
    return s


@pytest.mark.parametrize("kind, kw", [("none", {}), ("linear", dict(factor=4.0)), ("base", dict(factor=8.0)),
                                      ("ramp", dict(factor=32.0, original=4096.0, slow=1.0, fast=32.0)),
                                      ("ramp", dict(factor=8.0, original=8192.0, slow=1.0, fast=4.0))])
def test_frequencies(kind, kw):
    for count in (0, 4, 64, 128):
        st, f = _frequencies(count, _stretch(["none", "linear", "base", "ramp"].index(kind), 500000.0, **kw))
        assert st == tk.TOPKV_OK
        assert np.allclose(f, ot.frequencies(count, 500000.0, kind, **kw), rtol=1e-14)


def test_frequencies_by_hand():
    f = tk.topkv_rotary_frequencies(4, 100.0)
    assert f.tolist() == [1.0, 0.1]
    # the fastest pair stays, the slowest is divided by the factor
    g = tk.topkv_rotary_frequencies(64, 10000.0, tk.TOPKV_STRETCH_BASE, 16.0)
    plain = tk.topkv_rotary_frequencies(64, 10000.0)
    assert g[0] == 1.0 and abs(plain[-1] / g[-1] - 16.0) < 1e-9
    # 1000 tokens: the first pair turns 159 times (stays), the last 0.0016 times (divided)
    r = tk.topkv_rotary_frequencies(4, 1e10, tk.TOPKV_STRETCH_RAMP, 4.0, 1000.0, 1.0, 32.0)
    assert r[0] == 1.0 and r[1] == 1e-5 / 4


def test_frequency_refusals():
    nan, inf = float("nan"), float("inf")
    for count, s in [(3, _stretch()), (4, _stretch(kind=4)), (4, _stretch(base=0.0)), (4, _stretch(base=nan)), (4, _stretch(base=inf)),
                     (4, _stretch(1, factor=0.5)), (4, _stretch(1, factor=nan)), (2, _stretch(2, factor=2.0)), (4, _stretch(3, factor=2.0)),
                     (4, _stretch(3, factor=2.0, original=100.0, slow=4.0, fast=4.0)), (4, _stretch(3, factor=2.0, original=100.0, slow=-1.0, fast=4.0)),
                     (4, _stretch(3, factor=2.0, original=100.0, slow=1.0, fast=inf))]:
        assert _frequencies(count, s)[0] == INVALID
    s = _stretch()
    s.struct_size = 8
    assert _frequencies(4, s)[0] == INVALID
    f = np.array([1.0, nan])
    t = np.zeros(2, np.uint64)
    assert tk.lib().topkv_rotary_turns(f.ctypes.data, 2, t.ctypes.data) == INVALID
    assert tk.lib().topkv_rotary_turns(None, 1, t.ctypes.data) == INVALID and tk.lib().topkv_rotary_turns(None, 0, None) == tk.TOPKV_OK


def test_turns_are_exact_at_any_position():
    """position * turns modulo 2^64 against exact fractions of a turn: off by half a unit of the table a
    position, and by the 64 bits of two pi's mantissa (2^-63 of the turns made)."""
    two_pi = Fraction(6283185307179586476925286766559005768394, 10 ** 39)
    f = np.concatenate([ot.frequencies(128, 10000.0), -ot.frequencies(8, 5e5), [0.0, 6.25, 1e3]])
    turns = tk.topkv_rotary_turns(f)
    for j in range(len(f)):
        for pos in (0, 1, 4097, 10 ** 8 + 7, 2 ** 31 - 1):
            have = Fraction(int(turns[j]) * pos % 2 ** 64, 2 ** 64)
            want = Fraction(float(f[j])) * pos / two_pi
            off = (have - want) % 1
            assert min(off, 1 - off) <= Fraction(pos, 2 ** 65) + abs(want) / 2 ** 62, (j, pos)


# ---- refusals -----------------------------------------------------------------------------------------

def _rotary(**kw):
    t = tk.topkv_rotary()
    t.struct_size, t.style, t.first, t.count, t.scale, t.turns = ctypes.sizeof(t), tk.TOPKV_ROTARY_HALVES, 0, 128, 1.0, 0xE000000
    for k, v in kw.items():
        setattr(t, k, v)
    return t


def _tokens(H=8, D=128, Hq=64, rotary=None, **kw):
    n = tk.topkv_new_tokens()
    n.struct_size, n.cache_type, n.io_type, n.num_q_heads, n.num_rows, n.k_scale, n.v_scale = ctypes.sizeof(n), BF16, BF16, Hq, 4, 1.0, 1.0
    row = (Hq + 2 * H) * D * 2
    n.k_row_stride = n.v_row_stride = n.q_row_stride = row
    n.k_head_stride = n.v_head_stride = n.q_head_stride = n.q_out_head_stride = 2 * D
    n.q_out_row_stride = Hq * D * 2
    n.rotary = ctypes.pointer(_rotary() if rotary is None else rotary)
    for k, v in kw.items():
        setattr(n, k, v)
    return n


def _append(lo, b, n, layer=0, pool=0x7000000, k=0x8000000, v=0x9000000, q=0xA000000, q_out=0xB000000):
    return tk.topkv_append_layer(layer, pool, lo, b, n, k, v, q, q_out)


def test_append_accepts_what_the_header_allows():
    for lo, n, kw in [
        (_gqa(), _tokens(), {}), (_gqa(), _tokens(rotary=None, num_q_heads=0, q_out_row_stride=0), dict(q=None, q_out=None)),
        (_gqa(), _tokens(cu_tokens=0xC000000, num_rows=10 ** 6, positions=0xD000004), {}), (_gqa(E=1), _tokens(cache_type=E4M3, k_scale=-2.0, v_scale=0.5), {}),
        (_gqa(D=72, H=2), _tokens(H=2, D=72, Hq=6, rotary=_rotary(count=6, first=66)), {}), (_gqa(), _tokens(rotary=_rotary(count=0, turns=None)), {}),
        (_gqa(), _tokens(q_out_row_stride=256, q_out_head_stride=4 * 256), {}),                            # [heads][rows]
        (_gqa(), _tokens(q_out_row_stride=(64 + 16) * 256), dict(q_out=0xA000000)),                        # in place
        (tk.make_layout(2, 1, 1, 576, 2, 64, 100), _tokens(1, 576, 128, _rotary(first=512, count=64, style=tk.TOPKV_ROTARY_PAIRS)), dict(v=None)),
    ]:
        assert _append(lo, _batch(), n, **kw) == CUDA
    empty = _tokens()
    empty.rotary = None
    assert _append(_gqa(), _batch(), empty) == CUDA
    assert _append(_gqa(), _batch(R=0), _tokens()) == tk.TOPKV_OK
    assert _append(_gqa(), _batch(), _tokens(num_rows=0, cu_tokens=0xC000000), k=None, v=None, q=None, q_out=None) == tk.TOPKV_OK


def test_append_refusals():
    lo, b = _gqa(), _batch()
    nan, inf = float("nan"), float("inf")
    for status, change in [
        (INVALID, dict(struct_size=8)), (INVALID, dict(cache_type=0)), (INVALID, dict(cache_type=4)), (INVALID, dict(io_type=3)), (INVALID, dict(io_type=FP16)),
        (INVALID, dict(k_scale=2.0)), (INVALID, dict(v_scale=0.0)), (INVALID, dict(k_scale=nan)), (INVALID, dict(num_rows=-1)), (INVALID, dict(num_rows=3)),
        (INVALID, dict(num_rows=1 << 31, cu_tokens=0xC000000)), (INVALID, dict(num_q_heads=65536)), (INVALID, dict(k_row_stride=-16)), (ALIGN, dict(v_head_stride=264)),
        (INVALID, dict(q_row_stride=1 << 41)), (ALIGN, dict(q_out_row_stride=64 * 256 + 8)), (INVALID, dict(q_out_row_stride=63 * 256)), (INVALID, dict(q_out_head_stride=128)),
        (INVALID, dict(q_out_head_stride=0)), (ALIGN, dict(cu_tokens=0xC000004)), (ALIGN, dict(positions=0xD000002)), (LAYOUT, dict(cache_type=E4M3)),
    ]:
        assert _append(lo, b, _tokens(**change)) == status, change
    for status, change in [
        (INVALID, dict(struct_size=8)), (INVALID, dict(reserved=1)), (INVALID, dict(style=0)), (INVALID, dict(style=3)), (INVALID, dict(count=127)), (INVALID, dict(count=130)),
        (INVALID, dict(first=2)), (INVALID, dict(first=0xFFFFFFF0, count=64)), (INVALID, dict(scale=nan)), (INVALID, dict(scale=inf)), (INVALID, dict(turns=None)),
        (ALIGN, dict(turns=0xE000004)),
    ]:
        assert _append(lo, b, _tokens(rotary=_rotary(**change))) == status, change
    n = _tokens()
    assert _append(lo, b, n, layer=2) == LAYER and _append(lo, b, n, layer=-1) == LAYER
    for name in ("pool", "k", "v", "q", "q_out"):
        assert _append(lo, b, n, **{name: None}) == INVALID
        assert _append(lo, b, n, **{name: 0x7000008}) == ALIGN
    assert _append(lo, b, n, q_out=0xA000000) == INVALID                                 # in place with other strides
    assert _append(lo, _batch(window_tokens=4), n) == INVALID and _append(lo, _batch(maxp=-1), n) == INVALID
    for scale in (1e-45, 0.0, inf):
        assert _append(_gqa(E=1), b, _tokens(cache_type=E4M3, k_scale=scale)) == INVALID
    assert _append(_gqa(E=1), b, _tokens()) == LAYOUT and _append(_gqa(D=2056, H=1), b, _tokens(1, 2056, 1)) == LAYOUT
    assert _append(_gqa(D=20, H=2), b, _tokens(2, 20, 2)) == LAYOUT


def _shared(lo, b, a, layer=0, pool=0x7000000, plan=0xC000000, q=0x8000000, out=0x9000000, ws=0xA000000, n=1 << 50):
    return tk.topkv_attend_shared_layer(layer, pool, lo, b, a, plan, q, out, ws, n)


def test_shared_refusals():
    lo, b, a = _gqa(), _batch(), _attention()
    assert _shared(lo, b, a) == CUDA and _shared(_gqa(E=1), b, _attention(cache=E4M3, k_scale=0.5)) == CUDA
    assert _shared(_gqa(D=256, H=1), b, _attention(Hq=16, D=256)) == CUDA and _shared(lo, _batch(flags=3), a) == CUDA
    assert _shared(lo, _batch(R=0), a) == tk.TOPKV_OK
    assert _shared(lo, _batch(window_tokens=9), a) == INVALID and _shared(lo, b, _attention(sink_tokens=4)) == INVALID
    assert _shared(tk.make_layout(1, 1, 1, 576, 2, 64, 9), b, _attention(Hq=16, D=576, Dv=512)) == LAYOUT
    assert _shared(lo, b, _attention(num_q_heads=63)) == INVALID and _shared(lo, b, a, layer=2) == LAYER
    for name in ("pool", "q", "out", "ws"):
        assert _shared(lo, b, a, **{name: None}) == INVALID and _shared(lo, b, a, **{name: 0x7000008}) == ALIGN
    assert _shared(lo, b, a, plan=None) == INVALID and _shared(lo, b, a, plan=0xC000002) == ALIGN
    need = tk.topkv_attend_shared_workspace_bytes(lo, b, a)
    assert need > 0 and _shared(lo, b, a, n=need - 1) == CAP and _shared(lo, b, a, n=need) == CUDA
    assert tk.topkv_attend_shared_workspace_bytes(lo, _batch(R=0), a) == 0
    # more work than its line counts: 60,000 requests of two million tokens
    assert _shared(_gqa(P=64), _batch(R=60000, maxp=32768), _attention(R=60000)) == LAYOUT
    plan = lambda lo=lo, b=b, least=0, p=0xC000000: tk.topkv_plan_prefixes(lo, b, least, p)
    assert plan() == CUDA and plan(b=_batch(R=5000)) == CUDA and plan(b=_batch(R=0), p=None) == tk.TOPKV_OK
    assert plan(least=-1) == INVALID and plan(p=None) == INVALID and plan(p=0xC000002) == ALIGN and plan(b=_batch(window_tokens=3)) == INVALID
    before = tk.topkv_set_sharing_bytes(7)
    assert before == tk.TOPKV_DEFAULT_SHARING_BYTES and tk.topkv_set_sharing_bytes(-1) == INVALID and tk.topkv_set_sharing_bytes(before) == 7


def _choice(budget=8, first=1, last=1, **kw):
    c = tk.topkv_page_choice()
    c.struct_size, c.budget, c.first_pages, c.last_pages = ctypes.sizeof(c), budget, first, last
    c.bounds, c.steps, c.chosen = 0xB000000, 0xC000000, 0xD000000
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _choose(lo, b, a, c, q=0x8000000, ws=0xA000000, n=1 << 50):
    return tk.topkv_choose_pages_layer(lo, b, a, c, q, ws, n)


def _sparse(lo, b, a, c, layer=0, pool=0x7000000, q=0x8000000, out=0x9000000, ws=0xA000000, n=1 << 50):
    return tk.topkv_attend_pages_layer(layer, pool, lo, b, a, c, q, out, ws, n)


def test_chosen_pages_refusals():
    lo, b, a, c = _gqa(), _batch(), _attention(), _choice()
    for call in (_choose, _sparse):
        assert call(lo, b, a, c) == CUDA and call(lo, b, a, _choice(1, 0, 1)) == CUDA and call(lo, b, a, _choice(1, 100, 100)) == CUDA
        assert call(lo, _batch(R=0), a, c) == tk.TOPKV_OK and call(_gqa(E=1), b, _attention(cache=E4M3, k_scale=0.5), c) == CUDA
        for status, change in [(INVALID, dict(struct_size=8)), (INVALID, dict(budget=0)), (INVALID, dict(budget=1 << 31)), (INVALID, dict(last_pages=0)),
                               (INVALID, dict(last_pages=1 << 31)), (INVALID, dict(first_pages=1 << 31)), (INVALID, dict(chosen=None)), (ALIGN, dict(bounds=0xB000008)),
                               (ALIGN, dict(steps=0xC000002)), (ALIGN, dict(chosen=0xD000001))]:
            assert call(lo, b, a, _choice(**change)) == status, change
        assert call(lo, _batch(window_tokens=9), a, c) == INVALID and call(lo, b, _attention(sink_tokens=4), c) == INVALID
        assert call(_gqa(E=1), b, _attention(cache=E4M3, k_scale=-0.5), c) == INVALID and call(lo, b, _attention(num_q_heads=63), c) == INVALID
        assert call(tk.make_layout(1, 1, 1, 576, 2, 64, 9), b, _attention(Hq=16, D=576, Dv=512), c) == LAYOUT
        assert call(_gqa(H=1), b, _attention(Hq=129), c) == LAYOUT and call(_gqa(H=1), b, _attention(Hq=128), c) == CUDA
        assert call(lo, b, a, c, q=None) == INVALID and call(lo, b, a, c, q=0x8000008) == ALIGN
    for name in ("bounds", "steps"):  # which only the choice reads
        assert _choose(lo, b, a, _choice(**{name: None})) == INVALID and _sparse(lo, b, a, _choice(**{name: None})) == CUDA
    assert _sparse(lo, b, a, c, layer=2) == LAYER
    for name in ("pool", "out"):
        assert _sparse(lo, b, a, c, **{name: None}) == INVALID and _sparse(lo, b, a, c, **{name: 0x7000008}) == ALIGN
    # long lists need a workspace for the attention, very long tables one for the choice
    size = lambda b, c: tk.topkv_page_choice_workspace_bytes(lo, b, a, c)
    assert size(b, _choice(4)) == 0 and _sparse(lo, b, a, _choice(4), ws=None, n=0) == CUDA and _choose(lo, b, a, c, ws=None, n=0) == CUDA
    long = size(b, _choice(64))
    assert long > 0 and _sparse(lo, b, a, _choice(64), n=long - 1) == CAP and _sparse(lo, b, a, _choice(64), n=long) == CUDA
    wide, few = _batch(R=1, maxp=1 << 22), _choice(4)
    need = size(wide, few)
    assert need >= 8 * (4 << 22) and _choose(lo, wide, a, few, n=need // 2) == CAP and _choose(lo, wide, a, few, n=need) == CUDA
    assert _choose(lo, wide, a, few, ws=None) == INVALID and _choose(lo, wide, a, few, ws=0xA000008) == ALIGN


def test_a_choice_refuses_negative_scales():
    """They turn the order of the scores round; a caller's own list has no order."""
    lo, b, c = _gqa(), _batch(), _choice()
    for scale, status in [(-0.1, INVALID), (-1e-45, INVALID), (0.0, CUDA), (-0.0, CUDA), (0.1, CUDA)]:
        assert _choose(lo, b, _attention(scale=scale), c) == status and _sparse(lo, b, _attention(scale=scale), c) == CUDA
    assert tk.topkv_page_choice_workspace_bytes(lo, b, _attention(scale=-0.1), c) >= 0


def test_bounds_refusals():
    lo, b = _gqa(), _batch()
    call = lambda lo=lo, b=b, kind=BF16, layer=0, pool=0x7000000, bounds=0xB000000, steps=0xC000000: tk.topkv_bound_pages_layer(layer, pool, lo, b, kind, bounds, steps)
    assert call() == CUDA and call(b=_batch(window_tokens=7)) == CUDA and call(kind=FP16) == CUDA and call(lo=_gqa(E=1), kind=E4M3) == CUDA
    assert call(b=_batch(R=0)) == tk.TOPKV_OK and call(b=_batch(maxp=0)) == tk.TOPKV_OK
    assert call(kind=0) == INVALID and call(kind=4) == INVALID and call(kind=E4M3) == LAYOUT and call(lo=_gqa(E=1)) == LAYOUT
    assert call(layer=2) == LAYER and call(lo=_gqa(D=264)) == LAYOUT and call(lo=tk.make_layout(1, 1, 1, 576, 2, 64, 9)) == LAYOUT
    assert call(lo=_gqa(H=2, D=24, E=1), kind=E4M3) == LAYOUT
    for name in ("pool", "bounds", "steps"):
        assert call(**{name: None}) == INVALID and call(**{name: 0x7000002}) == ALIGN


def test_random_descriptors_come_back_with_a_status():
    known = {tk.TOPKV_OK, INVALID, LAYER, ALIGN, CAP, LAYOUT, CUDA}
    before = tk.topkv_kernel_launch_count()
    seen = set()
    for seed in range(400):
        rng = np.random.default_rng(seed)
        pick = lambda *xs: xs[int(rng.integers(0, len(xs)))]
        H, D, E = pick((8, 128, 2), (1, 64, 1), (5, 80, 2), (2, 256, 2), (3, 72, 1))
        lo = tk.make_layout(2, pick(2, 2, 2, 1), H, D, E, pick(1, 16, 24, 64), pick(1, 4096))
        b = _batch(R=pick(0, 1, 4, 3000), maxp=pick(0, 1, 64, 70000), window_tokens=pick(0, 0, 0, 5), flags=pick(0, 1, 2, 3, 4))
        kind = pick(0, 1, 1, 1, 2, 3, 4)
        a = _attention(Hq=H * pick(1, 4, 129), D=D, cache=kind, io=pick(0, 1, 1, 2, 3), R=max(b.num_requests, 1), k_scale=pick(1.0, -2.0, float("inf")))
        n = _tokens(H, D, H * 2, _rotary(count=pick(0, 3, 64, D), first=pick(0, 8, D)), cache_type=kind, io_type=pick(1, 2), num_rows=pick(-1, 0, 4, 10 ** 6),
                    cu_tokens=pick(None, 0xC000000), k_scale=pick(1.0, 0.0, 2.0))
        c = _choice(pick(0, 1, 8, 10 ** 9), pick(0, 3, 2 ** 31), pick(0, 1, 9), chosen=pick(0xD000000, None))
        for lie in range(int(rng.integers(0, 3))):
            what = pick(lo, b, a, n, c)
            name, ctype = what._fields_[int(rng.integers(0, len(what._fields_)))][:2]
            if ctype in (ctypes.c_uint32, ctypes.c_int32, ctypes.c_int64):
                setattr(what, name, pick(0, 1, 7, 2 ** 31 - 1) if name != "struct_size" else 12)
        layer = pick(-1, 0, 1, 2)
        size = pick(0, 1 << 20, 1 << 50)
        got = [_append(lo, b, n, layer), _shared(lo, b, a, layer, n=size), tk.topkv_plan_prefixes(lo, b, pick(-1, 0, 5), 0xC000000), _choose(lo, b, a, c, n=size),
               _sparse(lo, b, a, c, layer, n=size), tk.topkv_bound_pages_layer(layer, 0x7000000, lo, b, kind, 0xB000000, 0xC000000)]
        sizes = [tk.topkv_attend_shared_workspace_bytes(lo, b, a), tk.topkv_page_choice_workspace_bytes(lo, b, a, c)]
        assert all(x in known for x in got) and all(x >= 0 or x in known for x in sizes)
        seen.update(got)
    assert tk.topkv_kernel_launch_count() == before and {tk.TOPKV_OK, INVALID, LAYER, LAYOUT, CUDA} <= seen


# ---- binding and class --------------------------------------------------------------------------------

def test_binding_refuses_tensors_that_do_not_fit():
    t = lambda *shape, dtype=torch.bfloat16: torch.zeros(shape, dtype=dtype)
    k = t(4, 2, 16)
    for bad in [dict(v=t(4, 3, 16)), dict(v=t(4, 2, 16, dtype=torch.float16)), dict(q=t(4, 4, 16)), dict(q=t(3, 4, 16), q_out=t(3, 4, 16)), dict(q=t(4, 4, 16), q_out=t(4, 5, 16)),
                dict(cu_tokens=torch.zeros(5, dtype=torch.int32)), dict(positions=torch.zeros(3, dtype=torch.int32)), dict(positions=torch.zeros(4))]:
        with pytest.raises(ValueError):
            tk.make_new_tokens(k, bad.pop("v", k), BF16, BF16, **bad)
    with pytest.raises(ValueError):
        tk.make_new_tokens(k.transpose(1, 2), None, BF16, BF16)
    with pytest.raises(ValueError):
        tk.make_rotary(torch.zeros(4, dtype=torch.int32))
    b8, st, ch = torch.zeros((9, 2, 2, 16), dtype=torch.int8), torch.zeros((9, 2)), torch.zeros((3, 2, 5), dtype=torch.int32)
    assert tk.make_page_choice(5, 1, 1, b8, st, ch).budget == 5
    for args in [(4, b8, st, ch), (5, b8[:, :1], st, ch), (5, b8, st[:8], ch), (5, b8, st, ch.transpose(0, 1))]:
        with pytest.raises(ValueError):
            tk.make_page_choice(args[0], 1, 1, *args[1:])
    one = tk.make_new_tokens(t(1, 1, 16), None, BF16, BF16)
    assert one.k_row_stride == 0 and one.k_head_stride == 0 and one.num_q_heads == 0


def test_binding_refuses_turns_of_another_device():
    """A table left on the host would be an address that the kernel cannot read."""
    k, turns = torch.zeros((4, 2, 16), dtype=torch.bfloat16), torch.zeros(8, dtype=torch.int64)
    assert tk.make_new_tokens(k, k, BF16, BF16, rotary=tk.make_rotary(turns)).rotary.contents.count == 16
    with pytest.raises(ValueError):
        tk.make_new_tokens(k, k, BF16, BF16, rotary=tk.make_rotary(turns.to("meta")))
    with pytest.raises(ValueError):
        tk.make_new_tokens(k.to("meta"), None, BF16, BF16, rotary=tk.make_rotary(turns))
    bare = tk.topkv_rotary()  # a descriptor of the caller's own says nothing of devices
    assert tk.make_new_tokens(k, k, BF16, BF16, rotary=bare).rotary


@pytest.fixture
def cache(monkeypatch):
    """A cache whose library calls are noted, not made."""
    import contextlib

    class Idle:
        def synchronize(self):
            pass
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: Idle())
    monkeypatch.setattr(session.DecodeCache, "_on", lambda self, stream: contextlib.nullcontext())
    calls = []
    for name in ("append_layer", "plan_prefixes", "attend_shared_layer", "bound_pages_layer", "choose_pages_layer", "attend_pages_layer", "fork_requests", "free_requests",
                 "compact_pages", "extend_requests"):
        monkeypatch.setattr(tk, f"topkv_{name}", lambda *a, name=name, **kw: calls.append((name, a)) or 0)
    lo = tk.make_layout(2, 2, 2, 16, 2, 4, 8)
    bt = torch.tensor([[0, 1, -1], [2, 3, -1], [-1, -1, -1]], dtype=torch.int32)
    c = session.DecodeCache(torch.zeros(2 * 8 * 2 * 4 * 2 * 16, dtype=torch.bfloat16), lo, bt, torch.tensor([5, 8, 0], dtype=torch.int32))
    return c, calls


def test_class_asks_for_a_plan_after_forks_and_frees(cache):
    c, calls = cache
    q, ints = torch.zeros((3, 4, 16), dtype=torch.bfloat16), lambda *x: torch.tensor(x, dtype=torch.int32)
    for change in (None, lambda: c.fork(ints(0), ints(2), None), lambda: c.free(ints(0), None)):
        if change:
            change()
        with pytest.raises(ValueError):
            c.attend_shared(0, q, q.clone(), 1.0, None)
        c.plan_prefixes(None)
        c.attend_shared(0, q, q.clone(), 1.0, None)
        c.extend(ints(1, 1, 0), None)
        c.compact(None)
        c.attend_shared(1, q, q.clone(), 1.0, None)
    assert [n for n, _ in calls].count("attend_shared_layer") == 6


def test_class_bounds_all_pages_where_it_must(cache):
    c, calls = cache
    q, chosen, ints = torch.zeros((3, 4, 16), dtype=torch.bfloat16), torch.zeros((3, 2, 2), dtype=torch.int32), lambda *x: torch.tensor(x, dtype=torch.int32)
    with pytest.raises(ValueError):
        c.attend_chosen(0, q, q.clone(), chosen, 1.0, None)
    windows = lambda: [a[3].window_tokens for n, a in calls if n == "bound_pages_layer"]
    c.bound_pages(0, None, tokens=1)
    c.bound_pages(0, None, tokens=1)
    c.bound_pages(1, None)
    assert windows() == [0, 1, 0]
    c.attend_chosen(0, q, q.clone(), chosen, 1.0, None)
    c.free(ints(0), None)
    c.attend_chosen(1, q, q.clone(), chosen, 1.0, None)
    for change in (lambda: c.fork(ints(0), ints(2), None), lambda: c.compact(None)):
        change()
        with pytest.raises(ValueError):
            c.attend_chosen(1, q, q.clone(), chosen, 1.0, None)
        c.bound_pages(1, None, tokens=3)
        c.bound_pages(1, None, tokens=3)
    assert windows() == [0, 1, 0, 0, 3, 0, 3]
    for bad in (chosen[:2], chosen[:, :1], chosen.long()):
        with pytest.raises(ValueError):
            c.attend_chosen(1, q, q.clone(), bad, 1.0, None)
    for bad in (dict(layer=2), dict(layer=0, tokens=-1)):
        with pytest.raises(ValueError):
            c.bound_pages(stream=None, **bad)


def test_class_keeps_to_one_type_of_elements(cache):
    """Bounds of one type are not used with another; a type that is not given is what the tensors' are."""
    c, calls = cache
    q, chosen = torch.zeros((3, 4, 16), dtype=torch.float16), torch.zeros((3, 2, 2), dtype=torch.int32)
    bounds = lambda: [(a[3].window_tokens, a[4]) for n, a in calls if n == "bound_pages_layer"]
    c.bound_pages(0, None)
    with pytest.raises(ValueError):
        c.attend_chosen(0, q, q.clone(), chosen, 1.0, None)                # fp16 queries of a bfloat16 pool
    c.bound_pages(0, None, tokens=1, cache_type=FP16)                      # the pages' bounds were those of the other type
    c.attend_chosen(0, q, q.clone(), chosen, 1.0, None)
    c.bound_pages(0, None, tokens=1, cache_type=FP16)
    with pytest.raises(ValueError):
        c.attend_chosen(0, q.bfloat16(), q.bfloat16(), chosen, 1.0, None)
    c.pool = c.pool.half()
    c.bound_pages(1, None)
    c.pool = c.pool.view(torch.uint8)
    c.bound_pages(1, None, tokens=1)
    assert bounds() == [(0, BF16), (0, FP16), (1, FP16), (0, FP16), (0, BF16)]


def test_class_knows_8_bit_pools(monkeypatch, cache):
    c, calls = cache
    monkeypatch.setattr(c, "layout", tk.make_layout(2, 2, 2, 16, 1, 4, 8))
    k, q, chosen = torch.zeros((3, 2, 16), dtype=torch.float16), torch.zeros((3, 4, 16), dtype=torch.float16), torch.zeros((3, 2, 2), dtype=torch.int32)
    c.append_rotated(0, k, k, None, k_scale=0.5)
    assert calls[-1][1][4].cache_type == E4M3 and calls[-1][1][4].io_type == FP16
    c.bound_pages(0, None)
    c.plan_prefixes(None)
    monkeypatch.setattr(tk, "topkv_attend_layer", lambda *a: calls.append(("attend_layer", a)) or 0)
    for call in (c.attend, c.attend_shared):
        call(0, q, q.clone(), 1.0, None, k_scale=0.5)
        assert calls[-1][1][4].cache_type == E4M3 and calls[-1][1][4].io_type == FP16
    c.attend_chosen(0, q, q.clone(), chosen, 1.0, None, k_scale=0.5)
    assert calls[-1][0] == "attend_pages_layer" and calls[-1][1][4].cache_type == E4M3


def test_class_appends_what_has_grown(cache):
    c, calls = cache
    ints = lambda *x: torch.tensor(x, dtype=torch.int32)
    k = torch.zeros((3, 2, 16), dtype=torch.bfloat16)
    c.append_rotated(0, k, k, None)
    assert calls[-1][1][3].seq_lens == c.seq_lens.data_ptr()              # nothing is known to be new: all rows
    c.extend(ints(1, 0, 0), None)                                         # noted, not done: lengths stay, so no wish is met
    c.append_rotated(0, k, k, None)
    assert calls[-1][1][3].seq_lens == c._new.lens.data_ptr() and c._new.lens.tolist() == [0, 0, 0]
    c.append_rotated(1, k, k, None)
    assert not c._new.pending
    for bad in [dict(k=k[:2], v=k[:2]), dict(k=k, v=None), dict(k=k[:, :1], v=k[:, :1]), dict(k=k.float(), v=k.float()), dict(k=k, v=k, cu_tokens=torch.zeros(3, dtype=torch.int64))]:
        with pytest.raises(ValueError):
            c.append_rotated(0, stream=None, **bad)


# ---- the oracle by hand ---------------------------------------------------------------------------------

def test_oracle_rotation_by_hand():
    x = np.array([3.0, 1.0, 4.0, 1.0, 5.0])
    y, size = ot.rotate(x, 1, np.array([np.pi / 2]), 1, True, 2.0)       # a quarter turn of (1, 4)
    assert np.allclose(y, [3, -8, 2, 1, 5]) and size.tolist() == [0, 10, 10, 0, 0]
    y, _ = ot.rotate(x, 2, np.array([np.pi / 2, 0.0]), 0, False, 1.0)    # half a turn of (3, 4); (1, 1) stays
    assert np.allclose(y, [-3, 1, -4, 1, 5])


def test_oracle_plan_by_hand():
    bt = np.array([[5, 6, 7], [5, 6, 9], [5, 8, -1], [5, 6, -1], [3, 6, 7], [5, 6, 7]])
    plan = ot.plan_prefixes(4, 10, bt, np.array([12, 9, 6, 3, 12, 0]))
    assert plan.tolist() == [[0, 0, 0, 3, 4, 5], [12, 8, 4, 0, 12, 0], [4, 4, 4, 0, 0, 0], [3, 3, 3, 1, 1, 1], [0, 1, 2, 3, 4, 5], [0, 1, 2, 3, 4, 5]]
    assert ot.plan_prefixes(4, 10, bt, np.array([12, 9, 6, 3, 12, 0]), 5)[2].tolist() == [0] * 6


def test_oracle_choice_by_hand():
    bounds = np.zeros((4, 1, 2, 8), np.int8)
    bounds[:, 0, 0, 0], bounds[:, 0, 1, 0] = [-10, -3, -8, -2], [1, 2, 9, 4]
    steps = np.ones((4, 1), np.float32)
    q = np.zeros((1, 1, 8))
    choose = lambda x, budget, firsts=0: ot.choose_pages(2, np.array([[0, 1, 2, 3]]), np.array([8]), np.where(np.arange(8) == 0, x, q), 1, bounds, steps, budget, firsts, 1)[0, 0].tolist()
    assert choose(1.0, 2) == [2, 3] and choose(-1.0, 2) == [0, 3] and choose(1.0, 3) == [1, 2, 3] and choose(-1.0, 3, 2) == [0, 1, 3]
    assert choose(0.0, 2) == [0, 3] and choose(1.0, 6) == [0, 1, 2, 3, -1, -1]
    assert ot.of_chosen(2, np.array([7, 8, 9]), 5, [0, 2, -1])[1] == 3

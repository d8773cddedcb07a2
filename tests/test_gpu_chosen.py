"""GPU tests of sparse attention over chosen pages: bounds and choices against the definition, number for
number; the attention against the oracle in 64 bits over the chosen tokens."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import decode as od, tokens as ot
from paper_2607_28633_b200 import binding as tk
from test_gpu_decode import NAN, TORCH, TYPE, _check, _geom, _layout, _table

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


def _fill(g, bt, sl, kind, rng, layer=0, size=1.0):
    pool = np.empty(g.L * g.S_layer, np.uint8)
    pool[0::2], pool[1::2] = NAN[kind]
    n = g.d_h * g.b_p
    for r, s in enumerate(sl):
        x = od.encode_elements(size * rng.normal(size=max(int(s), 0) * 2 * g.h_kv * g.d_h), kind).reshape(-1, n)
        k = 0
        for i in range(int(s)):
            for c in range(2):
                for h in range(g.h_kv):
                    a = od.row_offset(g, layer, int(bt[r, i // g.P]), c, i % g.P, h)
                    pool[a:a + n] = x[k]
                    k += 1
    return pool


class Case:
    def __init__(self, dev, sl, H=2, G=2, D=64, P=16, kind="bf16", io=None, style="page", L=1, layer=0, seed=0, budget=3, firsts=1, lasts=1, ks=1.0,
                 vs=1.0, extra_cols=1, size=1.0):
        rng = np.random.default_rng(seed)
        self.dev, self.kind, self.layer, self.ks, self.vs, self.H = dev, kind, layer, ks, vs, H
        self.budget, self.firsts, self.lasts = budget, firsts, lasts
        self.io = io or (kind if kind != "e4m3" else "bf16")
        self.sl = np.asarray(sl)
        R = len(sl)
        self.bt, pages = _table(self.sl, P, 2, extra_cols, rng)
        self.g = _geom(2, H, D, 1 if kind == "e4m3" else 2, P, pages, style, L)
        self.lo = _layout(self.g)
        self.pool_h = _fill(self.g, self.bt, self.sl, kind, rng, layer, size)
        self.pool = torch.from_numpy(self.pool_h).to(dev)
        self.q_h = od.decode_elements(od.encode_elements(rng.normal(size=R * H * G * D), self.io), self.io).reshape(R, H * G, D)
        self.q = torch.from_numpy(self.q_h).to(dev).to(TORCH[self.io])
        self.out, self.lse = torch.full_like(self.q, 7.0), torch.full((R, H * G), 3.0, device=dev)
        self.bounds_h, self.steps_h = np.full((pages, H, 2, D), 99, np.int8), np.full((pages, H), 5, np.float32)
        self.bounds, self.steps = torch.from_numpy(self.bounds_h).to(dev), torch.from_numpy(self.steps_h).to(dev)
        self.chosen = torch.full((R, H, budget), -9, dtype=torch.int32, device=dev)
        self.d_bt, self.d_sl = torch.from_numpy(self.bt).to(dev), torch.from_numpy(self.sl.astype(np.int32)).to(dev)
        self.batch = tk.make_batch(self.d_bt, self.d_sl)
        self.scale = D ** -0.5
        self.att = tk.make_attention(self.q, self.out, TYPE[kind], TYPE[self.io], self.scale, k_scale=ks, v_scale=vs, lse=self.lse)
        self.choice = tk.make_page_choice(budget, firsts, lasts, self.bounds, self.steps, self.chosen)
        self.n = tk.check(tk.topkv_page_choice_workspace_bytes(self.lo, self.batch, self.att, self.choice))
        self.ws = torch.full((self.n + 32,), 0xFF, dtype=torch.uint8, device=dev)
        torch.cuda.synchronize()

    def bound(self, window=0, stream=None):
        b = tk.make_batch(self.d_bt, self.d_sl, window_tokens=window)
        tk.check(tk.topkv_bound_pages_layer(self.layer, self.pool, self.lo, b, TYPE[self.kind], self.bounds, self.steps, stream))

    def choose(self, stream=None):
        tk.check(tk.topkv_choose_pages_layer(self.lo, self.batch, self.att, self.choice, self.q, self.ws, self.n, stream))

    def attend(self, stream=None):
        tk.check(tk.topkv_attend_pages_layer(self.layer, self.pool, self.lo, self.batch, self.att, self.choice, self.q, self.out, self.ws, self.n, stream))

    def check_bounds(self, window=0):
        torch.cuda.synchronize()
        ot.bound_pages(self.g, self.layer, self.pool_h, self.bt, self.sl, window, self.kind, self.bounds_h, self.steps_h)
        assert np.array_equal(self.bounds.cpu().numpy(), self.bounds_h)
        assert np.array_equal(self.steps.cpu().numpy(), self.steps_h, equal_nan=True)

    def check_choice(self):
        torch.cuda.synchronize()
        want = ot.choose_pages(self.g.P, self.bt, self.sl, self.q_h, self.H, self.bounds_h, self.steps_h, self.budget, self.firsts, self.lasts)
        got = self.chosen.cpu().numpy()
        assert np.array_equal(got, want), np.argwhere(got != want)[:5]

    def result(self):
        torch.cuda.synchronize()
        assert (self.ws[self.n:] == 0xFF).all() and np.array_equal(self.pool.cpu().numpy(), self.pool_h)
        return self.out.double().cpu().numpy(), self.lse.double().cpu().numpy()

    def want(self, lists):
        whole = None
        G = self.q_h.shape[1] // self.H
        for h in range(self.H):
            rows = [ot.of_chosen(self.g.P, self.bt[r], int(s), lists[r, h]) for r, s in enumerate(self.sl)]
            bt = np.full((len(rows), max(len(x) for x, _ in rows)), -1, np.int32)
            for r, (x, _) in enumerate(rows):
                bt[r, :len(x)] = x
            part = od.attend(self.g, self.layer, self.pool_h, bt, [n for _, n in rows], self.q_h, self.kind, self.io, self.scale, k_scale=self.ks, v_scale=self.vs)
            whole = whole or tuple(np.zeros_like(x) for x in part)
            for x, y in zip(whole, part):
                x[:, h * G:(h + 1) * G] = y[:, h * G:(h + 1) * G]
        return whole

    def check(self):
        self.bound()
        self.choose()
        self.attend()
        self.check_bounds()
        self.check_choice()
        _check(self.result(), self.want(self.chosen.cpu().numpy()))


@pytest.mark.parametrize("sl, kw", [
    ([200, 33, 16], dict()), ([1, 15, 17, 0, 48, 49], dict()), ([500], dict(budget=1)), ([500], dict(budget=2, lasts=5)),
    ([500, 90], dict(budget=9, firsts=4, lasts=3)), ([500, 90], dict(budget=5, firsts=40, lasts=2)), ([500], dict(budget=31)), ([500], dict(budget=32)),
    ([500], dict(budget=100)), ([500], dict(firsts=0)),
    ([700, 300], dict(D=128, kind="fp16", style="head", budget=20)), ([700, 300], dict(D=128, kind="e4m3", ks=0.5, vs=1.5, budget=7)),
    ([700, 300], dict(D=128, kind="e4m3", io="fp16", style="padded", H=1, G=16, budget=30)),
    ([300, 77], dict(D=80, G=7)), ([300, 77], dict(D=72, kind="fp16")), ([300, 77], dict(D=96, kind="e4m3")), ([300, 77], dict(D=8, H=5, G=1)),
    ([300, 77], dict(D=16, H=3, kind="e4m3")), ([400], dict(D=256, H=1, G=24)), ([400], dict(D=200, H=1, G=33, kind="fp16")), ([400], dict(D=256, H=1, kind="e4m3")),
    ([130, 60], dict(P=1, budget=40, style="head")), ([2000], dict(P=256, style="plane")), ([300, 77], dict(P=24)), ([300], dict(P=8, budget=11)),
    ([300, 77], dict(L=3, layer=2, style="padded")), ([3000], dict(H=1, budget=100)), ([90] * 40, dict(H=1, D=16, G=1)),
    ([300, 77], dict(size=1e-30)), ([300, 77], dict(size=1e30)), ([300, 77], dict(size=1e-3, kind="fp16")),
])
def test_against_the_definition(dev, sl, kw):
    Case(dev, sl, **kw).check()


@pytest.mark.parametrize("sl, kw", [
    ([9000, 8000], dict(P=1, H=1, D=16, budget=500, lasts=8)),            # several CTAs a list
    ([70000], dict(P=2, H=1, D=8, G=1, budget=1000)),
    ([4000, 130], dict(P=1, H=1, D=16, budget=128, extra_cols=250_000)),  # keys in the workspace
])
def test_long_lists(dev, sl, kw):
    Case(dev, sl, **kw).check()


@pytest.mark.parametrize("window", [1, 16, 17, 40, 1000])
def test_bounds_of_the_last_tokens(dev, window):
    c = Case(dev, [200, 33, 16, 0, 1], P=16)
    c.bound(window)
    c.check_bounds(window)


def test_bounds_with_zeros_nan_and_infinity(dev):
    c = Case(dev, [48], H=1, D=16, P=16, budget=2, lasts=1, firsts=0)
    at = lambda page, t: od.row_offset(c.g, 0, int(c.bt[0, page]), 0, t, 0)
    for page, raw in ((0, (0, 0)), (1, (0x80, 0x7F))):
        for t in range(16):
            c.pool_h[at(page, t):at(page, t) + 32] = 0
        c.pool_h[at(page, 3) + 4:at(page, 3) + 6] = raw
    c.pool.copy_(torch.from_numpy(c.pool_h))
    c.bound()
    c.check_bounds()
    c.choose()
    c.check_choice()
    assert c.chosen.tolist() == [[[1, 2]]]                               # infinity is looked at first
    c.pool_h[at(0, 5):at(0, 5) + 2] = NAN["bf16"]
    c.pool.copy_(torch.from_numpy(c.pool_h))
    c.bound()
    c.check_bounds()
    c.choose()
    c.check_choice()
    assert c.chosen.tolist() == [[[0, 2]]]                               # of two such the lower column


def test_equal_scores_take_the_lowest_columns(dev):
    c = Case(dev, [3000], H=2, D=16, budget=60, firsts=2, lasts=3)
    c.bound()
    torch.cuda.synchronize()
    c.bounds.fill_(7)
    c.steps.fill_(1.0)
    c.choose()
    torch.cuda.synchronize()
    assert c.chosen.tolist() == [[list(range(57)) + [185, 186, 187]] * 2]
    c.bounds_h[:], c.steps_h[:] = 7, 1.0
    c.steps[c.d_bt[0, 100].long()] = c.steps_h[c.bt[0, 100]] = 1.5
    c.steps[c.d_bt[0, 30].long()] = c.steps_h[c.bt[0, 30]] = 0.5
    c.choose()
    c.check_choice()


def test_queries_of_zeros_nan_and_infinity(dev):
    c = Case(dev, [500], H=1, G=4, budget=4)
    c.bound()
    c.check_bounds()
    c.q[0, 0] = 0
    c.q[0, 1, 3] = float("nan")
    c.q[0, 2, 5] = float("inf")
    c.q_h = c.q.double().cpu().numpy()
    c.choose()
    with np.errstate(invalid="ignore"):
        c.check_choice()


def test_unusable_tables_are_reported(dev):
    c = Case(dev, [200, 77], H=1, P=8, budget=6, firsts=0, lasts=2)
    c.bound()
    c.check_bounds()
    good = c.bt.copy()
    c.bt[0, 4], c.bt[1, 9] = -3, c.g.num_pages
    c.d_bt.copy_(torch.from_numpy(c.bt))
    c.bounds.fill_(99)
    c.steps.fill_(5.0)
    c.bounds_h[:], c.steps_h[:] = 99, 5.0
    c.bound()
    c.check_bounds()
    assert tk.topkv_device_error_flags() == 2
    tk.check(tk.topkv_reset_device_error_flags())
    c.choose()
    torch.cuda.synchronize()
    assert tk.topkv_device_error_flags() == 2
    tk.check(tk.topkv_reset_device_error_flags())
    # a list of its own, with columns that are none of the request's, and one whose page is no page
    lists = np.array([[[0, 4, 7, 25, -1, 24]], [[1, 2, 2, 9, 1000, 9]]], np.int32)
    c.chosen.copy_(torch.from_numpy(lists))
    c.attend()
    got = c.result()
    assert tk.topkv_device_error_flags() == 2
    tk.check(tk.topkv_reset_device_error_flags())
    c.bt = good
    # the second request's last page holds 5 tokens; only its list's last place stands for them
    c.bt[1, 10:] = -1
    usable = [[0, 7, 24], [1, 2, 2]]
    lens = [24, 24]
    bt = np.array([[c.bt[r, j] for j in usable[r]] for r in range(2)], np.int32)
    _check(got, od.attend(c.g, 0, c.pool_h, bt, lens, c.q_h, "bf16", "bf16", c.scale))
    # lengths outside the table
    c.d_sl.copy_(torch.tensor([-5, 10 ** 6], dtype=torch.int32))
    c.bound()
    c.choose()
    c.attend()
    c.result()
    assert tk.topkv_device_error_flags() == 2
    tk.check(tk.topkv_reset_device_error_flags())


def test_same_bits_again_in_graphs_and_on_other_streams(dev):
    c = Case(dev, [2000, 300, 1], D=128, budget=40, firsts=2, lasts=3)
    c.check()
    first = [x.copy() for x in c.result()] + [c.chosen.cpu().numpy()]
    s = torch.cuda.Stream(dev)
    c.out.fill_(7.0)
    c.chosen.fill_(-9)
    torch.cuda.synchronize()
    c.bound(1, s)
    c.choose(s)
    c.attend(s)
    assert all(np.array_equal(a, b) for a, b in zip(first, list(c.result()) + [c.chosen.cpu().numpy()]))
    c.out.fill_(7.0)
    c.chosen.fill_(-9)
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        s = torch.cuda.current_stream()
        c.bound(1, s)
        c.choose(s)
        c.attend(s)
    for _ in range(3):
        gr.replay()
    assert all(np.array_equal(a, b) for a, b in zip(first, list(c.result()) + [c.chosen.cpu().numpy()]))


def test_all_pages_chosen_is_plain_attention(dev):
    c = Case(dev, [700, 300, 0, 5], D=128, budget=50)
    c.bound()
    c.choose()
    c.attend()
    sparse = c.result()
    n = tk.check(tk.topkv_attend_workspace_bytes(c.lo, c.batch, c.att))
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device=dev)
    out = c.out.clone()
    tk.check(tk.topkv_attend_layer(0, c.pool, c.lo, c.batch, c.att, c.q, c.out, ws, n))
    torch.cuda.synchronize()
    assert torch.equal(out, c.out) and np.array_equal(sparse[1], c.lse.double().cpu().numpy())


def test_settled_tables_and_known_totals(dev):
    c = Case(dev, [2000, 300, 0, 1], D=128, budget=40, firsts=2, lasts=3)
    c.check()
    lists, want = c.chosen.cpu().numpy(), None
    for flags in (0, tk.TOPKV_FLAG_TABLES_SETTLED):
        c.batch = tk.make_batch(c.d_bt, c.d_sl, total_tokens=2301, flags=flags)
        c.n = tk.check(tk.topkv_page_choice_workspace_bytes(c.lo, c.batch, c.att, c.choice))
        c.ws = torch.full((c.n + 32,), 0xFF, dtype=torch.uint8, device=dev)
        for _ in range(4):
            c.out.fill_(7.0)
            c.chosen.fill_(-9)
            c.choose()
            c.attend()
        assert np.array_equal(c.chosen.cpu().numpy(), lists)
        want = want or c.want(lists)
        _check(c.result(), want)


@pytest.mark.parametrize("kind", ["bf16", "e4m3"])
def test_offsets_beyond_32_bits(dev, kind):
    """Pages far apart: the bits of the same pages side by side."""
    c = Case(dev, [150, 20], kind=kind, budget=5)
    c.check()
    near = [x.copy() for x in c.result()] + [c.chosen.cpu().numpy()]
    far = 700_000_000
    big = torch.zeros(c.g.num_pages * far, dtype=torch.uint8, device=dev)
    big.view(c.g.num_pages, far)[:, :c.g.S_page] = c.pool.view(c.g.num_pages, c.g.S_page)
    c.lo.pool_page_stride, c.lo.pool_layer_stride = far, c.g.num_pages * far
    for t in (c.out, c.chosen):
        t.fill_(7)
    bounds, steps = c.bounds.clone(), c.steps.clone()
    c.bounds.fill_(99)
    c.steps.fill_(5)
    tk.check(tk.topkv_bound_pages_layer(0, big, c.lo, c.batch, TYPE[kind], c.bounds, c.steps))
    c.choose()
    tk.check(tk.topkv_attend_pages_layer(0, big, c.lo, c.batch, c.att, c.choice, c.q, c.out, c.ws, c.n))
    assert all(np.array_equal(a, b) for a, b in zip(near, list(c.result()) + [c.chosen.cpu().numpy()])) and c.g.num_pages * far > 1 << 32
    assert torch.equal(bounds, c.bounds) and torch.equal(steps, c.steps)


def test_scores_beyond_the_range_equal_those_without_a_finite_step(dev):
    """Both are infinite, so the lower columns win, whichever they are."""
    c = Case(dev, [640], H=1, G=2, D=16, budget=4, firsts=0, lasts=1)
    c.bound()
    torch.cuda.synchronize()
    c.bounds_h[:], c.steps_h[:] = 100, 1.0
    for column, step in ((7, 3e38), (11, np.inf), (5, 3e38), (20, np.nan), (3, 2.0)):
        c.steps_h[c.bt[0, column]] = step
    c.bounds_h[c.bt[0, 30], :, 0] = -100
    c.q.copy_(c.q.abs() * 1000)
    c.q_h = c.q.double().cpu().numpy()
    c.bounds.copy_(torch.from_numpy(c.bounds_h))
    c.steps.copy_(torch.from_numpy(c.steps_h))
    c.choose()
    c.check_choice()
    assert c.chosen.tolist() == [[[5, 7, 11, 39]]]

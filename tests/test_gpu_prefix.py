"""GPU tests of attention behind shared prefixes: the plan against plain loops, integer for integer, and the
attention against the oracle in 64 bits over all tokens (tolerances derived in oracle.decode.attend)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import decode as od, tokens as ot
from paper_2607_28633_b200 import binding as tk
from test_gpu_decode import NAN, TORCH, TYPE, _check, _geom, _layout

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
    """However little is shared, it is formed once: these cases are small."""
    tk.check(tk.topkv_reset_device_error_flags())
    before = tk.topkv_set_sharing_bytes(0)
    yield
    tk.topkv_set_sharing_bytes(before)
    assert tk.topkv_device_error_flags() == 0


def _tables(groups, P, rng, extra_cols=1, shuffle=True):
    """groups: (prefix pages, [tokens behind the prefix of each member]). Rows of all groups, mixed."""
    rows = []
    total = sum(n + sum(-(-t // P) for t in tails) for n, tails in groups) + 3
    ids, at = rng.permutation(total), 0
    for n, tails in groups:
        common, at = list(ids[at:at + n]), at + n
        for t in tails:
            k = -(-t // P)
            rows.append((n * P + t, common + list(ids[at:at + k])))
            at += k
    if shuffle:
        rows = [rows[i] for i in rng.permutation(len(rows))]
    bt = np.full((len(rows), max(len(x) for _, x in rows) + extra_cols), -1, np.int32)
    for r, (_, pages) in enumerate(rows):
        bt[r, :len(pages)] = pages
    return bt, np.array([s for s, _ in rows]), total


def _filled(g, bt, sl, kind, rng, layer=0):
    """NaN patterns everywhere but in the tokens that some request holds."""
    pool = np.empty(g.L * g.S_layer, np.uint8)
    pool[0::2], pool[1::2] = NAN[kind]
    n, done = g.d_h * g.b_p, set()
    for r, s in enumerate(sl):
        for i in range(max(int(s), 0)):
            where = (int(bt[r, i // g.P]), i % g.P)
            if where in done or not 0 <= where[0] < g.num_pages:
                continue
            done.add(where)
            for c in range(2):
                for h in range(g.h_kv):
                    a = od.row_offset(g, layer, where[0], c, where[1], h)
                    pool[a:a + n] = od.encode_elements(rng.normal(size=g.d_h), kind)
    return pool


class Case:
    def __init__(self, dev, groups, H=2, G=2, D=64, P=16, kind="bf16", io=None, style="page", L=1, layer=0, seed=0, ks=1.0, vs=1.0, tables=None,
                 q_size=1.0, scale=None):
        rng = np.random.default_rng(seed)
        self.dev, self.kind, self.layer, self.ks, self.vs = dev, kind, layer, ks, vs
        self.io = io or (kind if kind != "e4m3" else "bf16")
        self.bt, self.sl, pages = _tables(groups, P, rng) if tables is None else tables
        self.g = _geom(2, H, D, 1 if kind == "e4m3" else 2, P, pages, style, L)
        self.lo = _layout(self.g)
        self.pool_h = _filled(self.g, self.bt, self.sl, kind, rng, layer)
        self.pool = torch.from_numpy(self.pool_h).to(dev)
        R = len(self.sl)
        self.q_h = od.decode_elements(od.encode_elements(q_size * rng.normal(size=R * H * G * D), self.io), self.io).reshape(R, H * G, D)
        self.q = torch.from_numpy(self.q_h).to(dev).to(TORCH[self.io])
        self.out = torch.full_like(self.q, 7.0)
        self.lse = torch.full((R, H * G), 3.0, device=dev)
        self.d_bt = torch.from_numpy(self.bt).to(dev)
        self.d_sl = torch.from_numpy(self.sl.astype(np.int32)).to(dev)
        self.batch = tk.make_batch(self.d_bt, self.d_sl)
        self.scale = D ** -0.5 if scale is None else scale
        self.att = tk.make_attention(self.q, self.out, TYPE[kind], TYPE[self.io], self.scale, k_scale=ks, v_scale=vs, lse=self.lse)
        self.n = tk.check(tk.topkv_attend_shared_workspace_bytes(self.lo, self.batch, self.att))
        self.ws = torch.full((self.n + 32,), 0xFF, dtype=torch.uint8, device=dev)  # NaN patterns: nothing is assumed
        self.plan = torch.full((6, R), -7, dtype=torch.int32, device=dev)
        torch.cuda.synchronize()

    def make_plan(self, min_tokens=0, stream=None):
        tk.check(tk.topkv_plan_prefixes(self.lo, self.batch, min_tokens, self.plan, stream))

    def attend(self, stream=None):
        tk.check(tk.topkv_attend_shared_layer(self.layer, self.pool, self.lo, self.batch, self.att, self.plan, self.q, self.out, self.ws, self.n, stream))

    def result(self):
        torch.cuda.synchronize()
        assert (self.ws[self.n:] == 0xFF).all() and np.array_equal(self.pool.cpu().numpy(), self.pool_h)
        return self.out.double().cpu().numpy(), self.lse.double().cpu().numpy()

    def want(self):
        return od.attend(self.g, self.layer, self.pool_h, self.bt, self.sl, self.q_h, self.kind, self.io, self.scale, k_scale=self.ks, v_scale=self.vs)

    def check(self, min_tokens=0):
        self.make_plan(min_tokens)
        self.attend()
        got = self.result()
        assert np.array_equal(self.plan.cpu().numpy(), ot.plan_prefixes(self.g.P, self.g.num_pages, self.bt, self.sl, min_tokens))
        _check(got, self.want())


@pytest.mark.parametrize("groups, kw", [
    ([(3, [5, 9])], dict()),
    ([(1, [1] * 4)], dict()),
    ([(8, [5, 9, 0, 33])], dict()),                                   # one has nothing of its own; a whole tile
    ([(9, [20] * 70)], dict(G=2, H=1)),                               # 140 rows: two tiles of rows
    ([(9, [3] * 300)], dict(G=1, H=1)),                               # 300 rows: two units, the second of one tile
    ([(20, [3] * 129)], dict(G=1, H=2)),
    ([(40, [30, 700])], dict(P=24)),
    ([(0, [5, 70]), (4, [3, 3]), (30, [1, 2, 3, 200, 500]), (0, [0]), (2, [0, 0])], dict()),
    ([(0, [5, 70, 0])], dict()),                                      # nothing is shared
    ([(33, [3, 40])], dict(D=128, kind="fp16", style="head")),
    ([(33, [3, 40])], dict(D=128, kind="e4m3", ks=0.5, vs=1.5)),
    ([(33, [3, 40] * 40)], dict(D=128, kind="e4m3", io="fp16", H=1, style="padded")),
    ([(33, [3, 40])], dict(D=80, G=7)), ([(33, [3, 40])], dict(D=72, kind="fp16")), ([(33, [3, 40])], dict(D=96, kind="e4m3")),
    ([(33, [3, 40] * 5)], dict(D=256, H=1, G=16)), ([(33, [3, 40] * 5)], dict(D=192, H=1, G=24, kind="fp16")),
    ([(33, [3, 40] * 5)], dict(D=256, H=1, G=4, kind="e4m3", ks=0.25)), ([(50, [3] * 100)], dict(D=200, H=1, G=2)),
    ([(300, [3, 40])], dict(P=1, style="head")), ([(5, [3, 40])], dict(P=256, style="plane")),
    ([(7, [3, 40])], dict(D=8, H=5, G=1)), ([(7, [3, 40])], dict(D=16, H=5, G=3, kind="e4m3")),
    ([(300, [3, 900, 5])], dict(H=1, G=4, seed=3)),                   # many CTAs a unit
    ([(40, [3, 40])], dict(L=3, layer=2, style="padded")),
    ([(40, [3, 40])], dict(q_size=30.0)), ([(40, [3, 40])], dict(q_size=30.0, kind="fp16")),   # maxima that move
    ([(40, [3, 40])], dict(q_size=3e4, scale=1e-5, kind="e4m3")),
    ([(40, [3, 40])], dict(scale=-0.2)), ([(40, [3, 40])], dict(scale=0.0)),
    ([(1, [3] * 2)] * 30, dict(H=1)),                                 # many small groups
])
def test_against_the_oracle(dev, groups, kw):
    Case(dev, groups, **kw).check()


def test_long_prefix_over_all_ctas(dev):
    Case(dev, [(260, [9, 1000] + [3] * 5)], H=1, G=8, D=128, P=32).check()
    Case(dev, [(520, [9] + [3] * 7)], H=1, G=8, D=128, P=16, kind="e4m3").check()
    Case(dev, [(260, [9, 100])], H=1, G=4, D=256, P=16).check()


def test_a_plan_with_a_lower_limit_shares_less(dev):
    for least in (48, 49, 1000):
        Case(dev, [(3, [5, 9]), (6, [4, 3, 2])]).check(least)


def test_groups_within_a_group_share_what_all_of_it_shares(dev):
    bt = np.array([[4, 1, 2, 3, -1], [4, 1, 5, 6, -1], [4, 1, 2, 7, -1], [8, 1, 2, 9, -1], [-1] * 5], np.int32)
    sl = np.array([60, 50, 64, 60, 0])
    c = Case(dev, None, tables=(bt, sl, 10))
    c.check()
    assert c.plan[2].tolist() == [32, 32, 32, 0, 0]


def test_the_plan_stays_good_while_requests_grow(dev):
    c = Case(dev, [(9, [40, 70, 33]), (3, [20, 30])])
    whole = c.sl.copy()
    c.d_sl.copy_(torch.from_numpy(whole - 15))
    c.make_plan()
    c.d_sl.copy_(torch.from_numpy(whole))
    c.attend()
    _check(c.result(), c.want())


def test_a_freed_row_is_attended_to_on_its_own(dev):
    c = Case(dev, [(9, [40, 70, 33, 5])])
    c.make_plan()
    for r in (0, 2):
        c.sl[r] = 0
        c.d_sl[r] = 0
        c.attend()
        _check(c.result(), c.want())


def test_contradicting_plans_reach_nothing_outside(dev):
    """Every field by turns holds what no plan says: results are numbers of some kind, error bits may be raised."""
    c = Case(dev, [(9, [40, 70, 33]), (3, [20, 30]), (0, [17])])
    c.make_plan()
    torch.cuda.synchronize()
    good, rng = c.plan.clone(), np.random.default_rng(5)
    R = len(c.sl)
    for trial in range(40):
        bad = good.clone()
        for row in ([trial % 6] if trial < 24 else range(6)):
            bad[row] = torch.from_numpy(rng.integers(*[(-3, R + 3), (-2 ** 31, 2 ** 31 - 1), (0, 200), (0, R)][trial // 6 % 4], size=R).astype(np.int32)).to(dev)
        c.plan.copy_(bad)
        c.attend()
        c.result()
        tk.check(tk.topkv_reset_device_error_flags())
    c.plan.copy_(good)
    c.attend()
    _check(c.result(), c.want())


def test_pages_outside_the_pool_are_not_visible(dev):
    c = Case(dev, [(20, [40, 70, 33])], H=1, P=8)
    c.make_plan()
    torch.cuda.synchronize()
    alone = c.bt.copy()
    bad = c.bt.copy()
    bad[:, [3, 11]] = [[-5, c.g.num_pages]]
    c.d_bt.copy_(torch.from_numpy(bad))
    c.attend()
    torch.cuda.synchronize()
    assert tk.topkv_device_error_flags() == 2
    tk.check(tk.topkv_reset_device_error_flags())
    # the same without these pages
    keep = [j for j in range(c.bt.shape[1]) if j not in (3, 11)]
    c.bt, c.sl = np.ascontiguousarray(alone[:, keep]), c.sl - 16
    _check(c.result(), c.want())
    # no usable page at all in the prefix
    bad[:, :20] = -1
    c.bt, c.sl = np.ascontiguousarray(alone[:, 20:]), c.sl - 18 * 8
    c.d_bt.copy_(torch.from_numpy(bad))
    c.attend()
    torch.cuda.synchronize()
    assert tk.topkv_device_error_flags() == 2
    tk.check(tk.topkv_reset_device_error_flags())
    _check(c.result(), c.want())


def test_same_bits_again_and_equal_to_graphs_and_other_streams(dev):
    c = Case(dev, [(40, [30, 700, 9]), (7, [1] * 9)], D=128)
    c.make_plan()
    c.attend()
    first = [x.copy() for x in c.result()]
    for stream in (None, torch.cuda.Stream(dev)):
        c.out.fill_(7.0)
        c.lse.fill_(3.0)
        torch.cuda.synchronize()
        c.make_plan(stream=stream)
        c.attend(stream)
        assert all(np.array_equal(a, b) for a, b in zip(first, c.result()))
    c.out.fill_(7.0)
    c.plan.fill_(-1)
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        s = torch.cuda.current_stream()
        c.make_plan(stream=s)
        c.attend(s)
        c.attend(s)
    for _ in range(3):
        gr.replay()
    assert all(np.array_equal(a, b) for a, b in zip(first, c.result()))


def test_scores_of_minus_infinity_and_nan_stay_with_their_rows(dev):
    c = Case(dev, [(9, [20, 30, 40])], H=1, G=2)
    c.make_plan()
    c.q[1, 0, 0] = float("nan")
    c.q[2, 1, 3] = float("inf")
    c.attend()
    out, lse = c.result()
    ref, ref_lse, tol, tol_lse = c.want()
    bad = np.zeros(lse.shape, bool)
    bad[1, 0] = bad[2, 1] = True
    assert np.isnan(out[bad]).all()
    assert (np.abs(out - ref) <= tol)[~bad].all() and (np.abs(lse - ref_lse) <= tol_lse)[~bad].all()


def test_large_plan(dev):
    rng = np.random.default_rng(1)
    R, maxp = 1500, 200
    bt = rng.integers(0, 9, size=(R, 1)).astype(np.int32) * 1000 + np.arange(maxp, dtype=np.int32)
    for r in range(R):
        bt[r, rng.integers(50, maxp):] = rng.integers(0, 10000)
    bt[7, 0], bt[9, 0] = -1, 10 ** 6
    sl = rng.integers(0, maxp * 4, size=R)
    plan = torch.full((6, R), -7, dtype=torch.int32, device=dev)
    b = tk.make_batch(torch.from_numpy(bt).to(dev), torch.from_numpy(sl.astype(np.int32)).to(dev))
    tk.check(tk.topkv_plan_prefixes(tk.make_layout(1, 2, 1, 64, 2, 4, 10000), b, 8, plan))
    torch.cuda.synchronize()
    assert np.array_equal(plan.cpu().numpy(), ot.plan_prefixes(4, 10000, bt, sl, 8))


def test_small_groups_are_left_to_their_requests(dev):
    """The default limit: nothing here saves that much, alone or mixed with a group that does."""
    groups = [(9, [40, 70, 0]), (3, [20, 30]), (0, [0, 17])]
    for limit in (tk.TOPKV_DEFAULT_SHARING_BYTES, 2 * 9 * 16 * 2 * 2 * 64 * 2, 2 * 9 * 16 * 2 * 2 * 64 * 2 + 512):
        tk.topkv_set_sharing_bytes(limit)
        Case(dev, groups).check()
    tk.topkv_set_sharing_bytes(tk.TOPKV_DEFAULT_SHARING_BYTES)
    c = Case(dev, groups)
    c.make_plan()
    c.attend()
    out, lse = c.result()
    n = tk.check(tk.topkv_attend_workspace_bytes(c.lo, c.batch, c.att))
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device=dev)
    tk.check(tk.topkv_attend_layer(0, c.pool, c.lo, c.batch, c.att, c.q, c.out, ws, n))
    again, lse2 = c.result()
    assert np.array_equal(out, again) and np.array_equal(lse, lse2)
    # many short requests, a warp each
    tk.topkv_set_sharing_bytes(0)
    Case(dev, [(1, [1, 5] * 60), (0, [3] * 400)], H=8, G=1, D=16).check()
    tk.topkv_set_sharing_bytes(tk.TOPKV_DEFAULT_SHARING_BYTES)
    Case(dev, [(1, [1, 5] * 60), (0, [3, 0] * 200)], H=8, G=1, D=16).check()


@pytest.mark.parametrize("limit", [1, 2 * 9 * 16 * 2 * 2 * 64, 1 << 40])
def test_small_groups_of_an_8_bit_cache(dev, limit):
    """Two and three members are left to their requests at any limit but 0, four and more by what they save."""
    tk.topkv_set_sharing_bytes(limit)
    Case(dev, [(9, [40, 70]), (8, [5, 0, 30]), (9, [1, 2, 3, 4]), (9, [9, 8, 7, 6, 5]), (0, [17, 0])], kind="e4m3", vs=0.5).check()


@pytest.mark.parametrize("tails, kw", [
    ([0], dict(H=8)),  # a request alone: nothing to join but its own parts
    ([9, 100, 0, 2000], dict(H=8, D=128)),
    ([3, 1], dict(H=1, D=64, G=1)),
    ([3, 700, 0], dict(H=1, G=16, D=256)),
    ([5, 60], dict(H=1, G=3, D=16, kind="e4m3")),
    ([2] * 40, dict(H=2, G=8, D=128)),
])
def test_prefix_of_many_parts(dev, tails, kw):
    """A long prefix of few heads is cut into many ranges: the join's threads share a row's parts, or have several rows."""
    Case(dev, [(500, tails)], **kw).check()


def test_sharing_limit_refuses_negative_values(dev):
    assert tk.topkv_set_sharing_bytes(-1) == tk.TOPKV_ERR_INVALID_ARG and tk.topkv_set_sharing_bytes(0) == 0


def test_a_plan_with_more_work_than_its_line_counts(dev):
    """Every row its own leader of all rows behind it, a million tokens each: refused on the device."""
    R, maxp, P = 2400, 4096, 256
    lo = tk.make_layout(1, 2, 1, 16, 2, P, 1)
    pool = torch.zeros(2 * P * 16, dtype=torch.bfloat16, device=dev)
    bt, sl = torch.zeros((R, maxp), dtype=torch.int32, device=dev), torch.full((R,), maxp * P, dtype=torch.int32, device=dev)
    row = torch.arange(R, dtype=torch.int32, device=dev)
    plan = torch.stack([row, sl, sl, torch.full_like(row, R), row, row]).contiguous()
    q = torch.zeros((R, 16, 16), dtype=torch.bfloat16, device=dev)
    out = torch.full_like(q, 7.0)
    b, att = tk.make_batch(bt, sl), tk.make_attention(q, out, TYPE["bf16"], TYPE["bf16"], 0.25)
    n = tk.check(tk.topkv_attend_shared_workspace_bytes(lo, b, att))
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device=dev)
    torch.cuda.synchronize()
    tk.check(tk.topkv_attend_shared_layer(0, pool, lo, b, att, plan, q, out, ws, n))
    torch.cuda.synchronize()
    assert tk.topkv_device_error_flags() == 2 and (out == 0).all()
    tk.check(tk.topkv_reset_device_error_flags())


def test_settled_tables_and_known_totals(dev):
    """Tables and plan that stay as they are, calls behind each other, lengths' sum known or not."""
    c = Case(dev, [(40, [30, 700, 9]), (7, [1] * 9), (0, [1, 0, 300])], D=128)
    c.make_plan()
    c.attend()
    first = [x.copy() for x in c.result()]
    plain = c.batch
    c.batch = tk.make_batch(c.d_bt, c.d_sl, flags=tk.TOPKV_FLAG_TABLES_SETTLED)
    for _ in range(5):
        c.out.fill_(7.0)
        for _ in range(3):
            c.attend()
        assert all(np.array_equal(a, b) for a, b in zip(first, c.result()))
    for flags in (0, tk.TOPKV_FLAG_TABLES_SETTLED):
        c.batch = tk.make_batch(c.d_bt, c.d_sl, total_tokens=int(sum(c.sl)), flags=flags)
        c.out.fill_(7.0)
        c.n = tk.check(tk.topkv_attend_shared_workspace_bytes(c.lo, c.batch, c.att))
        c.ws = torch.full((c.n + 32,), 0xFF, dtype=torch.uint8, device=dev)
        c.attend()
        c.attend()
        _check(c.result(), c.want())
    assert plain.flags == 0


def test_two_calls_at_once(dev):
    cases = [Case(dev, [(40, [30, 700, 9]), (7, [1] * 9)], D=128), Case(dev, [(130, [30, 7, 9, 1])], D=64, P=24, kind="e4m3")]
    first = []
    for c in cases:
        c.make_plan()
        c.attend()
        first.append([x.copy() for x in c.result()])
        c.out.fill_(7.0)
    streams = [torch.cuda.Stream(dev) for _ in cases]
    torch.cuda.synchronize()
    for _ in range(20):
        for c, s in zip(cases, streams):
            c.make_plan(stream=s)
            c.attend(s)
    for c, want in zip(cases, first):
        assert all(np.array_equal(a, b) for a, b in zip(want, c.result()))


@pytest.mark.parametrize("P, kind", [(16, "bf16"), (12, "fp16"), (16, "e4m3"), (12, "e4m3")])
def test_offsets_beyond_32_bits(dev, P, kind):
    """Pages far apart, which come by tensor copies (P 16) or row by row: the bits of the same pages side by side."""
    c = Case(dev, [(4, [5, 30])], P=P, kind=kind)
    c.make_plan()
    c.attend()
    near = [x.copy() for x in c.result()]
    far = 800_000_000
    big = torch.zeros(c.g.num_pages * far, dtype=torch.uint8, device=dev)
    big.view(c.g.num_pages, far)[:, :c.g.S_page] = c.pool.view(c.g.num_pages, c.g.S_page)
    c.lo.pool_page_stride, c.lo.pool_layer_stride = far, c.g.num_pages * far
    c.out.fill_(7.0)
    tk.check(tk.topkv_attend_shared_layer(0, big, c.lo, c.batch, c.att, c.plan, c.q, c.out, c.ws, c.n))
    assert all(np.array_equal(a, b) for a, b in zip(near, c.result())) and c.g.num_pages * far > 1 << 32


def _formed(c):
    """Leaders of the groups whose shared tokens were formed once: their records in the workspace are written."""
    R = len(c.sl)
    at = 16 * R + 16  # behind the join records and the line's header
    records = c.ws[at:at + 48 * R].view(R, 48).cpu()
    return [r for r in range(R) if not (records[r] == 0xFF).all()]


def _alone(c):
    """The same requests, each attended to on its own."""
    n = tk.check(tk.topkv_attend_workspace_bytes(c.lo, c.batch, c.att))
    ws = torch.empty(max(n, 16), dtype=torch.uint8, device=c.dev)
    tk.check(tk.topkv_attend_layer(c.layer, c.pool, c.lo, c.batch, c.att, c.q, c.out, ws, n))
    return c.result()


@pytest.mark.parametrize("kind, members, counted", [("bf16", 2, 1), ("fp16", 5, 4), ("e4m3", 4, 1), ("e4m3", 6, 3)])
def test_a_group_is_formed_from_the_limit_on(dev, kind, members, counted):
    """The limit is a number of bytes that the group has to save at least, whatever a token's bytes are."""
    saved = counted * 9 * 16 * 2 * 2 * 64 * (1 if kind == "e4m3" else 2)
    for limit, formed in [(1, True), (saved - 1, True), (saved, True), (saved + 1, False), (saved + 511, False), (2 ** 63 - 1, False)]:
        tk.topkv_set_sharing_bytes(limit)
        c = Case(dev, [(9, [40, 70, 5, 0, 9, 1][:members])], kind=kind)
        c.check()
        assert _formed(c) == ([0] if formed else []), limit
        if not formed:
            got = [x.copy() for x in c.result()]
            assert all(np.array_equal(a, b) for a, b in zip(got, _alone(c)))


def test_two_and_three_members_of_an_8_bit_cache_are_left_to_their_requests(dev):
    """... at any limit but 0: converting a tile costs as much as two more members' reading."""
    groups = [(9, [40, 70]), (8, [5, 0, 30]), (9, [1, 2, 3, 4]), (9, [9, 8, 7, 6, 5]), (0, [17, 0])]
    for limit, sizes in [(0, [2, 3, 4, 5]), (1, [4, 5]), (2 * 2 * 64 - 1, [4, 5]), (1 << 40, [])]:
        tk.topkv_set_sharing_bytes(limit)
        c = Case(dev, groups, kind="e4m3", vs=0.5)
        c.check()
        plan = c.plan.cpu().numpy()
        assert sorted(plan[tk.TOPKV_PLAN_MEMBERS][r] for r in _formed(c)) == sizes, limit
    out, lse = [x.copy() for x in c.result()]
    again, lse2 = _alone(c)
    assert np.array_equal(out, again) and np.array_equal(lse, lse2)


@pytest.mark.parametrize("q_size, scale, ks", [(1e-18, 0.0, 1.0), (1e-37, 0.125, 1e-9), (1e-37, -0.125, 1e-9), (1e-30, 1e-12, 0.5), (0.0, 0.0, 1.0)])
@pytest.mark.parametrize("kind, io", [("e4m3", "bf16"), ("e4m3", "fp16"), ("bf16", "bf16")])
def test_factors_of_scores_below_the_range_of_32_bits(dev, kind, io, q_size, scale, ks):
    """A prefix that ends inside a tile, of which a row's factor is zero or rounds to it: all tokens weigh the same."""
    c = Case(dev, [(3, [5, 9]), (11, [1, 0, 2])], kind=kind, io=io, q_size=q_size, scale=scale, ks=ks if kind == "e4m3" else 1.0)
    c.check()


@pytest.mark.parametrize("D, pages", [(64, 1), (128, 1), (128, 9), (40, 20)])
def test_bf16_weights_of_shared_tokens_keep_sixteen_bits(dev, D, pages):
    """Two values that nearly cancel, as for attention to each request's own tokens: a weight is split into two bf16
    values, the second of what the first leaves, 2^-8 of 2^-8. The other tokens have values of zero."""
    G = 16
    c = Case(dev, [(pages, [0, 1, 3])], H=1, G=G, D=D)
    q = np.zeros((3, G, D))
    q[:, :, 0] = -np.arange(1, G + 1) / 8
    w = np.exp(q[0, :, 0])
    k, v = np.zeros((16 * pages + 3, D)), np.zeros((16 * pages + 3, D))
    k[1, 0] = 1.0
    v[0, :G], v[1, :G] = od.decode_elements(od.encode_elements(w, "bf16"), "bf16"), -1.0
    for r, s in enumerate(c.sl):
        for i in range(int(s)):
            for plane, x in ((0, k), (1, v)):
                a = od.row_offset(c.g, 0, int(c.bt[r, i // 16]), plane, i % 16, 0)
                c.pool_h[a:a + 2 * D] = od.encode_elements(x[i], "bf16")
    c.pool.copy_(torch.from_numpy(c.pool_h))
    c.q.copy_(torch.from_numpy(q))
    c.scale = c.att.scale = 1.0
    c.make_plan()
    c.attend()
    got = c.result()
    want = od.attend(c.g, 0, c.pool_h, c.bt, c.sl, q, "bf16", "bf16", 1.0, weight_step=2.0 ** -16)
    coarse = od.attend(c.g, 0, c.pool_h, c.bt, c.sl, q, "bf16", "bf16", 1.0)
    assert _formed(c) == [0]
    _check(got, want)
    own = np.arange(G)  # the bound would not let 8 bits through
    assert (want[2][:, own, own] < coarse[2][:, own, own] / 4).all()


def test_a_shared_prefix_is_as_exact_as_reading_it_again(dev):
    """The same cache both ways: results differ by the rounding of the output."""
    c = Case(dev, [(64, [9, 40, 0, 17])], D=128, H=2, G=4, seed=4)
    c.make_plan()
    c.attend()
    once, lse = [x.copy() for x in c.result()]
    each, lse_each = _alone(c)
    want = od.attend(c.g, 0, c.pool_h, c.bt, c.sl, c.q_h, "bf16", "bf16", c.scale, weight_step=2.0 ** -16)
    for got in ((once, lse), (each, lse_each)):
        _check(got, want)
    assert (np.abs(once - each) <= 2 * want[2]).all()


@pytest.mark.parametrize("kw", [dict(), dict(D=128, G=4, kind="e4m3"), dict(D=256, H=1, G=16), dict(H=8, G=8, D=64, kind="fp16", style="head")])
def test_a_callers_plan_has_its_groups_in_any_order(dev, kw):
    """Groups stand in ORDER last first, or mixed, members behind a leader that is not the lowest of them, and share
    fewer tokens than they could, down to parts of a page."""
    groups = [(9, [40, 70, 33]), (30, [20, 30] * 9), (12, [1, 0, 5, 9]), (0, [17, 3]), (50, [2, 3])]
    for seed in range(4):
        c = Case(dev, groups, seed=seed, **kw)
        c.make_plan()
        torch.cuda.synchronize()
        auto, rng = c.plan.cpu().numpy(), np.random.default_rng(seed)
        plan, place = np.zeros_like(auto), 0
        leaders = sorted(set(auto[tk.TOPKV_PLAN_LEADER].tolist()), reverse=True)
        for lead in leaders if seed == 0 else rng.permutation(leaders):
            members = rng.permutation(np.flatnonzero(auto[tk.TOPKV_PLAN_LEADER] == lead))
            shared = int(auto[tk.TOPKV_PLAN_SHARED][lead])
            shared = shared if seed < 2 else int(rng.integers(0, shared + 1))
            for r in members:
                plan[tk.TOPKV_PLAN_LEADER, r], plan[tk.TOPKV_PLAN_SHARED, r] = members[0], shared
                plan[tk.TOPKV_PLAN_MEMBERS, r], plan[tk.TOPKV_PLAN_PLACE, r], plan[tk.TOPKV_PLAN_ORDER, place] = len(members), place, r
                place += 1
        c.plan.copy_(torch.from_numpy(plan))
        c.attend()
        _check(c.result(), c.want())


def test_a_plan_whose_groups_overlap_is_reported(dev):
    """More rows in all groups than there are: no room for their parts, so nothing is formed."""
    c = Case(dev, [(9, [40, 70, 33]), (4, [3, 9, 5])])
    c.make_plan()
    c.plan[tk.TOPKV_PLAN_MEMBERS] = 6
    c.plan[tk.TOPKV_PLAN_PLACE] = torch.where(c.plan[tk.TOPKV_PLAN_LEADER] == 0, c.plan[tk.TOPKV_PLAN_PLACE], c.plan[tk.TOPKV_PLAN_PLACE] - 3)
    c.attend()
    c.result()
    assert tk.topkv_device_error_flags() == 2
    tk.check(tk.topkv_reset_device_error_flags())

"""The paged KV cache on the GPU against its definition in 64 bits: append, and
attention within the bound that tests/paged_ref.py derives."""
import numpy as np
import pytest
import torch

from paper_2510_26843_amd import cas
from tests import paged_ref as P
from tests.kv4_ref import bf16

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _rng(*what):
    return np.random.default_rng([12, *what])


def _bf(x):
    return torch.from_numpy(np.asarray(x, dtype=np.float32)).to(torch.bfloat16).to(DEV)


def _i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def _np(x):
    return x.double().cpu().numpy()


def _rope(hd, n, theta=1e4):
    a = np.arange(n)[:, None] * theta ** (-2.0 * np.arange(hd // 2) / hd)
    return np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)


def _tree(r, n):
    """Ancestor-or-self masks of a random tree."""
    masks = [1]
    for i in range(1, n):
        masks.append(masks[int(r.integers(max(0, i - 4), i))] | 1 << i)
    return masks


def _words(masks):
    w = np.array([[m & (2**64 - 1), m >> 64] for m in masks], dtype=np.uint64).reshape(-1, 2)
    return torch.from_numpy(w.view(np.int64).copy()).to(DEV)


class _Batch:
    """Sequences of (rows, committed slots, earlier nodes) with random keys and
    values, in pages of a shuffled pool.  Everything no row may see holds NaN:
    free pages, slots past a sequence's, and the table past its pages."""

    slots = 0  # the least length of a table

    def __init__(self, seqs, H, Hkv, hd, page=32, tree=False, sink=0, window=0, std=1.28, spare_rows=0, seed=0):
        r = _rng(H, hd, page, seed, *[x for s in seqs for x in s])
        self.seqs, self.H, self.Hkv, self.hd, self.page = seqs, H, Hkv, hd, page
        self.sink, self.window = sink, window
        need = [-(-sum(s) // page) if s[0] else -(-s[1] // page) for s in seqs]
        n_pages = sum(need) + 2
        ids, width = r.permutation(n_pages), max(need + [1, -(-self.slots // page)]) + 1
        self.table = np.full((len(seqs), width), -7, np.int32)
        self.pool = np.full((n_pages, 2, Hkv, page * hd), np.nan)
        self.kv, at = [], 0
        for b, (s, n) in enumerate(zip(seqs, need)):
            self.table[b, :n] = ids[at : at + n]
            at += n
            k, v = (bf16(r.normal(0, std, (Hkv, sum(s), hd))) for _ in "kv")
            self.kv.append((k, v))
            if s[0]:
                for slot in range(sum(s)):
                    P.put(self.pool, hd, page, self.table[b], slot, k[:, slot], v[:, slot])
        self.rows = [s[0] for s in seqs]
        self.N = sum(self.rows) + spare_rows
        self.start = np.concatenate([[0], np.cumsum(self.rows)])
        self.q = bf16(r.normal(0, 1, (self.N, H, hd)))
        self.masks = None
        if tree:
            self.masks = []
            for t, _, nodes in seqs:
                self.masks.append(_tree(r, nodes + t)[nodes:] if t else [])
        self.pages, self.qd = _bf(self.pool), _bf(self.q)
        self.anc = _words([m for ms in self.masks for m in ms] + [0] * spare_rows) if tree else None
        self.device_table, self.device_start = _i32(self.table), _i32(self.start)
        self.ctx, self.nodes = _i32([s[1] for s in seqs]), _i32([s[2] for s in seqs])

    def cache(self, max_rows=0):
        return cas.Paged(self.pages, self.page, self.hd, self.device_table, self.device_start, self.ctx, self.N, max_rows,
                         self.nodes)

    def run(self, max_rows=0, **kw):
        out = torch.full((self.N, self.H * self.hd), 7.0, dtype=torch.bfloat16, device=DEV)
        cas.op_attention_paged(self.cache(max_rows), self.qd, out, anc=self.anc, sink=self.sink, window=self.window, **kw)
        return out

    def check(self, out):
        got = _np(out).reshape(self.N, self.H, self.hd)
        assert (got[self.start[-1] :] == 7.0).all()
        for b, (t, Lc, nodes) in enumerate(self.seqs):
            if t == 0:
                continue
            see = P.visible(t, Lc, nodes, self.masks and self.masks[b], self.sink, self.window)
            rows = slice(self.start[b], self.start[b + 1])
            ref, err = P.attention(self.q[rows], *self.kv[b], see)
            over = np.abs(got[rows] - ref) / err
            assert np.isfinite(got[rows]).all() and over.max() <= 1, (b, np.isfinite(got[rows]).all(), over.max())


@pytest.fixture(params=[0, 8193], ids=["short table", "long table"])
def table(request, monkeypatch):
    """Few rows go 32 to a unit where no sequence can be long, 128 to one where one can."""
    monkeypatch.setattr(_Batch, "slots", request.param)


HEADS = [(8, 2, 64), (4, 4, 128), (8, 1, 128), (6, 2, 64), (10, 2, 128)]
BATCHES = {
    "one token": [(1, 0, 0)],
    "tile edges": [(1, 30, 0), (1, 31, 0), (1, 32, 0), (1, 63, 0), (1, 64, 0)],
    "decode": [(1, 700, 0), (1, 3, 0), (0, 50, 0), (1, 0, 0), (1, 129, 0), (0, 0, 0)],
    "small chunks": [(3, 61, 0), (17, 0, 0), (1, 255, 0), (5, 100, 7)],
    "chunk": [(67, 33, 0)],
    "chunk and decode": [(130, 200, 0), (1, 500, 0), (1, 31, 0), (33, 0, 0)],
    "long chunk": [(300, 77, 0)],
}


@pytest.mark.usefixtures("table")
@pytest.mark.parametrize("H,Hkv,hd", HEADS)
@pytest.mark.parametrize("seqs", BATCHES.values(), ids=BATCHES)
def test_causal(H, Hkv, hd, seqs):
    c = _Batch(seqs, H, Hkv, hd, page=64, spare_rows=3)
    c.check(c.run())
    c.check(c.run(max_rows=max(c.rows)))


@pytest.mark.usefixtures("table")
@pytest.mark.parametrize("H,Hkv,hd", HEADS[:3])
@pytest.mark.parametrize("seqs", [[(1, 0, 0)], [(1, 31, 3), (4, 64, 60), (128, 40, 0)], [(61, 300, 0), (0, 9, 0), (7, 5, 121)],
                                  [(32, 97, 0), (32, 0, 0), (15, 700, 17), (16, 33, 0)]])
def test_trees(H, Hkv, hd, seqs):
    c = _Batch(seqs, H, Hkv, hd, tree=True)
    c.check(c.run())
    c.check(c.run(max_rows=max(c.rows)))


@pytest.mark.usefixtures("table")
@pytest.mark.parametrize("H,Hkv,hd", HEADS[:2])
@pytest.mark.parametrize("tree", [False, True])
@pytest.mark.parametrize("sink,window", [(4, 64), (0, 1), (100, 33), (33, 3), (0, 500), (5000, 7), (2**31 - 1, 1), (4, 2**31 - 1)])
def test_window(H, Hkv, hd, tree, sink, window):
    c = _Batch([(1, 500, 0), (70, 130, 9), (3, 40, 0), (1, 0, 0), (20, 0, 0)], H, Hkv, hd, tree=tree, sink=sink, window=window)
    c.check(c.run())


@pytest.mark.usefixtures("table")
@pytest.mark.parametrize("page", [32, 128, 1024, 4096])
def test_page_sizes(page):
    c = _Batch([(1, 1500, 0), (40, 1000, 0), (1, 33, 0)], 8, 2, 64, page=page)
    c.check(c.run())


@pytest.mark.usefixtures("table")
@pytest.mark.parametrize("H,Hkv,hd", [(8, 1, 128), (4, 2, 64), (4, 4, 128)])
@pytest.mark.parametrize("seqs", [[(1, 20001, 0)], [(1, 9000, 0), (1, 40, 0), (2, 3000, 0)], [(40, 6000, 0), (1, 5000, 0)]],
                         ids=["one", "ragged", "chunk"])
def test_split(H, Hkv, hd, seqs):
    """Long sequences: shares of a unit, joined by the second kernel."""
    c = _Batch(seqs, H, Hkv, hd, page=256)
    assert cas.paged_work_bytes(c.cache(), H) > 0
    first = c.run()
    c.check(first)
    assert torch.equal(first, c.run())  # (no order of atomics, no stale share)


@pytest.mark.usefixtures("table")
def test_many_sequences():
    """More sequences than lanes, idle ones among them."""
    r = _rng(77)
    seqs = [(int(r.integers(0, 4)), int(r.integers(0, 90)), int(r.integers(0, 3))) for _ in range(203)]
    seqs[150] = (2, 4000, 0)
    c = _Batch(seqs, 4, 2, 64, spare_rows=1)
    c.check(c.run())
    c.check(c.run(max_rows=3))


@pytest.mark.usefixtures("table")
@pytest.mark.parametrize("std", [1e-20, 0.02, 30.0])
def test_ranges(std):
    c = _Batch([(9, 200, 0), (50, 100, 0)], 8, 2, 64, std=std)
    c.check(c.run())


def test_a_row_that_sees_nothing_gives_zeros():
    c = _Batch([(3, 0, 0), (2, 0, 0)], 4, 2, 64, tree=True)
    c.masks = [[1, 0, 5], [0, 0]]
    c.anc = _words([1, 0, 5, 0, 0])
    out = c.run()
    assert (out[1] == 0).all() and (out[3:] == 0).all()
    c.check(out)


@pytest.mark.usefixtures("table")
@pytest.mark.parametrize("hd", [64, 128])
def test_rows_of_a_large_unit_that_see_nothing_give_zeros(hd):
    seqs = [(60, 0, 0), (40, 5, 0), (50, 0, 70)]
    c = _Batch(seqs, 4, 1, hd, tree=True)
    c.masks[0] = [0] * 60
    c.masks[2][7:30] = [0] * 23
    c.anc = _words([m for ms in c.masks for m in ms])
    out = c.run()
    assert (out[:60] == 0).all() and (out[107:130] == 0).all()
    c.check(out)


@pytest.mark.usefixtures("table")
@pytest.mark.parametrize("max_rows", [1, 0])
@pytest.mark.parametrize("seqs,slot", [([(6, 100, 0), (1, 40, 0)], 102), ([(6, 100, 0), (1, 40, 0)], 5),
                                       ([(80, 60, 0), (1, 40, 0)], 130), ([(80, 60, 0), (1, 40, 0)], 33)])
def test_values_that_are_not_finite_reach_their_rows_only(seqs, slot, max_rows):
    for what in "kv":
        c = _Batch(seqs, 4, 2, 64)
        want = _np(c.run(max_rows)).reshape(-1, 4, 64)
        p, at = c.table[0, slot // 32], slot // 32 * 32 % 32
        places = (P.key_places if what == "k" else P.value_places)(64)[slot % 32, 32:]
        c.pages[p, "kv".index(what), 1, torch.from_numpy(at + places).to(DEV)] = float("nan") if what == "k" else float("inf")
        got = _np(c.run(max_rows)).reshape(-1, 4, 64)
        sees = P.visible(*seqs[0], None, 0, 0)[:, slot]
        bad = np.zeros(got.shape, bool)
        bad[np.ix_(np.flatnonzero(sees), [2, 3], np.arange(64) if what == "k" else np.arange(32, 64))] = True
        assert np.array_equal(~np.isfinite(got), bad)
        assert np.array_equal(got[~bad], want[~bad])


@pytest.mark.usefixtures("table")
@pytest.mark.parametrize("seqs", [[(6, 100, 0)], [(80, 60, 0)]])
@pytest.mark.parametrize("slot", [5, 40])
@pytest.mark.parametrize("value", [float("inf"), float("-inf")])
def test_infinite_keys(seqs, slot, value):
    """A score of +infinity gives NaN, one of -infinity takes its slot out."""
    c = _Batch(seqs, 4, 2, 64)
    t, Lc, _ = seqs[0]
    c.pages[c.table[0, slot // 32], 0, 1, int(P.key_places(64)[slot % 32, 7])] = value
    got = _np(c.run()).reshape(-1, 4, 64)
    see = P.visible(t, Lc, 0, None, 0, 0)
    without = see.copy()
    without[:, slot] = False
    (ref, err), (ref0, err0) = (P.attention(c.q, *c.kv[0], x) for x in (see, without))
    ref[:, 2:], err[:, 2:] = ref0[:, 2:], err0[:, 2:]
    nan = see[:, slot, None] & (np.sign(c.q[..., 7]) == np.sign(value))
    nan[:, :2] = False
    assert np.isnan(got[nan]).all() and (np.abs(got - ref) <= err)[~nan].all()


@pytest.mark.usefixtures("table")
def test_pages_outside_the_pool_and_lengths_outside_the_table():
    """Rows that see such a page, and sequences that do not fit: NaN.  The others as ever."""
    seqs = [(2, 70, 0), (2, 70, 0), (1, 40, 0), (3, 10, 0), (2, 5, 0)]
    for max_rows in (0, 3):
        c = _Batch(seqs, 4, 2, 64)
        want = _np(c.run(max_rows))
        t = c.table.copy()
        t[0, 1] = c.pool.shape[0]
        t[1, 0] = -1
        c.device_table = _i32(t)
        c.ctx = _i32([70, 70, 40, c.table.shape[1] * 32 - 2, -1])
        got = _np(c.run(max_rows))
        assert np.isnan(got[:4]).all() and np.isnan(got[5:]).all()
        assert np.array_equal(got[4], want[4])


def test_trees_of_more_than_128_nodes_give_nan():
    c = _Batch([(2, 70, 127), (2, 70, 126)], 4, 2, 64)
    c.anc = _words([0] * 4)
    got = _np(c.run())
    assert np.isnan(got[:2]).all() and np.isfinite(got[2:]).all()


@pytest.mark.usefixtures("table")
def test_row_numbers_that_are_not_rows():
    """Sequences whose rows do not lie in the call's take no part."""
    c = _Batch([(2, 70, 0), (2, 40, 0), (1, 10, 0)], 4, 2, 64)
    want = _np(c.run())
    c.device_start = _i32([0, 2, 99, 5])
    got = _np(c.run())
    assert np.array_equal(got[:2], want[:2]) and (got[2:] == 7.0).all()
    c.device_start = _i32([-3, 2, 4, 5])
    got = _np(c.run())
    assert (got[:2] == 7.0).all() and np.array_equal(got[2:], want[2:])


def test_shared_pages():
    """Two sequences over the same committed pages (a common prompt)."""
    c = _Batch([(1, 200, 0), (1, 230, 0)], 4, 2, 64)
    c.table[1, :6] = c.table[0, :6]
    c.device_table = _i32(c.table)
    for x, y in zip(c.kv[0], c.kv[1]):
        y[:, :192] = x[:, :192]
    c.check(c.run())


# ---------------------------------------------------------------- append

@pytest.mark.parametrize("H,Hkv,hd", [(8, 2, 64), (4, 4, 128), (3, 1, 128)])
@pytest.mark.parametrize("seqs", [[(1, 0, 0)], [(1, 31, 0), (1, 32, 0), (0, 5, 0), (2, 63, 0)], [(33, 31, 0), (100, 0, 0), (3, 6, 4)],
                                  [(300, 17, 0)], [(32, 32, 0), (64, 64, 0)]])
@pytest.mark.parametrize("form", ["packed", "plain", "fused", "odd rows", "in place"])
def test_append(H, Hkv, hd, seqs, form):
    c = _Batch(seqs, H, Hkv, hd, page=64, spare_rows=2)
    r = _rng(5, H, hd)
    N, w, wq = c.N, Hkv * hd, H * hd
    q, k, v = (bf16(r.normal(0, 1.28, (N, h, hd))) for h in (H, Hkv, Hkv))
    n_pos = max(sum(s) for s in seqs) + 1
    cos, sin = _rope(hd, n_pos)
    slots = np.concatenate([np.arange(s[1] + s[2], sum(s)) for s in seqs])
    if form == "plain":
        kw, pos = {}, None
    else:
        kw = dict(cos=torch.from_numpy(cos).to(DEV), sin=torch.from_numpy(sin).to(DEV))
        pos = slots
        if form == "odd rows":
            pos = r.integers(0, n_pos, len(slots))
            kw["pos"] = _i32(np.concatenate([pos, [0, 0]]))
    qd, kd, vd = (_bf(x).reshape(N, -1) for x in (q, k, v))
    if form in ("fused", "odd rows"):
        pad = 8 if form == "fused" else 3
        rows = torch.zeros((N, wq + 2 * w + pad), dtype=torch.bfloat16, device=DEV)
        o = 0 if form == "fused" else 1
        qd, kd, vd = (rows[:, o + a : o + b].copy_(x) for a, b, x in ((0, wq, qd), (wq, wq + w, kd), (wq + w, wq + 2 * w, vd)))
    out = torch.full((N, H, hd), 7.0, dtype=torch.bfloat16, device=DEV)
    if form == "in place":
        out = qd.view(N, H, hd)
    if form != "plain" or H != 3:
        kw.update(q=qd, q_out=out)
    n = len(slots)
    before = c.pages.view(torch.int16).cpu().numpy().copy()
    cas.op_paged_append(c.cache(), kd, vd, **kw)
    rk, rq = (k[:n], q[:n]) if pos is None else (P.rotate(x[:n], cos, sin, pos) for x in (k, q))
    bk, bq = (np.zeros_like(y) if pos is None else P.rotate_bound(x[:n], y) for x, y in ((k, rk), (q, rq)))
    if "q" in kw:
        got = _np(out)
        assert (np.abs(got[:n] - rq) <= bq).all()
        assert np.array_equal(got[n:], q[n:]) if form == "in place" else (got[n:] == 7.0).all()
    got, touched = _np(c.pages), np.zeros(c.pool.shape, bool)
    kp, vp, at = P.key_places(hd), P.value_places(hd), 0
    for b, s in enumerate(seqs):
        for slot in range(s[1] + s[2], sum(s)) if s[0] else []:
            p, t = c.table[b, slot // 64], slot % 64 // 32 * 32 * hd
            assert (np.abs(got[p, 0][:, t + kp[slot % 32]] - rk[at]) <= bk[at]).all(), (b, slot)
            assert np.array_equal(got[p, 1][:, t + vp[slot % 32]], v[at]), (b, slot)
            touched[p, 0][:, t + kp[slot % 32]] = True
            touched[p, 1][:, t + vp[slot % 32]] = True
            at += 1
    after = c.pages.view(torch.int16).cpu().numpy()
    assert np.array_equal(after[~touched], before[~touched])


def test_append_refused_on_the_device():
    """Positions outside the table: NaN; pages outside the pool and sequences that do not fit: nothing is stored."""
    c = _Batch([(2, 30, 0), (1, 40, 0), (1, 5, 0)], 4, 2, 64)
    t = c.table.copy()
    t[1, 1] = -1
    c.device_table, c.ctx = _i32(t), _i32([30, 40, t.shape[1] * 32])
    cos, sin = _rope(64, 31)
    k = torch.ones((4, 128), dtype=torch.bfloat16, device=DEV)
    before = _np(c.pages)
    cas.op_paged_append(c.cache(), k, k, cos=torch.from_numpy(cos).to(DEV), sin=torch.from_numpy(sin).to(DEV))
    got = _np(c.pages)
    kp, vp = P.key_places(64), P.value_places(64)
    assert np.isfinite(got[t[0, 0], 0][:, kp[30]]).all() and np.isnan(got[t[0, 0], 0][:, kp[31]]).all()
    assert (got[t[0, 0], 1][:, vp[30:32]] == 1).all()
    got[t[0, 0], 0][:, kp[30:32]] = before[t[0, 0], 0][:, kp[30:32]]
    got[t[0, 0], 1][:, vp[30:32]] = before[t[0, 0], 1][:, vp[30:32]]
    assert np.array_equal(got, before, equal_nan=True)


# ---------------------------------------------------------------- together

def _step(c, rows, cos, sin, work, q, out):
    H, Hkv, hd = c.H, c.Hkv, c.hd
    cache = c.cache()
    k, v = rows[:, H * hd : (H + Hkv) * hd], rows[:, (H + Hkv) * hd :]
    cas.op_paged_append(cache, k, v, q=rows[:, : H * hd], q_out=q, cos=cos, sin=sin)
    cas.op_attention_paged(cache, q, out, work=work)


@pytest.mark.usefixtures("table")
@pytest.mark.parametrize("seqs", [[(1, 5000, 0), (1, 17, 0), (1, 62, 0)], [(90, 100, 0), (1, 2000, 0), (3, 0, 0)]])
def test_captured_step_replays_with_the_lengths_of_its_time(seqs):
    """Append and attention in one graph, replayed while the lengths grow and a
    page is taken; each replay against the eager calls on a copy."""
    H, Hkv, hd, N = 8, 2, 64, sum(s[0] for s in seqs)
    c, e = (_Batch(seqs, H, Hkv, hd, page=32, seed=4) for _ in "ce")
    wide = np.full((len(seqs), c.table.shape[1] + 3), -1, np.int32)
    wide[:, : c.table.shape[1]] = c.table
    c.pages, e.pages = (torch.cat([x.pages, torch.zeros_like(x.pages[: len(seqs)])]) for x in (c, e))
    c.device_table, e.device_table = _i32(wide), _i32(wide)
    cos, sin = (torch.from_numpy(x).to(DEV) for x in _rope(hd, 6000))
    rows = torch.zeros((N, (H + 2 * Hkv) * hd), dtype=torch.bfloat16, device=DEV)
    q, out, eq, eout = (torch.zeros((N, H, hd) if i % 2 == 0 else (N, H * hd), dtype=torch.bfloat16, device=DEV) for i in range(4))
    work = torch.empty(cas.paged_work_bytes(c.cache(), H), dtype=torch.uint8, device=DEV)
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        _step(c, rows, cos, sin, work, q, out)
    ctx = np.array([x[1] for x in seqs])
    for i in range(4):
        rows.copy_(torch.randn(rows.shape, generator=g, device="cuda"))
        for b, x in enumerate(seqs):  # the pages up to the step's last slot
            last = (int(ctx[b]) + x[0] - 1) // 32
            wide[b, last] = wide[b, last] if wide[b, last] >= 0 else c.pool.shape[0] + b
        for x in (c, e):
            x.device_table.copy_(_i32(wide))
            x.ctx.copy_(_i32(ctx))
        graph.replay()
        _step(e, rows, cos, sin, None, eq, eout)
        torch.cuda.synchronize()
        assert torch.equal(q, eq) and torch.equal(out, eout), i
        assert torch.equal(c.pages.view(torch.int16), e.pages.view(torch.int16))
        assert torch.isfinite(out).all()
        ctx += [x[0] if x[0] == 1 else 0 for x in seqs]  # (a chunk is written over its own slots)


def test_another_stream():
    c = _Batch([(1, 9000, 0), (1, 100, 0)], 8, 1, 128, page=64)
    want = c.run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = torch.zeros_like(want)
    cas.op_attention_paged(c.cache(), c.qd, got, stream=s.cuda_stream)
    s.synchronize()
    assert torch.equal(got, want)


def test_as_the_contiguous_attention():
    """One sequence's tree against the same call on a contiguous cache."""
    c = _Batch([(17, 500, 0)], 8, 2, 64, tree=True)
    k, v = (_bf(np.concatenate([x, np.zeros((2, 544 - 517, 64))], 1)) for x in c.kv[0])
    out = torch.zeros((17, 512), dtype=torch.bfloat16, device=DEV)
    cas.op_attention(c.qd, k, v, 544, 500, 17, 17, 8, 2, 64, c.anc, out)
    see = P.visible(17, 500, 0, c.masks[0], 0, 0)
    _, err = P.attention(c.q, *c.kv[0], see)
    assert (np.abs(_np(out) - _np(c.run())).reshape(err.shape) <= 2 * err).all()


def test_a_serving_step():
    """Three conversations through one layer: their prompts' chunks, then steps of a
    token each, chosen among the top alternatives.  Every call against its
    definition on what the calls before it left."""
    H, Hkv, hd, V, page = 8, 2, 64, 1000, 32
    d, w = H * hd, (H + 2 * Hkv) * hd
    g = torch.Generator(device="cuda")
    g.manual_seed(8)
    embed, wqkv, head = (torch.randn(s, generator=g, device="cuda") for s in ((V, d), (d, w), (d, V)))
    cos, sin = _rope(hd, 200)
    dcos, dsin = torch.from_numpy(cos).to(DEV), torch.from_numpy(sin).to(DEV)
    table = _rng(9).permutation(12).reshape(3, 4).astype(np.int32)
    pages = torch.full((12, 2, Hkv, page * hd), float("nan"), dtype=torch.bfloat16, device=DEV)
    texts = [list(_rng(9, b).integers(0, V, n)) for b, n in enumerate((37, 1, 64))]
    past = [0, 0, 0]
    kp, vp = P.key_places(hd), P.value_places(hd)
    for step in range(5):
        rows = [t[c:] for t, c in zip(texts, past)]
        n = [len(r) for r in rows]
        ids = np.concatenate(rows).astype(np.int64)
        x = (embed[torch.from_numpy(ids).to(DEV)] @ wqkv * d**-0.5).to(torch.bfloat16)
        start = np.concatenate([[0], np.cumsum(n)])
        cache = cas.Paged(pages, page, hd, _i32(table), _i32(start), _i32(past), len(ids), max(n))
        q = torch.empty((len(ids), H, hd), dtype=torch.bfloat16, device=DEV)
        o = torch.empty((len(ids), d), dtype=torch.bfloat16, device=DEV)
        cas.op_paged_append(cache, x[:, d : d + Hkv * hd], x[:, d + Hkv * hd :], q=x[:, :d], q_out=q, cos=dcos, sin=dsin)
        cas.op_attention_paged(cache, q, o)
        last = torch.from_numpy(start[1:] - 1).to(DEV)
        logits = o[last].float() @ head * (4 * d**-0.5)
        logp, entropy = torch.empty((3, 1), device=DEV), torch.empty(3, device=DEV)
        top, best = torch.empty((3, 5), dtype=torch.int32, device=DEV), torch.empty((3, 5), device=DEV)
        cas.op_logprobs(logits, _i32([[7], [8], [9]]), logp, entropy, top, best)
        got_q, got_o, pool, xs = _np(q), _np(o).reshape(-1, H, hd), _np(pages), _np(x)
        for b in range(3):
            r, slots = slice(start[b], start[b + 1]), np.arange(past[b], past[b] + n[b])
            for new, h0, h1, got in ((got_q[r], 0, H, None), (None, H, H + Hkv, "k")):
                raw = xs[r].reshape(n[b], -1, hd)[:, h0:h1]
                ref = P.rotate(raw, cos, sin, slots)
                if got:
                    new = np.stack([pool[table[b, s // page], 0][:, kp[s % 32]] for s in slots])
                assert (np.abs(new - ref) <= P.rotate_bound(raw, ref)).all(), (step, b)
            every = np.arange(past[b] + n[b])
            k = np.stack([pool[table[b, s // page], 0][:, kp[s % 32]] for s in every], 1)
            v = np.stack([pool[table[b, s // page], 1][:, vp[s % 32]] for s in every], 1)
            assert np.array_equal(v[:, slots].transpose(1, 0, 2), xs[r].reshape(n[b], -1, hd)[:, H + Hkv :])
            ref, err = P.attention(got_q[r], k, v, P.visible(n[b], past[b], 0, None, 0, 0))
            assert (np.abs(got_o[r] - ref) <= err).all(), (step, b)
        y = _np(logits)
        lp = y - y.max(1, keepdims=True)
        lp -= np.log(np.exp(lp).sum(1, keepdims=True))
        assert np.array_equal(top.cpu().numpy(), np.argsort(-y, axis=1, kind="stable")[:, :5])
        assert np.abs(_np(best) - np.take_along_axis(lp, top.cpu().numpy().astype(np.int64), 1)).max() < 1e-5
        assert np.abs(_np(logp)[:, 0] - lp[[0, 1, 2], [7, 8, 9]]).max() < 1e-5
        past = [len(t) for t in texts]
        texts = [t + [int(top[b, step])] for b, t in enumerate(texts)]

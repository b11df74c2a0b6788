"""The 4-bit KV cache on the GPU against its definition in 64 bits: append and
read exact, attention within the bound that tests/kv4_ref.py derives."""
import numpy as np
import pytest
import torch

from paper_2510_26843_amd import cas
from tests import kv4_ref as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _rng(*what):
    return np.random.default_rng([11, *what])


def _dev_bf16(x):
    return torch.from_numpy(np.asarray(x, dtype=np.float32)).to(torch.bfloat16).to(DEV)


def _rope(hd, n, theta=1e4):
    a = np.arange(n)[:, None] * theta ** (-2.0 * np.arange(hd // 2) / hd)
    return np.cos(a).astype(np.float32), np.sin(a).astype(np.float32)


def _read(rec, cap, slot0, n, Hkv, hd):
    k = torch.full((Hkv, n, hd), 7.0, dtype=torch.bfloat16, device=DEV)
    v = torch.full_like(k, 7.0)
    cas.op_kv4_read(rec, cap, slot0, n, Hkv, hd, k, v)
    return k.double().cpu().numpy(), v.double().cpu().numpy()


def _same(got, want):
    return np.array_equal(got, want, equal_nan=True)


# ---------------------------------------------------------------- append, read

@pytest.mark.parametrize("Hkv,hd,T,slot0", [
    (1, 128, 1, 0), (8, 128, 1, 31), (8, 128, 1, 32), (2, 64, 1, 95), (3, 64, 33, 31), (5, 128, 32, 32),
    (2, 64, 64, 0), (4, 128, 61, 2047), (40, 128, 2, 63), (2, 64, 1000, 17), (1, 128, 2049, 0), (7, 64, 31, 1)])
@pytest.mark.parametrize("form", ["plain", "rotated", "tree positions in wider rows", "odd rows"])
def test_append_and_read(Hkv, hd, T, slot0, form):
    r = _rng(Hkv, hd, T, slot0)
    k, v = (R.bf16(r.normal(0, 1.28, (T, Hkv, hd)) * np.exp2(r.integers(-9, 9, (T, 1, 1)))) for _ in "kv")
    cap = (slot0 + T + 31) // 32 * 32 + 32
    before = r.integers(0, 256, (Hkv, cap // 32, 34 * hd), dtype=np.uint8)
    rec = torch.from_numpy(before).to(DEV)
    kd, vd = _dev_bf16(k).reshape(T, -1), _dev_bf16(v).reshape(T, -1)
    kw, want_k = {}, k
    if form != "plain":
        n_pos = slot0 + T
        cos, sin = _rope(hd, n_pos)
        pos = slot0 + np.arange(T)
        if form != "rotated":
            pos = r.integers(0, n_pos, T)
            kw["pos"] = torch.from_numpy(pos.astype(np.int32)).to(DEV)
        kw.update(cos=torch.from_numpy(cos).to(DEV), sin=torch.from_numpy(sin).to(DEV))
        want_k = R.rotate(k, cos, sin, pos)
    if form in ("tree positions in wider rows", "odd rows"):
        w = Hkv * hd
        first, ld = (64, 3 * w + 64) if form != "odd rows" else (1, 2 * w + 3)  # 2-byte aligned rows
        rows = torch.zeros((T, ld), dtype=torch.bfloat16, device=DEV)
        rows[:, first : first + w], rows[:, first + w : first + 2 * w] = kd, vd
        kd, vd = rows[:, first : first + w], rows[:, first + w : first + 2 * w]
        kw.update(ldk=ld, ldv=ld)
    cas.op_kv4_append(kd, vd, T, Hkv, hd, rec, cap, slot0, **kw)
    k4, v4 = R.quantise(want_k.transpose(1, 0, 2)), R.quantise(v.transpose(1, 0, 2))
    got_k, got_v = _read(rec, cap, slot0, T, Hkv, hd)
    assert _same(got_k, R.values(*k4)) and _same(got_v, R.values(*v4))
    # the bytes of these slots as documented, those of the others as they were:
    # the slots before are put back over the expected records
    pad = lambda x, fill: np.concatenate([np.full((Hkv, slot0, x.shape[-1]), fill, np.uint8), x], 1)  # noqa: E731
    want = R.pack((pad(k4[0], 0), pad(k4[1], 0)), (pad(v4[0], 0), pad(v4[1], 0)), cap, before)
    if slot0:
        pk, _, pv, _, pks, pvs = R._places(hd)
        for t in range((slot0 + 31) // 32):
            m = min(32, slot0 - 32 * t)
            for p in (pk, pv, pks, pvs):
                want[:, t, p[:m].ravel()] = before[:, t, p[:m].ravel()]
    assert np.array_equal(rec.cpu().numpy(), want)


def test_special_values():
    hd, T = 128, 9
    k = np.zeros((T, 1, hd))
    k[1, 0, :32] = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0] * 4) * np.tile([1, -1], 16)  # ties, at scale 1
    k[1, 0, 0] = 4.0
    k[2, 0, :] = R.bf16(np.full(hd, 7.96875))  # saturates at 6
    k[2, 0, 32:64] = -0.0
    k[3, 0, 5] = np.nan
    k[4, 0, 40] = np.inf
    k[4, 0, 90] = -np.inf
    k[5, 0, :] = R.bf16(np.full(hd, 3.38e38)) * np.tile([1, -1], 64)
    k[6, 0, :] = 2.0**-126 * np.tile([1, -1, 0, 1], 32)  # the smallest scale
    k[7, 0, :] = 2.0**-133  # subnormal: below the smallest step
    k[8, 0, :] = R.bf16(np.random.default_rng(0).normal(0, 1e30, hd))
    v = k[::-1].copy()
    rec = torch.zeros((1, 1, 34 * hd), dtype=torch.uint8, device=DEV)
    cas.op_kv4_append(_dev_bf16(k).reshape(T, -1), _dev_bf16(v).reshape(T, -1), T, 1, hd, rec, 32, 3)
    got_k, got_v = _read(rec, 32, 3, T, 1, hd)
    assert _same(got_k[0], R.values(*R.quantise(k[:, 0]))) and _same(got_v[0], R.values(*R.quantise(v[:, 0])))
    assert np.isnan(got_k[0, 3, :32]).all() and np.isfinite(got_k[0, 3, 32:]).all()


def test_positions_outside_the_table_read_as_nan():
    hd, T = 64, 3
    cos, sin = _rope(hd, 10)
    k = R.bf16(_rng(5).normal(0, 1, (T, 2, hd)))
    rec = torch.zeros((2, 1, 34 * hd), dtype=torch.uint8, device=DEV)
    pos = np.array([9, 10, -1])
    cas.op_kv4_append(_dev_bf16(k).reshape(T, -1), _dev_bf16(k).reshape(T, -1), T, 2, hd, rec, 32, 0,
                      pos=torch.from_numpy(pos.astype(np.int32)).to(DEV), cos=torch.from_numpy(cos).to(DEV),
                      sin=torch.from_numpy(sin).to(DEV))
    got, gv = _read(rec, 32, 0, T, 2, hd)
    assert _same(got, R.values(*R.quantise(R.rotate(k, cos, sin, pos).transpose(1, 0, 2))))
    assert np.isnan(got[:, 1:]).all() and np.isfinite(gv).all()


# ---------------------------------------------------------------- attention

def _masks(T, n_tree, r):
    parent = [-1] + [int(r.integers(max(0, i - 6), i)) for i in range(1, n_tree)]
    m = []
    for i, p in enumerate(parent):
        m.append((m[p] if p >= 0 else 0) | 1 << i)
    return m[n_tree - T :] if T <= n_tree else [m[int(r.integers(n_tree))] for _ in range(T)]


def _words(masks):
    return torch.from_numpy(np.array([[m & (2**64 - 1), m >> 64] for m in masks], np.uint64).view(np.int64)).to(DEV)


class _Case:
    """Inputs of one attention call; where `junk`, everything that no row sees
    (unused slots, masked nodes, slots outside the window) holds NaN."""

    def __init__(self, H, Hkv, hd, T, n_tree, Lc, n4, sink=0, window=0, junk=True, masks=None, seed=0, std=1.28):
        r = _rng(H, Hkv, hd, T, n_tree, Lc, seed)
        self.H, self.Hkv, self.hd, self.T, self.n_tree, self.Lc = H, Hkv, hd, T, n_tree, Lc
        n = Lc + n_tree
        self.n4 = n if n4 is None else n4
        self.sink, self.window = sink, window
        self.masks = _masks(T, n_tree, r) if masks is None else masks
        self.q = R.bf16(r.normal(0, 1, (T, H, hd)))
        self.cap = (self.n4 + 31) // 32 * 32 + 32
        kv = [R.bf16(r.normal(0, std, (Hkv, n, hd))) for _ in "kv"]
        self.see = R.visible(T, n_tree, Lc, self.masks, sink, window)
        hidden = ~self.see.any(0)
        x4 = [R.quantise(x[:, : self.n4]) for x in kv]
        self.k, self.v = (np.concatenate([R.values(*a), x[:, self.n4 :]], 1) for a, x in zip(x4, kv))
        fill = r.integers(0, 256, (Hkv, self.cap // 32, 34 * hd), dtype=np.uint8) if junk else None
        if junk:
            fill[..., 32 * hd :] = 255
            for a in x4:
                a[1][:, hidden[: self.n4]] = 255
            for x in kv:
                x[:, hidden] = np.nan
        self.rec = torch.from_numpy(R.pack(x4[0], x4[1], self.cap, fill)).to(DEV)
        self.kr = self.vr = None
        if self.n4 < n:
            extra = np.full((Hkv, 3, hd), np.nan if junk else 0.0)
            self.kr, self.vr = (_dev_bf16(np.concatenate([x[:, self.n4 :], extra], 1)) for x in kv)
        self.qd, self.anc = _dev_bf16(self.q), _words(self.masks)

    def run(self, out=None, **kw):
        out = torch.full((self.T, self.H * self.hd), 7.0, dtype=torch.bfloat16, device=DEV) if out is None else out
        cas.op_attention_kv4(self.qd, self.rec, self.cap, self.n4, self.Lc, self.n_tree, self.T, self.H, self.Hkv,
                             self.hd, self.anc, out, k=self.kr, v=self.vr, sink=self.sink, window=self.window, **kw)
        return out

    def check(self, out):
        k, v = (np.where(np.isnan(x) & ~self.see.any(0)[None, :, None], 0.0, x) for x in (self.k, self.v))
        ref, size, mass = R.attention(self.q, k, v, self.see)
        got = out.double().cpu().numpy()
        over = np.abs(got - ref) / R.bound(ref, size, mass, self.hd, self.Lc + self.n_tree)
        assert np.isfinite(got).all() and over.max() <= 1, (np.isfinite(got).all(), over.max())


HEADS = [(8, 2, 64), (4, 4, 128), (8, 1, 128), (6, 2, 64), (5, 5, 64)]


@pytest.mark.parametrize("H,Hkv,hd", HEADS)
@pytest.mark.parametrize("T,n_tree,Lc,n4", [
    (1, 1, 0, None), (1, 1, 0, 0), (1, 1, 31, None), (1, 1, 31, 0), (1, 1, 32, 32), (1, 1, 255, None),
    (2, 5, 63, 32), (3, 3, 64, 64), (16, 16, 100, None), (17, 40, 97, 96), (7, 128, 513, 512), (32, 32, 1023, None),
    (61, 61, 700, 672), (128, 128, 33, None), (128, 128, 300, 288), (5, 3, 20, None), (1, 1, 4097, None)])
def test_attention(H, Hkv, hd, T, n_tree, Lc, n4):
    c = _Case(H, Hkv, hd, T, n_tree, Lc, n4)
    c.check(c.run())


@pytest.mark.parametrize("H,Hkv,hd", HEADS[:2])
@pytest.mark.parametrize("T,n_tree,Lc,n4,sink,window", [
    (1, 1, 500, None, 4, 64), (3, 12, 500, 480, 4, 64), (3, 12, 500, 480, 0, 1), (20, 20, 500, 480, 100, 33),
    (2, 2, 40, 32, 4, 64), (2, 2, 40, None, 33, 3), (9, 9, 2000, 1984, 4, 1024), (1, 4, 300, 0, 2, 31),
    (4, 4, 300, 96, 40, 100)])
def test_attention_window(H, Hkv, hd, T, n_tree, Lc, n4, sink, window):
    c = _Case(H, Hkv, hd, T, n_tree, Lc, n4, sink, window)
    c.check(c.run())


@pytest.mark.parametrize("std", [1e-20, 0.02, 30.0])
def test_attention_ranges(std):
    """Scores near 0 (all keys alike) and in the hundreds (one key takes all)."""
    c = _Case(8, 2, 64, 9, 9, 200, 192, std=std)
    c.check(c.run())


def test_a_row_that_sees_nothing_gives_zeros():
    for n4 in (None, 0):
        c = _Case(4, 2, 64, 3, 3, 0, n4, masks=[1, 0, 5])
        out = c.run()
        assert (out[1] == 0).all()
        c.check(out)


@pytest.mark.parametrize("n4", [None, 96])
def test_values_that_are_not_finite_reach_their_rows_only(n4):
    """A node's key (value) with a NaN: NaN rows (elements) where it is seen, nothing else."""
    clean = _Case(4, 2, 64, 6, 6, 100, n4, masks=[1, 3, 5, 11, 21, 37], junk=False)
    want = clean.run().double().cpu().numpy().reshape(6, 4, 64)
    for what in "kv":
        c = _Case(4, 2, 64, 6, 6, 100, n4, masks=[1, 3, 5, 11, 21, 37], junk=False)
        node = 100 + 1  # seen by the rows of masks 3 and 11
        sees = np.array([0, 1, 0, 1, 0, 0], bool)
        if n4 is None:
            pk, _, pv, _, pks, pvs = R._places(64)
            b = c.rec.cpu().numpy()
            b[1, node // 32, (pks if what == "k" else pvs)[node % 32, 1]] = 255  # elements 32 .. 63 of kv head 1
            c.rec = torch.from_numpy(b).to(DEV)
        else:
            (c.kr if what == "k" else c.vr)[1, node - n4, 32:] = float("nan")
        got = c.run().double().cpu().numpy().reshape(6, 4, 64)
        bad = np.zeros((6, 4, 64), bool)
        bad[np.ix_(sees, [2, 3], np.arange(64) if what == "k" else np.arange(32, 64))] = True
        assert np.array_equal(np.isnan(got), bad)
        assert np.array_equal(got[~bad], want[~bad])


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_a_query_that_is_not_finite_spoils_its_row_only(value):
    c = _Case(4, 2, 64, 3, 3, 200, 192, junk=False)
    want = c.run().double().cpu().numpy().reshape(3, 4, 64)
    c.qd[1, 2, 17] = value
    got = c.run().double().cpu().numpy().reshape(3, 4, 64)
    assert np.isnan(got[1, 2]).all()
    got[1, 2] = want[1, 2]
    assert np.array_equal(got, want)


def test_query_ranges():
    """Queries whose elements differ by many binades, tiny and large ones: the
    scores stay those of bf16 queries."""
    r = _rng(3)
    for scale in (2.0**-60, 2.0**-8, 1.0):
        c = _Case(4, 2, 128, 5, 5, 300, 288)
        c.q = R.bf16(r.normal(0, 1, c.q.shape) * np.exp2(r.integers(-12, 3, c.q.shape)) * scale)
        c.qd = _dev_bf16(c.q)
        c.check(c.run())


def test_many_query_heads_of_one_kv_head():
    c = _Case(96, 1, 64, 2, 2, 77, None)
    c.check(c.run())


@pytest.mark.parametrize("H,Hkv,hd", HEADS[:3])
@pytest.mark.parametrize("T,n_tree,Lc,n4", [(128, 128, 33, 96), (40, 100, 20, 64), (3, 40, 0, 32), (9, 70, 60, 128)])
def test_some_of_the_rounds_nodes_in_4_bits(H, Hkv, hd, T, n_tree, Lc, n4):
    c = _Case(H, Hkv, hd, T, n_tree, Lc, n4)
    c.check(c.run())


@pytest.mark.parametrize("H,Hkv,hd,T", [(33, 1, 128, 128), (64, 1, 64, 128), (41, 1, 64, 100), (80, 2, 128, 61)])
@pytest.mark.parametrize("Lc,n4,sink,window", [(700, None, 0, 0), (700, 672, 0, 0), (333, 0, 0, 0), (30, None, 0, 0),
                                               (900, 896, 40, 300)])
def test_more_query_tiles_than_the_card_has_places(H, Hkv, hd, T, Lc, n4, sink, window):
    """Over 256 tiles of 16 query rows: workgroups of two (in the third shape
    an odd number of them)."""
    c = _Case(H, Hkv, hd, T, T, Lc, n4, sink, window)
    c.check(c.run())


@pytest.mark.parametrize("H,Hkv,hd,T", [(8, 1, 128, 1), (4, 2, 64, 3)])
def test_many_splits(H, Hkv, hd, T):
    c = _Case(H, Hkv, hd, T, T, 40001, None)
    assert cas.lib().cas_op_attention_kv4_work_bytes(40001, T, T, H, Hkv, hd, 0, 0) > 32 * H * T * (hd + 2) * 4
    c.check(c.run())


def test_calls_with_a_tensor_of_the_host_are_refused():
    c = _Case(4, 2, 64, 3, 3, 100, 96)
    for name in ("qd", "rec", "kr", "vr", "anc"):
        x = getattr(c, name)
        setattr(c, name, x.cpu())
        with pytest.raises(cas.CasError, match="not on the current device"):
            c.run()
        setattr(c, name, x)
    with pytest.raises(cas.CasError, match="not on the current device"):
        c.run(work=torch.empty(64, dtype=torch.uint8))
    rows = torch.zeros((2, 128), dtype=torch.bfloat16, device=DEV)
    cos, sin = (torch.from_numpy(x).to(DEV) for x in _rope(64, 40))
    pos = torch.zeros(2, dtype=torch.int32, device=DEV)
    good = [rows, rows, c.rec, pos, cos, sin]
    for i in range(6):
        a = list(good)
        a[i] = a[i].cpu()
        with pytest.raises(cas.CasError, match="not on the current device"):
            cas.op_kv4_append(a[0], a[1], 2, 2, 64, a[2], c.cap, 0, pos=a[3], cos=a[4], sin=a[5])
    out = torch.zeros((2, 2, 64), dtype=torch.bfloat16, device=DEV)
    for a in ([c.rec.cpu(), out, out], [c.rec, out.cpu(), out], [c.rec, out, out.cpu()]):
        with pytest.raises(cas.CasError, match="not on the current device"):
            cas.op_kv4_read(a[0], c.cap, 0, 2, 2, 64, a[1], a[2])
    c.check(c.run())


def test_same_bits_again_and_on_another_stream():
    c = _Case(8, 2, 128, 5, 20, 3000, 2976)
    a = c.run()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = c.run()
    s.synchronize()
    assert torch.equal(a, b) and torch.equal(a, c.run())


@pytest.mark.parametrize("split", [3, 13, 16, 30])
def test_two_streams_append_to_the_same_records(split):
    """No byte belongs to two slots: appends to different slots need no order."""
    Hkv, hd, n = 8, 128, 64
    r = _rng(split)
    k, v = (R.bf16(r.normal(0, 1.28, (n, Hkv, hd))) for _ in "kv")
    kd, vd = (_dev_bf16(x).reshape(n, -1) for x in (k, v))
    rec = torch.zeros((Hkv, 2, 34 * hd), dtype=torch.uint8, device=DEV)
    streams = [torch.cuda.Stream() for _ in range(3)]
    cuts = [0, split, 32 + split, n]
    torch.cuda.synchronize()
    for s, a, b in zip(streams, cuts, cuts[1:]):
        cas.op_kv4_append(kd[a:b], vd[a:b], b - a, Hkv, hd, rec, 64, a, stream=s.cuda_stream)
    torch.cuda.synchronize()
    got_k, got_v = _read(rec, 64, 0, n, Hkv, hd)
    assert _same(got_k, R.values(*R.quantise(k.transpose(1, 0, 2))))
    assert _same(got_v, R.values(*R.quantise(v.transpose(1, 0, 2))))


def test_captured_and_replayed():
    """Append and attention in one graph, replayed over changed inputs."""
    c = _Case(8, 2, 64, 4, 4, 131, None)
    work = torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    rows = [torch.zeros((4, 2 * 64), dtype=torch.bfloat16, device=DEV) for _ in "kv"]
    out = torch.zeros((4, 8 * 64), dtype=torch.bfloat16, device=DEV)

    def step(to):
        cas.op_kv4_append(rows[0], rows[1], 4, 2, 64, c.rec, c.cap, 131)
        c.run(out=to, work=work)

    for x in rows:
        x.normal_()
    step(out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(out)
    for i in range(3):
        for x in rows:
            x.normal_()
        want = torch.empty_like(out)
        step(want)
        torch.cuda.synchronize()
        out.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), i


def test_offsets_past_32_bits():
    """The last head of a cache of more than 4 GB, at its last slots."""
    Hkv, hd, cap = 32, 128, 1 << 20
    nbytes = cas.kv4_bytes(Hkv, hd, cap)
    assert nbytes > 1 << 32
    rec = torch.empty(nbytes, dtype=torch.uint8, device=DEV)
    rec.zero_()
    r = _rng(77)
    n, Lc = 40, cap - 40
    k, v = (R.bf16(r.normal(0, 1.28, (n, Hkv, hd))) for _ in "kv")
    cas.op_kv4_append(_dev_bf16(k).reshape(n, -1), _dev_bf16(v).reshape(n, -1), n, Hkv, hd, rec, cap, Lc)
    k4, v4 = (R.values(*R.quantise(x.transpose(1, 0, 2))) for x in (k, v))
    got_k, got_v = _read(rec, cap, Lc, n, Hkv, hd)
    assert _same(got_k, k4) and _same(got_v, v4)
    q = R.bf16(r.normal(0, 1, (1, Hkv, hd)))
    out = torch.zeros((1, Hkv * hd), dtype=torch.bfloat16, device=DEV)
    cas.op_attention_kv4(_dev_bf16(q), rec, cap, cap, cap - 1, 1, 1, Hkv, Hkv, hd, _words([1]), out, window=39)
    ref, size, mass = R.attention(q, k4, v4, np.ones((1, n), bool))
    over = np.abs(out.double().cpu().numpy() - ref) / R.bound(ref, size, mass, hd, n)
    assert over.max() <= 1


def test_prompt_then_decoding():
    """As a program uses them: the prompt's rows appended and attended as a
    chain, then token after token, every step over the whole 4-bit cache."""
    H, Hkv, hd, n = 8, 2, 128, 70
    r = _rng(9)
    cos, sin = _rope(hd, 128)
    cd, sd = torch.from_numpy(cos).to(DEV), torch.from_numpy(sin).to(DEV)
    k, v = (R.bf16(r.normal(0, 1.28, (n + 5, Hkv, hd))) for _ in "kv")
    q = R.bf16(r.normal(0, 1, (n + 5, H, hd)))
    kd, vd, qd = _dev_bf16(k), _dev_bf16(v), _dev_bf16(q)
    rec = torch.zeros((Hkv, 4, 34 * hd), dtype=torch.uint8, device=DEV)
    k4 = R.values(*R.quantise(R.rotate(k, cos, sin, np.arange(n + 5)).transpose(1, 0, 2)))
    v4 = R.values(*R.quantise(v.transpose(1, 0, 2)))
    for t0, t1 in [(0, n)] + [(i, i + 1) for i in range(n, n + 5)]:
        T = t1 - t0
        cas.op_kv4_append(kd[t0:t1], vd[t0:t1], T, Hkv, hd, rec, 128, t0, cos=cd, sin=sd)
        out = torch.zeros((T, H * hd), dtype=torch.bfloat16, device=DEV)
        cas.op_attention_kv4(qd[t0:t1], rec, 128, t1, t0, T, T, H, Hkv, hd, _words([2 ** (i + 1) - 1 for i in range(T)]),
                             out)
        see = np.tril(np.ones((t1, t1), bool))[t0:t1]
        ref, size, mass = R.attention(q[t0:t1], k4[:, :t1], v4[:, :t1], see)
        over = np.abs(out.double().cpu().numpy() - ref) / R.bound(ref, size, mass, hd, t1)
        assert over.max() <= 1, (t0, over.max())

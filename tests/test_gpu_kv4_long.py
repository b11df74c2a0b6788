"""Attention over the 4-bit KV cache where a call's key tiles are split over
workgroups and a wave takes many of them, against its 64-bit form on the GPU
(the bound of tests/kv4_ref.py), and what a row's result may depend on."""
import math

import numpy as np
import pytest
import torch

from paper_2510_26843_amd import cas
from tests import kv4_ref as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _masks(n_tree, seed):
    r = np.random.default_rng([5, n_tree, seed])
    m = []
    for i in range(n_tree):
        m.append((m[int(r.integers(max(0, i - 6), i))] if i else 0) | 1 << i)
    return m


def _words(masks):
    return torch.from_numpy(np.array([[m & (2**64 - 1), m >> 64] for m in masks], np.uint64).view(np.int64)).to(DEV)


class _Call:
    """One attention call over slots that the append wrote; tail: the slots
    from the last whole committed record on are bf16 rows."""

    def __init__(self, H, Hkv, hd, T, Lc, tail=False, sink=0, window=0, seed=0, cap=None):
        g = torch.Generator(device=DEV)
        g.manual_seed(1000 * seed + Lc)
        normal = lambda *s, std=1.28: (torch.randn(s, generator=g, device=DEV) * std).to(torch.bfloat16)  # noqa: E731
        self.H, self.Hkv, self.hd, self.T, self.Lc, self.sink, self.window = H, Hkv, hd, T, Lc, sink, window
        n = Lc + T
        self.n4 = Lc // 32 * 32 if tail else n
        self.cap = (self.n4 + 31) // 32 * 32 if cap is None else cap
        k, v = normal(n, Hkv, hd), normal(n, Hkv, hd)
        self.rec = torch.zeros((Hkv, self.cap // 32, 34 * hd), dtype=torch.uint8, device=DEV)
        cas.op_kv4_append(k[: self.n4].reshape(self.n4, -1), v[: self.n4].reshape(self.n4, -1), self.n4, Hkv, hd,
                          self.rec, self.cap, 0)
        held = torch.empty((2, Hkv, self.n4, hd), dtype=torch.bfloat16, device=DEV)
        cas.op_kv4_read(self.rec, self.cap, 0, self.n4, Hkv, hd, held[0], held[1])
        self.kr = self.vr = None
        rest = [x[self.n4 :].transpose(0, 1).contiguous() for x in (k, v)]
        if tail:
            self.kr, self.vr = rest
        self.k, self.v = (torch.cat((a.double(), b.double()), 1) for a, b in zip(held, rest))
        self.q = normal(T, H, hd, std=1.0)
        self.masks = _masks(T, seed)

    def splits(self):
        """The runs of key tiles that the call is split into."""
        b = cas.lib().cas_op_attention_kv4_work_bytes(self.Lc, self.T, self.T, self.H, self.Hkv, self.hd, self.sink,
                                                      self.window)
        return max(1, b // (4 * self.T * self.H * (self.hd + 2)))

    def run(self, **kw):
        out = torch.full((self.T, self.H * self.hd), 7.0, dtype=torch.bfloat16, device=DEV)
        cas.op_attention_kv4(self.q, self.rec, self.cap, self.n4, self.Lc, self.T, self.T, self.H, self.Hkv, self.hd,
                             _words(self.masks), out, k=self.kr, v=self.vr, sink=self.sink, window=self.window, **kw)
        return out

    def check(self, out):
        T, H, hd, n = self.T, self.H, self.hd, self.Lc + self.T
        see = torch.from_numpy(R.visible(T, T, self.Lc, self.masks, self.sink, self.window)).to(DEV)
        ref, size = (torch.empty((T, H, hd), dtype=torch.float64, device=DEV) for _ in range(2))
        mass = torch.empty((T, H), dtype=torch.float64, device=DEV)
        for h in range(H):
            k, v = self.k[h // (H // self.Hkv)], self.v[h // (H // self.Hkv)]
            q, kt = self.q[:, h].double(), k.t().contiguous()
            x = (q @ kt / math.sqrt(hd)).masked_fill(~see, -math.inf)
            p = torch.exp(x - x.amax(1, keepdim=True))
            p /= p.sum(1, keepdim=True)
            ref[:, h], size[:, h] = p @ v, p @ v.abs()
            mass[:, h] = (q.abs() @ kt.abs() / math.sqrt(hd)).masked_fill(~see, 0.0).amax(1)
        ref, size, mass = ref.reshape(T, -1).cpu().numpy(), size.reshape(T, -1).cpu().numpy(), mass.cpu().numpy()
        got = out.double().cpu().numpy()
        over = np.abs(got - ref) / R.bound(ref, size, mass, hd, n)
        assert np.isfinite(got).all() and over.max() <= 1, over.max()


@pytest.mark.parametrize("H,Hkv,hd,T,Lc", [(16, 16, 64, 128, 4000), (33, 1, 128, 128, 3000), (8, 8, 128, 17, 9000)])
def test_a_row_does_not_depend_on_the_queries_beside_it(H, Hkv, hd, T, Lc):
    """Every second row's queries and mask changed: the others keep their bits
    (the running maximum of a row follows its own scores only)."""
    c = _Call(H, Hkv, hd, T, Lc)
    want = c.run()
    c.check(want)
    for scale in (0.0, 12.0):
        q, masks = c.q.clone(), list(c.masks)
        q[1::2] = q[1::2].flip(0) * scale
        masks[1::2] = [1] * len(masks[1::2])
        other = _Call(H, Hkv, hd, T, Lc)
        other.q, other.masks = q, masks
        got = other.run()
        assert torch.equal(got[0::2], want[0::2]), (scale, int((got[0::2] != want[0::2]).sum()))
        assert not torch.equal(got[1::2], want[1::2])


def test_views_of_wider_rows_and_longer_caches():
    """Tensors passed as views give the bits of their packed copies: rows of a
    fused product without ldk and ldv, the last slots of a bf16 cache without
    kv_cap."""
    c = _Call(8, 2, 64, 5, 200, tail=True)
    want = c.run()
    c.check(want)
    long = torch.full((2, 2, 300, 64), float("nan"), dtype=torch.bfloat16, device=DEV)
    long[0, :, c.n4 : c.n4 + 13], long[1, :, c.n4 : c.n4 + 13] = c.kr, c.vr
    c.kr, c.vr = long[0, :, c.n4 : c.n4 + 13], long[1, :, c.n4 : c.n4 + 13]
    assert torch.equal(c.run(), want)
    rows = torch.randn((7, 3 * 128), device=DEV).to(torch.bfloat16)
    k, v = rows[:, 128:256], rows[:, 256:]
    recs = [torch.zeros((2, 1, 34 * 64), dtype=torch.uint8, device=DEV) for _ in range(2)]
    cas.op_kv4_append(k, v, 7, 2, 64, recs[0], 32, 5)
    cas.op_kv4_append(k.contiguous(), v.contiguous(), 7, 2, 64, recs[1], 32, 5)
    assert torch.equal(*recs) and bool(recs[0].any())


# (splits: the runs of key tiles that the plan gives each, which work_bytes
# tells; the first two and the last are 128 or 256 tiles of query rows, whose
# splits fill the card's 256 places with two tiles per workgroup)
@pytest.mark.parametrize("H,Hkv,hd,T,Lc,sink,window,splits", [
    (16, 4, 128, 128, 7000, 0, 0, 4), (32, 8, 128, 128, 16001, 0, 0, 2),
    (8, 8, 128, 128, 8190, 0, 0, 4), (8, 8, 128, 64, 8190, 0, 0, 7), (4, 2, 64, 128, 8190, 0, 0, 7),
    (32, 32, 128, 32, 8190, 0, 0, 4), (8, 2, 64, 20, 6000, 0, 0, 12), (4, 4, 128, 1, 8190, 0, 0, 32),
    (8, 2, 64, 3, 9000, 40, 3000, 16), (4, 4, 128, 20, 9000, 40, 3000, 16), (8, 2, 64, 1, 9000, 4, 5000, 20),
    (16, 4, 128, 128, 9000, 100, 7000, 4)])
@pytest.mark.parametrize("tail", [False, True], ids=["4-bit", "bf16 tail"])
def test_splits(H, Hkv, hd, T, Lc, tail, sink, window, splits):
    c = _Call(H, Hkv, hd, T, Lc, tail, sink, window)
    assert c.splits() == splits
    c.check(c.run())


@pytest.mark.parametrize("H,Hkv,hd", [(8, 2, 64), (4, 4, 128)])
@pytest.mark.parametrize("T,Lc", [(1, 0), (1, 30), (1, 31), (9, 11), (32, 0)])
def test_a_cache_of_one_record(H, Hkv, hd, T, Lc):
    c = _Call(H, Hkv, hd, T, Lc, cap=32)
    c.check(c.run())

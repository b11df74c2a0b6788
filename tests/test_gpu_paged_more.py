"""More of the paged KV cache on the GPU: groups of more heads than an append holds at
a time, more sequences than lanes, pools past 4 GiB, and every tile of a split
sequence weighed once."""
import numpy as np
import pytest
import torch

from paper_2510_26843_amd import cas
from tests import paged_ref as P
from tests.test_gpu_paged import _bf, _Batch, _i32, _np, _rng, _rope, table  # noqa: F401 (a fixture)
from tests.test_gpu_paged import test_append as _append_case

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("H,Hkv,hd", [(10, 2, 128), (8, 1, 64), (18, 2, 64)])
@pytest.mark.parametrize("seqs", [[(33, 31, 0), (100, 0, 0), (3, 6, 4)], [(300, 17, 0)], [(32, 32, 0), (64, 64, 0)]])
@pytest.mark.parametrize("form", ["packed", "plain", "in place"])
def test_append_of_more_than_four_heads_to_a_group(H, Hkv, hd, seqs, form):
    _append_case(H, Hkv, hd, seqs, form)


@pytest.mark.parametrize("form", ["fused", "in place"])
def test_append_of_many_sequences(form):
    """Idle ones where a wave's turn ends, whole tiles behind the first 64."""
    r = _rng(78)
    seqs = [(int(r.integers(0, 4)), int(r.integers(0, 90)), int(r.integers(0, 3))) for _ in range(200)]
    for b in (0, 63, 64, 127, 128, 199):
        seqs[b] = (0,) + seqs[b][1:]
    seqs[70], seqs[129], seqs[191], seqs[192] = (75, 10, 0), (32, 64, 0), (1, 31, 0), (40, 0, 0)
    _append_case(8, 1, 64, seqs, form)


@pytest.mark.parametrize("seqs", [[(1, 700, 0), (3, 65, 0)], [(20, 600, 0)], [(200, 500, 0), (1, 5000, 0)]])
def test_pools_past_4_gib(seqs):
    """Pages at both ends of a pool of 5 GiB: the bits of a small pool's."""
    c = _Batch(seqs, 8, 8, 128, page=128, seed=3)
    n = c.pool.shape[0]
    most = 5 * 2**30 // (c.pages[0].numel() * 2)
    place = np.array([most - 1 - i if i % 3 else i for i in range(n)])
    pages = torch.zeros((most,) + c.pages.shape[1:], dtype=torch.bfloat16, device=DEV)
    at = torch.from_numpy(place).to(DEV)
    pages[at] = c.pages
    t = np.where(c.table >= 0, place[np.maximum(c.table, 0)], -1).astype(np.int32)
    big = cas.Paged(pages, 128, 128, _i32(t), c.device_start, c.ctx, c.N, 0, c.nodes)
    for max_rows in (0, 1):
        want = c.run(max_rows)
        big.max_rows = max_rows
        got = torch.zeros_like(want)
        cas.op_attention_paged(big, c.qd, got)
        assert torch.equal(got, want)
        c.check(got)
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    k, v = (torch.randn((c.N, 8 * 128), generator=g, device="cuda", dtype=torch.bfloat16) for _ in "kv")
    cos, sin = (torch.from_numpy(x).to(DEV) for x in _rope(128, 6000))
    for cache in (c.cache(), big):
        cas.op_paged_append(cache, k, v, cos=cos, sin=sin)
    assert torch.equal(pages[at].view(torch.int16), c.pages.view(torch.int16))
    rest = torch.ones(most, dtype=torch.bool, device=DEV)
    rest[at] = False
    assert all((x[y] == 0).all() for x, y in zip(pages.split(1024), rest.split(1024)))


@pytest.mark.usefixtures("table")
@pytest.mark.parametrize("H,Hkv,hd", [(8, 1, 128), (4, 4, 64)])
@pytest.mark.parametrize("seqs", [[(1, 20001, 0)], [(40, 6000, 0), (1, 5000, 0), (2, 40, 0)], [(300, 3000, 0), (1, 900, 0)]],
                         ids=["one", "chunk", "long chunk"])
def test_every_tile_of_a_split_sequence_counts_once(H, Hkv, hd, seqs):
    """Scores of two levels, one product each: a row's output is the mean of the eight
    values of the higher one, each in a tile of its own; every tile has its turn.  A
    tile left out or counted twice moves it by an eighth of a value.  Eight equal
    probabilities are rounded alike, so what is left is the sums' (n / 32 + 64) 2^-23 and
    the output's rounding."""
    c = _Batch(seqs, H, Hkv, hd, page=256)
    q = np.zeros((c.N, H, hd))
    q[..., 0] = 181.0
    c.qd = _bf(q)
    keys = c.pages[:, 0]
    keys.masked_fill_(~keys.isnan(), 0)
    flat = c.pages.view(-1)
    heads = torch.arange(Hkv, device=DEV)
    at, values = [], []
    for b, (t, Lc, _) in enumerate(seqs):
        s = np.arange(t + Lc)
        pid, tile = c.table[b][s // 256].astype(np.int64), s % 256 // 32
        place = P.key_places(hd)[s % 32, 0]
        x = torch.from_numpy(pid * 2 * Hkv * 256 * hd + tile * 32 * hd + place).to(DEV)
        at.append(x[:, None] + heads * 256 * hd)
        values.append(c.kv[b][1])
    r = _rng(H, hd, len(seqs))
    tiles = [r.permutation(Lc // 32) for _, Lc, _ in seqs]  # (of committed slots: every row sees them)
    for step in range(max(len(x) for x in tiles) // 8 + 1):
        loud = []
        for b in range(len(seqs)):
            chosen = np.take(tiles[b], np.arange(8 * step, 8 * step + 8), mode="wrap")[: len(tiles[b])]
            loud.append(np.unique(chosen * 32 + r.integers(0, 32, len(chosen))))
            flat[at[b].reshape(-1)] = 0.0
            flat[at[b][torch.from_numpy(loud[b]).to(DEV)].reshape(-1)] = 9.0
        got = _np(c.run()).reshape(c.N, H, hd)
        for b, (t, Lc, _) in enumerate(seqs):
            v = values[b][:, loud[b]]
            ref, size = (np.repeat(x.mean(1), H // Hkv, 0) for x in (v, np.abs(v)))
            err = (((t + Lc) / 32 + 64) * 2.0**-23 * size + 2.0**-8 * np.abs(ref)) * (1 + 2.0**-6)
            assert (np.abs(got[c.start[b] : c.start[b + 1]] - ref) <= err).all(), (step, b)

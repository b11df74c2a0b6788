"""Probabilities of the paged attention in two bf16 terms, where sequences have up to
32 packed rows."""
import numpy as np
import pytest
import torch

from tests import paged_ref as P
from tests.test_gpu_paged import _Batch, _np

pytestmark = pytest.mark.gpu


def _bound(q, k, v, see):
    """As P.attention, with probabilities and their sum off by 2^-16 each."""
    ref, _ = P.attention(q, k, v, see)
    T, H, hd = q.shape
    G, n, err = H // k.shape[0], see.shape[1], np.zeros(q.shape)
    for h in range(H):
        kk, vv = k[h // G], v[h // G]
        x = np.where(see, q[:, h] @ kk.T / np.sqrt(hd), -np.inf)
        p = np.exp(x - x.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        size, o = p @ np.abs(vv), np.abs(ref[:, h])
        mass = np.where(see, np.abs(q[:, h]) @ np.abs(kk).T, 0).max(1, keepdims=True) / np.sqrt(hd)
        d = 2.0**-16 + 2 * (hd + 4) * 2.0**-24 * mass + 2.0**-18
        err[:, h] = (d * (size + o) + (n / 32 + 64) * 2.0**-23 * size + 2.0**-8 * o) * (1 + 2.0**-6)
    return ref, err


@pytest.mark.parametrize("H,Hkv,hd", [(8, 2, 64), (4, 4, 128), (8, 1, 128)])
@pytest.mark.parametrize("seqs,tree", [([(1, 300, 0), (1, 31, 0), (1, 2000, 0)], False), ([(1, 9000, 0)], False),
                                       ([(4, 500, 0), (3, 77, 5)], False), ([(4, 500, 0), (2, 70, 9)], True)])
def test_few_rows_keep_the_bits_of_their_probabilities(H, Hkv, hd, seqs, tree):
    c = _Batch(seqs, H, Hkv, hd, tree=tree, std=0.3)
    got = _np(c.run(max(c.rows))).reshape(c.N, H, hd)
    for b, (t, Lc, nodes) in enumerate(seqs):
        rows = slice(c.start[b], c.start[b + 1])
        ref, err = _bound(c.q[rows], *c.kv[b], P.visible(t, Lc, nodes, c.masks and c.masks[b], 0, 0))
        assert (np.abs(got[rows] - ref) <= err).all(), (b, (np.abs(got[rows] - ref) / err).max())


@pytest.mark.parametrize("H,Hkv,hd", [(4, 4, 128), (8, 4, 64)])
def test_a_tree_of_32_rows(H, Hkv, hd):
    c = _Batch([(32 * Hkv // H, 700, 0), (5, 40, 0), (1, 1200, 0)], H, Hkv, hd, tree=True, std=0.3)
    got = _np(c.run(max(c.rows))).reshape(c.N, H, hd)
    for b, (t, Lc, _) in enumerate(c.seqs):
        rows = slice(c.start[b], c.start[b + 1])
        ref, err = _bound(c.q[rows], *c.kv[b], P.visible(t, Lc, 0, c.masks[b], 0, 0))
        assert (np.abs(got[rows] - ref) <= err).all(), (b, (np.abs(got[rows] - ref) / err).max())

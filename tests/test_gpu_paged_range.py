"""The paged attention at scores of every size that fp32 holds.  Queries and keys
have one element that is not 0, so a score is one exact product; the slots' scores
are of three levels, far enough apart that a row's output is the mean of the values
at its largest one."""
import numpy as np
import pytest
import torch

from tests import paged_ref as P
from tests.test_gpu_paged import _bf, _Batch, _np, _rng, table  # noqa: F401 (a fixture)

pytestmark = pytest.mark.gpu


def _mean(v, see, level, sign):
    """v [n][hd], see [T][n]: the mean over a row's slots of highest sign * level, and
    the largest error of one: equal probabilities are rounded alike, sums of n terms
    in runs of 32 and their joins give (n / 32 + 64) 2^-23 of the terms, the output's
    rounding 2^-8."""
    x = np.where(see, sign[:, None] * level, -np.inf)
    p = (x == x.max(1, keepdims=True)).astype(np.float64)
    p /= p.sum(1, keepdims=True)
    o, size = p @ v, p @ np.abs(v)
    return o, ((see.shape[1] / 32 + 64) * 2.0**-23 * size + 2.0**-8 * np.abs(o)) * (1 + 2.0**-6)


@pytest.mark.usefixtures("table")
@pytest.mark.parametrize("exponent", [14, 16, 19, 24, 40, 84, 90, 110])
@pytest.mark.parametrize("seqs", [[(1, 500, 0), (9, 200, 0)], [(40, 100, 0), (50, 33, 0)], [(1, 20001, 0)], [(300, 77, 0)]],
                         ids=["few", "chunks", "split", "long chunk"])
@pytest.mark.parametrize("hd", [64, 128])
def test_scores_of_every_size(seqs, exponent, hd):
    """Scores of 181 times 129, 193 or 255 times 2^exponent, of either sign."""
    c = _Batch(seqs, 4, 2, hd)
    r = _rng(exponent, hd)
    levels = [r.choice([129.0, 193.0, 255.0], sum(s)) * r.choice([-1, 1]) for s in seqs]
    a = exponent // 2
    for b, (s, x) in enumerate(zip(seqs, levels)):
        k = np.zeros_like(c.kv[b][0])
        k[..., 0] = x * 2.0 ** (exponent - a)
        for slot in range(sum(s)):
            P.put(c.pool, hd, c.page, c.table[b], slot, k[:, slot], c.kv[b][1][:, slot])
    sign = r.choice([-1.0, 1.0], (c.N, 4))
    q = np.zeros((c.N, 4, hd))
    q[..., 0] = sign * 181 * 2.0**a
    c.pages, c.qd = _bf(c.pool), _bf(q)
    got = _np(c.run()).reshape(c.N, 4, hd)
    for b, (t, Lc, _) in enumerate(seqs):
        rows = slice(c.start[b], c.start[b + 1])
        see = P.visible(t, Lc, 0, None, 0, 0)
        for h in range(4):
            ref, err = _mean(c.kv[b][1][h // 2], see, levels[b], sign[rows, h])
            over = np.abs(got[rows, h] - ref) / err
            assert np.isfinite(got[rows, h]).all() and over.max() <= 1, (b, h, over.max())
    torch.cuda.synchronize()

"""The 4-bit cache's attention at scores of every size that fp32 holds (as
test_gpu_paged_range.py: one element that is not 0, three levels of scores, which
four bits hold exactly)."""
import numpy as np
import pytest
import torch

from paper_2510_26843_amd import cas
from tests import paged_ref as P
from tests.test_gpu_paged import _bf, _np, _rng, _words
from tests.test_gpu_paged_range import _mean

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("exponent", [10, 20, 26, 40, 90, 110])
@pytest.mark.parametrize("T,Lc,tail", [(1, 500, 0), (9, 200, 0), (64, 4000, 0), (3, 20000, 0), (5, 300, 32)])
@pytest.mark.parametrize("hd", [64, 128])
def test_scores_of_every_size(T, Lc, tail, exponent, hd):
    """Scores of 181 times 3, 4 or 6 times 2^exponent, of either sign; tail: the last slots in bf16."""
    H, Hkv, n = 4, 2, Lc + T
    cap = (n + 31) // 32 * 32
    r = _rng(exponent, hd, T, Lc)
    level = r.choice([3.0, 4.0, 6.0], n) * r.choice([-1, 1])
    a = exponent // 2
    k = np.zeros((n, Hkv, hd))
    k[..., 0] = level[:, None] * 2.0 ** (exponent - a)
    v = np.exp2(r.integers(-2, 3, (n, Hkv, hd)).astype(np.float64)) * r.choice([-1, 1], (n, Hkv, hd))
    kd, vd = _bf(k), _bf(v)
    cache = torch.zeros(cas.kv4_bytes(Hkv, hd, cap), dtype=torch.uint8, device="cuda")
    cas.op_kv4_append(kd.reshape(n, -1), vd.reshape(n, -1), n, Hkv, hd, cache, cap, 0)
    n4, kw = n, {}
    if tail:
        n4 = Lc // 32 * 32 - tail
        kw = dict(k=kd[n4:].transpose(0, 1).contiguous(), v=vd[n4:].transpose(0, 1).contiguous())
    kept_k, kept_v = (torch.zeros((Hkv, n, hd), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    cas.op_kv4_read(cache, cap, 0, n, Hkv, hd, kept_k, kept_v)
    assert np.array_equal(_np(kept_k), k.transpose(1, 0, 2))
    values = v.transpose(1, 0, 2).copy()
    values[:, :n4] = _np(kept_v)[:, :n4]
    sign = r.choice([-1.0, 1.0], (T, H))
    q = np.zeros((T, H, hd))
    q[..., 0] = sign * 181 * 2.0**a
    anc = _words([(1 << (i + 1)) - 1 for i in range(T)])
    out = torch.full((T, H * hd), 7.0, dtype=torch.bfloat16, device="cuda")
    cas.op_attention_kv4(_bf(q), cache, cap, n4, Lc, T, T, H, Hkv, hd, anc, out, **kw)
    got = _np(out).reshape(T, H, hd)
    see = P.visible(T, Lc, 0, None, 0, 0)
    for h in range(H):
        ref, err = _mean(values[h // 2], see, level, sign[:, h])
        assert np.isfinite(got[:, h]).all() and (np.abs(got[:, h] - ref) <= err).all(), h

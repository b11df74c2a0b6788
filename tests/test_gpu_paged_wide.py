"""The paged attention with as many query heads to a kv head as it takes: a packed
row's token and head come from a division that has to be exact."""
import numpy as np
import pytest
import torch

from tests import paged_ref as P
from tests.test_gpu_paged import _Batch, _np

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("max_rows", [1, 0])
@pytest.mark.parametrize("T,H,Hkv", [(258, 4092, 1), (1030, 4092, 2)])
def test_thousands_of_heads_to_a_group(T, H, Hkv, max_rows):
    c = _Batch([(T, 3, 0)], Hkv, Hkv, 64)
    c.H = H
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    c.qd = torch.randn((T, H, 64), generator=g, device="cuda", dtype=torch.bfloat16)
    out = c.run(max_rows).view(T, H, 64)
    assert torch.isfinite(out).all()
    G = H // Hkv
    heads = [h for k in range(Hkv) for h in (k * G, k * G + G - 1)]
    ref, err = P.attention(_np(c.qd[:, heads]), *c.kv[0], P.visible(T, 3, 0, None, 0, 0))
    assert (np.abs(_np(out[:, heads]) - ref) <= err).all()

"""4-bit drafts of the decoder in the forms of long contexts and of cascades."""
import numpy as np
import pytest

from paper_2510_26843_amd import cas, synth

pytestmark = pytest.mark.gpu

# two layers whose gate/up matrix (2 x 4096 rows) and LM head have the 8192
# rows from which the GEMV-style tiles are taken
WIDE = synth.ModelShape("wide", 2, 1024, 8, 8, 128, 4096, 8192, 1e4, 1e-6, "bf16")
TOL = 2e-2


def _row_err(got, ref):
    return float((np.abs(got - ref).max(axis=1) / np.abs(ref).max(axis=1)).max())


def _bits(a):
    return a.view(np.uint32)


@pytest.mark.parametrize("opts", [{}, {"skip": [0, 1]}, {"attn_window": (4, 64)}], ids=["4-bit KV only", "skip", "window"])
def test_gemv_tiles_of_one_row_drafts(opts):
    """cas_set_gemv moves a one-row draft over the copy by rounding (other sums'
    order), and leaves drafts of two rows and verify calls as they are."""
    m = cas.Model(WIDE, max_ctx=512, max_tree=32)
    m.load_weights(synth.gen_weights(WIDE, seed=3))
    m.build_kv4()
    m.prefill([int(x) for x in synth.gen_prompt(WIDE.vocab, 200, seed=1)])
    calls = [lambda: m.forward([5], [-1], kv4=True, **opts), lambda: m.forward([5, 6], [-1, 0], kv4=True, **opts),
             lambda: m.forward([5], [-1])]
    before = [f() for f in calls]
    m.set_gemv(True)
    gemv = [f() for f in calls]
    m.set_gemv(False)
    assert not np.array_equal(_bits(gemv[0]), _bits(before[0])) and _row_err(gemv[0], before[0]) < TOL
    assert np.array_equal(_bits(gemv[1]), _bits(before[1])) and np.array_equal(_bits(gemv[2]), _bits(before[2]))
    assert np.array_equal(_bits(calls[0]()), _bits(before[0]))
    m.close()

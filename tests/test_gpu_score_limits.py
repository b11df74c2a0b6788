"""Scores at the ends of what the calls take: the largest scale, parts of as many
chunks as one may have, scratch of exactly the reported size."""
import numpy as np
import pytest
import torch

from paper_2510_26843_amd import cas, synth
from tests.test_gpu_logprobs import DEV, _check, _logits, _run

pytestmark = pytest.mark.gpu

# the largest fp32 whose product with log2(e) is one
LARGEST = np.nextafter(np.float32(np.finfo(np.float32).max / np.log2(np.e)), np.float32(0))


@pytest.mark.parametrize("V", [500, 40000])
def test_the_largest_scale(V):
    x = _logits(3, V, False)
    x[1] = -2.0
    x[2, 3:7] = x[2].max()
    best = x[2].max().item()
    logp, ent, ids, top = _run(x, [[3, 0]] * 3, 2, scale=float(LARGEST))
    M = int(x[0].argmax())
    assert logp[0, 0] == (0 if M == 3 else -np.inf) and ent[0] == 0 and ids[0, 0] == M and top[0, 0] == 0
    # (equal logits: - log n, within 2^-22 of it and of the sum's 2^-18)
    assert np.abs(logp[1] + np.log(V)).max() < 1e-5 and abs(ent[1] - np.log(V)) < 1e-5 and list(ids[1]) == [0, 1]
    n = int((x[2] == best).sum())
    assert abs(logp[2, 0] + np.log(n)) < 1e-5 and abs(ent[2] - np.log(n)) < 1e-5
    for scale in (float(np.nextafter(LARGEST, np.float32(np.inf))) * (1 + 1e-6), 3e38):
        with pytest.raises(cas.CasError, match="CAS_ERR_ARG"):
            _run(x, [[3, 0]] * 3, 2, scale=scale)


def test_the_largest_scale_of_a_model():
    shape = synth.SHAPES["tiny"]
    m = cas.Model(shape, max_ctx=128)
    m.load_weights(synth.gen_weights(shape, seed=3))
    logits = m.forward([1, 2], [-1, 0])
    logp, ent, ids, best = m.logprobs(logits.argmax(1), 1, float(LARGEST))
    assert (logp == 0).all() and (ent == 0).all() and np.array_equal(ids[:, 0], logits.argmax(1)) and (best == 0).all()
    with pytest.raises(cas.CasError) as e:
        m.logprobs([1, 2], 0, 3e38)
    assert e.value.status == cas.ERR_ARG
    m.close()


def test_a_row_without_a_distribution_is_called_that():
    """A logit of +infinity leaves none, and holds no NaN; one of -infinity has probability 0."""
    shape = synth.SHAPES["tiny"]
    w = synth.gen_weights(shape, seed=3)
    w["lm_head"] = w["lm_head"].copy()
    signs = set()
    for value in (np.inf, -np.inf):
        w["lm_head"][5, 0] = value
        m = cas.Model(shape, max_ctx=128)
        m.load_weights(w)
        logits = m.forward([1], [-1])
        assert np.isinf(logits[0, 5]) and np.isfinite(np.delete(logits[0], 5)).all()
        signs.add(float(np.sign(logits[0, 5])))
        if logits[0, 5] > 0:
            with pytest.raises(cas.CasError, match="row 0 has no distribution") as e:
                m.logprobs([5])
            assert e.value.status == cas.ERR_DEVICE
        else:
            assert m.logprobs([5])[0][0] == -np.inf
        m.close()
    assert len(signs) == 2


@pytest.mark.parametrize("n,V", [(1100, 270000), (600, 20000), (2100, 70000), (513, 32768)])
def test_parts_of_many_rows(n, V):
    """Parts of as many chunks as one may have (270000 logits in two), many short rows in
    parts, rows more than the records' first bound; in scratch of the reported size."""
    g = torch.Generator(device="cuda")
    g.manual_seed(V)
    x = torch.randn((n, V), generator=g, device="cuda", dtype=torch.bfloat16)
    rows = [0, 1, n // 2, n - 2, n - 1]
    # the best of some rows in the last chunks of their parts
    for r, ids in zip(rows, ([V - 1, V - 2, 0], [31 * 8192 + 7, 32 * 8192 - 1, 32 * 8192], [V // 2, 8191, 8192])):
        for i, best in zip(ids, (9.0, 8.0, 8.0)):
            if i < V:
                x[r, i] = best
    tokens = torch.randint(V, (n, 2), generator=g, device="cuda").cpu().numpy()
    need = cas.lib().cas_op_logprobs_work_bytes(n, V, 32)
    room = torch.full((need + (1 << 16),), 77, dtype=torch.uint8, device=DEV)
    got = _run(x, tokens, 32, work=room[:need])
    assert (room[need:] == 77).all()
    assert np.isfinite(got[0]).all() and np.isfinite(got[1]).all() and (got[2] >= 0).all()
    _check(x[rows], tokens[rows], 32, 1.0, [y[rows] for y in got])

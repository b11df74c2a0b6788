"""Model.logprobs and decode.score on the GPU: against 64 bits on the very logits
that the library produced."""
import numpy as np
import pytest

from paper_2510_26843_amd import cas, decode, synth

pytestmark = pytest.mark.gpu

TINY = synth.SHAPES["tiny"]
GQA = synth.ModelShape("gqa_small", 2, 512, 8, 2, 64, 1376, 1024, 5e5, 1e-6, "bf16")


@pytest.fixture(scope="module", params=[TINY, GQA], ids=["fp32", "bf16"])
def model(request):
    m = cas.Model(request.param, max_ctx=512, max_tree=48)
    m.load_weights(synth.gen_weights(request.param, seed=3))
    yield m
    m.close()


def _reference(logits, scale=1.0):
    x = logits.astype(np.float64) * scale
    x = x - x.max(1, keepdims=True)
    lp = x - np.log(np.exp(x).sum(1, keepdims=True))
    return lp, -(np.exp(lp) * lp).sum(1)


# (see test_gpu_logprobs.py: below 8e-6 for sums, below 1e-4 for entropies, at these sizes)
@pytest.mark.parametrize("n,m,K,scale", [(1, 1, 0, 1.0), (1, 3, 5, 0.7), (15, 4, 16, 1.0), (48, 128, 32, 2.0)])
def test_logprobs_of_the_last_forward(model, n, m, K, scale):
    r = np.random.default_rng([n, m])
    V = model.shape.vocab
    model.set_committed(0)
    logits = model.forward(r.integers(0, V, n), [-1] + [int(r.integers(0, i)) for i in range(1, n)])
    tokens = r.integers(0, V, (n, m))
    logp, entropy, ids, best = model.logprobs(tokens, K, scale)
    lp, h = _reference(logits, scale)
    assert np.abs(logp - np.take_along_axis(lp, tokens, 1)).max() < 8e-6
    assert np.abs(entropy - h).max() < 1e-4
    order = np.argsort(-logits, axis=1, kind="stable")[:, :K]
    assert np.array_equal(ids, order)
    if K:
        assert np.abs(best - np.take_along_axis(lp, order, 1)).max() < 8e-6
    if 0 < K <= 16 and scale == 1.0:
        top, probs = model.topk(K, n)
        assert np.array_equal(top, ids) and np.allclose(np.exp(best), probs, rtol=1e-5)


def test_tokens_outside_the_vocabulary(model):
    model.set_committed(0)
    model.forward([1, 2], [-1, 0], logits=False)
    logp, entropy, _, _ = model.logprobs([[-1, 0], [model.shape.vocab, 2**31 - 1]])
    assert np.array_equal(np.isnan(logp), [[True, False], [True, True]]) and np.isfinite(entropy).all()
    assert model.logprobs(np.zeros((2, 0)), 3)[0].shape == (2, 0)


def test_refusals(model):
    model.set_committed(0)
    model.forward([1, 2], [-1, 0], logits=False)
    for args in [([1],), ([1, 2], 33), ([1, 2], 0, 0.0), ([1, 2], 0, float("nan")), (np.zeros((2, 129)),)]:
        with pytest.raises(cas.CasError) as e:
            model.logprobs(*args)
        assert e.value.status == cas.ERR_ARG
    model.logprobs([1, 2])


def test_needs_a_forward():
    m = cas.Model(TINY, max_ctx=128)
    m.load_weights(synth.gen_weights(TINY, seed=3))
    with pytest.raises(cas.CasError) as e:
        m.logprobs([1])
    assert e.value.status == cas.ERR_STATE
    m.close()


@pytest.mark.parametrize("n", [1, 2, 48, 49, 131])
def test_score(model, n):
    """A text's log probabilities, chunk by chunk, against those of one token at a
    time: bf16 forwards give a row the same bits in both; fp32 ones sum in another
    order (1e-5 of a row's largest logit, which is below 4)."""
    tol = 8e-6 + (4e-5 if model.shape.dtype == "f32" else 0)
    V = model.shape.vocab
    text = synth.gen_prompt(V, n, seed=7)
    logp, entropy, ids, best = decode.score(model, text, K=3)
    assert model.committed == n and logp.shape == (n - 1,) and ids.shape == (n - 1, 3)
    model.set_committed(0)
    for i in range(n - 1):
        lp, h = _reference(model.forward([int(text[i])], [-1]))
        model.compact([0])
        assert abs(logp[i] - lp[0, text[i + 1]]) < tol and abs(entropy[i] - h[0]) < 1e-4 + tol, i
        order = np.argsort(-lp[0], kind="stable")[:3]
        assert np.array_equal(ids[i], order) and np.abs(best[i] - lp[0, order]).max() < tol

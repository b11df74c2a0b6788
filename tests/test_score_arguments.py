"""What Model.logprobs and decode.score make of their arguments.  CPU: a model
whose library notes what reaches it."""
import ctypes

import numpy as np
import pytest

from paper_2510_26843_amd import cas, decode

V = 100


class _Lib:
    """cas_logprobs answers -1 - token, so that a result shows whose it is."""

    def __init__(self):
        self.calls = []

    def cas_logprobs(self, h, n, scale, tokens, m, logp, entropy, K, ids, best):
        read = lambda at, k, t: np.ctypeslib.as_array(ctypes.cast(at, ctypes.POINTER(t)), (k,))  # noqa: E731
        t = read(tokens, n * m, ctypes.c_int32).copy() if n * m else np.zeros(0, np.int32)
        self.calls.append((n, m, K, t.tolist()))
        if n * m:
            read(logp, n * m, ctypes.c_float)[:] = np.where((t >= 0) & (t < V), -1.0 - t, np.nan)
        return 0

    def __getattr__(self, name):
        return lambda *a: 0


@pytest.fixture
def model():
    m = cas.Model.__new__(cas.Model)
    m.h, m._L, m.max_tree = 1, _Lib(), 4
    return m


@pytest.mark.parametrize("tokens,n,m", [([3, 4], 2, 1), ([[3, 4, 5]], 1, 3), (np.arange(6, dtype=np.int64).reshape(2, 3), 2, 3),
                                        (np.zeros((2, 0)), 2, 0)])
def test_tokens_of_rows(model, tokens, n, m):
    logp = model.logprobs(tokens)[0]
    assert model._L.calls[0][:3] == (n, m, 0) and logp.shape == np.shape(tokens)
    assert np.array_equal(logp, -1.0 - np.asarray(tokens))


@pytest.mark.parametrize("tokens", [np.zeros((2, 3, 2), np.int32), np.zeros((2, 1, 1), np.int32)])
def test_tokens_that_are_not_of_rows(model, tokens):
    with pytest.raises(cas.CasError) as e:
        model.logprobs(tokens)
    assert e.value.status == cas.ERR_ARG and not model._L.calls


def test_ids_that_32_bits_do_not_hold_are_no_tokens(model):
    logp = model.logprobs(np.array([[2**32 + 5, 7], [-(2**32) + 5, 2**31]], dtype=np.int64))[0]
    assert np.array_equal(np.isnan(logp), [[True, False], [True, True]]) and logp[0, 1] == -8
    logp = model.logprobs(np.array([2**64 - 2**32 + 5, 6], dtype=np.uint64))[0]
    assert np.isnan(logp[0]) and logp[1] == -7


def test_a_text_with_such_an_id_reaches_no_other_token(model, monkeypatch):
    seen = []
    monkeypatch.setattr(model, "forward", lambda t, *a, **kw: seen.extend(np.asarray(t, dtype=np.int32).tolist()))
    decode.score(model, np.array([1, 2**32 + 5, 3], dtype=np.int64))
    assert seen == [1, -1, 3]  # (the library refuses a token of -1)


@pytest.mark.parametrize("K", [0, 3])
def test_a_text_without_tokens_has_no_scores(model, K):
    logp, entropy, ids, best = decode.score(model, [], K)
    assert logp.shape == entropy.shape == (0,) and ids.shape == best.shape == (0, K)
    one = decode.score(model, [7], K)
    assert [(x.shape, x.dtype) for x in one] == [(x.shape, x.dtype) for x in (logp, entropy, ids, best)]


def test_several_texts_at_once_are_refused(model, monkeypatch):
    """(the first row's tokens would have been scored as each other's continuations)"""
    seen = []
    monkeypatch.setattr(model, "forward", lambda t, *a, **kw: seen.append(np.shape(t)))
    with pytest.raises(cas.CasError) as e:
        decode.score(model, [[1, 2, 3], [4, 5, 6]])
    assert e.value.status == cas.ERR_ARG and not seen

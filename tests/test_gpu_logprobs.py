"""Log probabilities, entropy and top alternatives on the GPU against 64 bits.

Tolerance: with d = x - M (exact to 2^-24 of it) times the scale, a term e^l is
off by (|l| 2^-22 + 2^-21) of itself (l's three roundings and the exponential's,
absolute in l), where |l| <= 104 counts (below, a term is 0 against S >= 1).
S sums up to 2^20 positive terms in runs of 32 and short trees: 64 2^-24 of it.
So log S is off by at most E = 104 * 2^-22 + 2^-21 + 64 * 2^-24 < 3e-5 at the
very worst; only terms that count move it, and weighted by its own p a term's
|l| is at most log V + 1 in the mean: e = (log V + 2) 2^-22 + 64 * 2^-24 < 8e-6.
logp = l - log S: 2 * 2^-24 (|l| + log S) more.  The entropy adds sum p |l|
errors: (log V + 1) e and 2^-22 (log V + 1)."""
import numpy as np
import pytest
import torch

from paper_2510_26843_amd import cas

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _logits(n, V, bf16, seed=0, spread=2.5):
    r = np.random.default_rng([3, n, V, seed])
    x = r.normal(0, spread, (n, V))
    x[np.arange(n)[:, None], r.integers(0, V, (n, 6))] += r.uniform(0, 14, (n, 6))
    return torch.from_numpy(x).to(torch.bfloat16 if bf16 else torch.float32).to(DEV)


def _run(x, tokens, K, scale=1.0, entropy=True, **kw):
    n = x.shape[0]
    t = None if tokens is None else torch.tensor(np.asarray(tokens), dtype=torch.int32, device=DEV)
    logp = None if t is None else torch.full(t.shape, 7.0, device=DEV)
    ent = torch.full((n,), 7.0, device=DEV) if entropy else None
    ids = torch.full((n, K), 7, dtype=torch.int32, device=DEV) if K else None
    best = torch.full((n, K), 7.0, device=DEV) if K else None
    cas.op_logprobs(x, t, logp, ent, ids, best, scale=scale, **kw)
    return [None if y is None else y.cpu().numpy() for y in (logp, ent, ids, best)]


def _check(x, tokens, K, scale, got):
    y = x.double().cpu().numpy()
    n, V = y.shape
    logp, ent, ids, best = got
    for r in range(n):
        M = y[r].max()
        l = np.where(y[r] == -np.inf, -np.inf, (y[r] - M) * scale)
        S = np.exp(l).sum()
        lp = l - np.log(S)
        e = (np.log(V) + 2) * 2.0**-22 + 64 * 2.0**-24
        tol = lambda t: e + 2.0**-23 * (np.abs(np.where(np.isfinite(t), t, 0)) + np.log(S))  # noqa: E731
        if logp is not None:
            for t, p in zip(tokens[r], logp[r]):
                if not 0 <= t < V:
                    assert np.isnan(p)
                elif lp[t] == -np.inf:
                    assert p == -np.inf
                else:
                    assert abs(p - lp[t]) <= tol(lp[t]), (r, t, p, lp[t])
        p = np.exp(lp)
        h = -(p * np.where(p > 0, lp, 0)).sum()
        if ent is not None:
            assert abs(ent[r] - h) <= (np.log(V) + 2) * e + 2.0**-22 * (np.log(V) + 1), (r, ent[r], h)
        if K:
            order = np.lexsort((np.arange(V), -y[r]))[:K]
            order = order[y[r][order] > -np.inf]
            want = np.concatenate([order, np.full(K - len(order), -1)])
            assert np.array_equal(ids[r], want), r
            assert (np.abs(best[r][: len(order)] - lp[order]) <= tol(lp[order])).all()
            assert (best[r][len(order) :] == -np.inf).all()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("n,V,m,K,scale", [
    (1, 1, 1, 1, 1.0), (1, 2, 3, 5, 1.0), (3, 63, 1, 32, 0.5), (2, 100, 0, 3, 1.0), (5, 1000, 4, 0, 2.0), (1, 8191, 2, 16, 1.0),
    (2, 8192, 2, 16, 1.0), (2, 8193, 2, 16, 1.0), (61, 32000, 4, 8, 1.25), (3, 128256, 1, 20, 0.7), (1, 300007, 300, 32, 1.0),
    (3, 64000, 1, 32, 1.0), (40, 64000, 1, 31, 1.0), (300, 9000, 2, 8, 1.0), (130, 50000, 1, 20, 1.0), (600, 33000, 1, 9, 1.0)])
def test_logprobs(n, V, m, K, scale, bf16):
    x = _logits(n, V, bf16)
    t = np.random.default_rng(n + V).integers(0, V, (n, m)) if m else None
    _check(x, t, K, scale, _run(x, t, K, scale))


def test_the_longest_row():
    x = _logits(1, 1 << 20, False)
    t = [[0, (1 << 20) - 1]]
    _check(x, t, 32, 1.0, _run(x, t, 32))


@pytest.mark.parametrize("V", [20000, 64000])
@pytest.mark.parametrize("bf16", [False, True])
def test_ties(bf16, V):
    """Equal logits everywhere, in one wave's part, or in bands: lowest ids first."""
    x = torch.zeros((6, V), device=DEV)
    x[1, 300:900] = 3.0
    x[2] = torch.arange(V, device=DEV) % 7
    x[3, 8000:8400] = -0.0
    x[4] = -1.0
    x[4, V - 10 :] = 0.0
    x[5, :10] = -0.0
    if bf16:
        x = x.to(torch.bfloat16)
    t = [[0, V - 1]] * 6
    _check(x, t, 32, 1.0, _run(x, t, 32))


@pytest.mark.parametrize("V", [5, 70, 9000])
def test_masked_tokens(V):
    """Logits of -infinity have no part; fewer finite ones than alternatives."""
    x = torch.full((4, V), -float("inf"), device=DEV)
    x[0, V - 1] = -3.0
    x[1, ::3] = torch.arange(len(x[1, ::3]), device=DEV).float() * -0.01
    x[2, 1:4] = 2.0
    x[3] = 1.0
    x[3, 0] = -float("inf")
    t = [[0, V - 1, V // 2, -1, V, 2**31 - 1, -(2**31)]] * 4
    _check(x, t, 20, 1.0, _run(x, t, 20))


def test_large_logits():
    """Differences past what an exponential or fp32 holds."""
    x = torch.zeros((4, 500), device=DEV)
    x[0] = -3.0e38
    x[0, 7] = 3.0e38
    x[1] = 3.0e38
    x[2] = torch.linspace(-1e4, 1e4, 500)
    x[3] = torch.linspace(-80, -160, 500)
    logp, ent, ids, best = _run(x, [[7, 8]] * 4, 3, 1.0)
    assert logp[0, 0] == 0 and logp[0, 1] == -np.inf and ent[0] == 0 and ids[0, 0] == 7
    assert abs(logp[1, 0] + np.log(500)) < 1e-5 and list(ids[1]) == [0, 1, 2]
    _check(x[2:], [[7, 8]] * 2, 3, 1.0, [y[2:] for y in (logp, ent, ids, best)])


@pytest.mark.parametrize("value", [float("nan"), float("inf"), None])
def test_rows_without_a_distribution(value):
    x = _logits(3, 20000, False)
    want = _run(x, [[5]] * 3, 4)
    if value is None:
        x[1] = -float("inf")
    else:
        x[1, 12345] = value
    got = _run(x, [[5]] * 3, 4)
    for w, g in zip(want, got):
        assert np.array_equal(w[[0, 2]], g[[0, 2]])
    assert np.isnan(got[0][1]).all() and np.isnan(got[1][1]) and (got[2][1] == -1).all() and np.isnan(got[3][1]).all()


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("first,ld", [(0, 1003), (1, 1003), (3, 2000), (5, 1009)])
def test_strided_rows(first, ld, bf16):
    """Rows within a wider buffer, at every alignment an element allows."""
    wide = _logits(4, ld + 8, bf16, seed=first)
    flat = wide.reshape(-1)[: 3 * ld + 1003 + first]
    x = torch.as_strided(flat, (4, 1003), (ld, 1), first)
    t = [[1, 1002]] * 4
    _check(x, t, 5, 1.0, _run(x, t, 5))


def test_replayed():
    """A captured call reads what its tensors hold at the time of the replay."""
    x, work = _logits(3, 40000, False), torch.empty(1 << 20, dtype=torch.uint8, device=DEV)
    t = torch.tensor([[1], [2], [3]], dtype=torch.int32, device=DEV)
    out = [torch.zeros((3, 1), device=DEV), torch.zeros(3, device=DEV), torch.zeros((3, 6), dtype=torch.int32, device=DEV),
           torch.zeros((3, 6), device=DEV)]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        cas.op_logprobs(x, t, *out, work=work)
    for i in range(4):
        x.copy_(_logits(3, 40000, False, seed=i))
        t.fill_(100 * i)
        graph.replay()
        want = _run(x, t.cpu().numpy(), 6)
        torch.cuda.synchronize()
        for w, g in zip(want, out):
            assert np.array_equal(w, g.cpu().numpy())


@pytest.mark.parametrize("V", [32000, 70000])
def test_scratch_of_more_rows(V):
    """One scratch, sized for the most rows, serves calls of fewer; nothing behind it is written."""
    need = cas.lib().cas_op_logprobs_work_bytes(128, V, 32)
    room = torch.full((need + (1 << 20),), 77, dtype=torch.uint8, device=DEV)
    x = _logits(128, V, False)
    for n in (1, 2, 17, 31, 32, 33, 64, 65, 128):
        _check(x[:n], [[n]] * n, 32, 1.0, _run(x[:n], [[n]] * n, 32, work=room[:need]))
        assert (room[need:] == 77).all()

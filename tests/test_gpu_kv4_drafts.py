"""4-bit drafts of the decoder in the forms of long contexts and of cascades."""
import numpy as np
import pytest
import torch

from oracle import oracle as O
from paper_2510_26843_amd import cas, dytc, synth

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


# ---------------------------------------------------------------- long contexts

GQA = synth.ModelShape("gqa_small", 2, 512, 8, 2, 64, 1376, 1024, 5e5, 1e-6, "bf16")
MHA = synth.ModelShape("mha_small", 2, 1024, 8, 8, 128, 2752, 4096, 1e4, 1e-6, "bf16")
LONG = 8190


def _splits(shape, T, Lc, window=(0, 0)):
    """The runs of key tiles that a draft's attention is split into."""
    b = cas.lib().cas_op_attention_kv4_work_bytes(Lc, T, T, shape.n_heads, shape.n_kv_heads, shape.head_dim, *window)
    return max(1, b // (4 * T * shape.n_heads * (shape.head_dim + 2)))


def _held(k, v):
    """bf16 bits [Hkv][n][hd] of the values that the 4-bit copy of such keys and
    values stands for (its form: tests/test_gpu_kv4.py)."""
    Hkv, n, hd = k.shape
    rows = [torch.from_numpy(x.view(np.int16)).cuda().transpose(0, 1).reshape(n, -1) for x in (k, v)]
    rec = torch.zeros((Hkv, n // 32, 34 * hd), dtype=torch.uint8, device="cuda")
    cas.op_kv4_append(*rows, n, Hkv, hd, rec, n, 0)
    out = torch.empty((2, Hkv, n, hd), dtype=torch.int16, device="cuda")
    cas.op_kv4_read(rec, n, 0, n, Hkv, hd, out[0], out[1])
    return out.cpu().numpy().view(np.uint16)


class _Pair:
    """A model with a copy, and one whose bf16 cache holds what the copy stands for."""

    def __init__(self, shape, max_ctx=LONG + 130, max_tree=128):
        self.shape = shape
        k, v = synth.gen_kv(shape.n_layers, shape.n_kv_heads, LONG, shape.head_dim, seed=5)
        self.kv = [[synth.f32_to_bf16_bits(x[l]) for x in (k, v)] for l in range(shape.n_layers)]
        w = synth.gen_weights(shape, seed=9)
        self.m, self.ref = (cas.Model(shape, max_ctx=max_ctx, max_tree=max_tree) for _ in range(2))
        for x in (self.m, self.ref):
            x.load_weights(w)
            x.build_int8()
        self.m.build_kv4()

    def commit(self, Lc):
        c = Lc // 32 * 32
        for l, (k, v) in enumerate(self.kv):
            self.m.kv_load(l, k[:, :Lc], v[:, :Lc])
            k4, v4 = _held(np.ascontiguousarray(k[:, :c]), np.ascontiguousarray(v[:, :c]))
            self.ref.kv_load(l, np.concatenate((k4, k[:, c:Lc]), 1), np.concatenate((v4, v[:, c:Lc]), 1))
        for x in (self.m, self.ref):
            x.set_committed(Lc)

    def close(self):
        self.m.close()
        self.ref.close()


@pytest.fixture(scope="module", params=[GQA, MHA], ids=lambda s: s.name)
def pair(request):
    p = _Pair(request.param)
    yield p
    p.close()


def _tree(shape, n, seed=2):
    parents = synth.balanced_tree(n)
    return synth.gen_tree_tokens(parents, shape.vocab, seed=seed), parents


@pytest.mark.parametrize("Lc", [LONG, 4100, 2240])
def test_long_drafts_are_those_of_the_copys_values(pair, Lc):
    """Split attention in the decoder: its partials joined by the O projection
    (one or two rows), by the merge into the tiled rows, and with int8
    activations by the quantiser on load or by the merge that writes codes
    (bar: 6e-2, a rounding may move a code by a whole step)."""
    shape = pair.shape
    pair.commit(Lc)
    for T in (1, 2, 3, 16, 33, 128):
        toks, parents = _tree(shape, T)
        assert _splits(shape, T, Lc) > 1 or T > 16
        for aq, bar in ((0, TOL), (1, 6e-2)):
            got = pair.m.forward(toks, parents, act_quant=aq, kv4=True)
            want = pair.ref.forward(toks, parents, act_quant=aq)
            err = _row_err(got, want)
            assert err < bar, (T, aq, err)
            if not aq:  # the cache's quantisation moves the logits by more than that rounding
                assert _row_err(pair.m.forward(toks, parents), want) > 2 * err, (T, err)


@pytest.mark.parametrize("window", [(4, 5000), (40, 3000)])
def test_long_window_drafts(pair, window):
    pair.commit(LONG)
    for T in (1, 3, 16):
        toks, parents = _tree(pair.shape, T)
        assert _splits(pair.shape, T, LONG, window) > 1
        err = _row_err(pair.m.forward(toks, parents, attn_window=window, kv4=True),
                       pair.ref.forward(toks, parents, attn_window=window))
        assert err < TOL, (T, err)


def test_graphs_of_other_split_counts(pair):
    """Graph replays and direct launches give the same bits while the context,
    and with it the number of splits, changes between the calls."""
    shape, m = pair.shape, pair.m
    pair.commit(LONG)
    seen = {T: set() for T in (1, 2, 16)}
    first = {}
    for Lc in (LONG, 6000, 2240, 100):  # (nodes are written behind Lc, so downwards)
        for T in seen:
            m.set_committed(Lc)
            seen[T].add(_splits(shape, T, Lc))
            toks, parents = _tree(shape, T)
            for aq in (0, 1):
                a = m.forward(toks, parents, act_quant=aq, kv4=True)
                b = m.forward(toks, parents, act_quant=aq, kv4=True)
                m.set_graphs(False)
                c = m.forward(toks, parents, act_quant=aq, kv4=True)
                m.set_graphs(True)
                assert np.array_equal(_bits(a), _bits(b)) and np.array_equal(_bits(a), _bits(c)), (Lc, T, aq)
                first[Lc, T, aq] = a
    assert all(len(s) >= 3 for s in seen.values()), seen
    pair.commit(LONG)  # ... and again, from the graphs captured above
    for Lc in (LONG, 6000, 2240, 100):
        for T in seen:
            m.set_committed(Lc)
            toks, parents = _tree(shape, T)
            assert np.array_equal(_bits(m.forward(toks, parents, kv4=True)), _bits(first[Lc, T, 0])), (Lc, T)


@pytest.mark.parametrize("shape", [GQA, MHA], ids=lambda s: s.name)
def test_no_more_splits_than_the_partials_buffer_holds(shape):
    """A cache of 2304 slots has room for the partial states of 9 splits of the
    largest tree; the plan for 71 key tiles would take 10."""
    assert _splits(shape, 16, 2240) == 10
    p = _Pair(shape, max_ctx=2304, max_tree=16)
    p.commit(2240)
    toks, parents = _tree(shape, 16)
    for aq, bar in ((0, TOL), (1, 6e-2)):
        err = _row_err(p.m.forward(toks, parents, act_quant=aq, kv4=True), p.ref.forward(toks, parents, act_quant=aq))
        assert err < bar, (aq, err)
    p.close()


# ---------------------------------------------------------------- a cascade

@pytest.mark.parametrize("full", [True, False], ids=["all layers too", "skips only"])
def test_dytc_over_4_bit_drafts_is_lossless(full):
    """A cascade whose levels read the 4-bit copy decodes what greedy decoding
    does, over a prompt and an output that fill record after record: draft,
    appended levels, verify, acceptance, commit and the next pack.  As in
    tests/test_gpu_dytc.py, another token is excused only where the oracle's
    top-1/top-2 margin is at most 0.05."""
    shape = synth.ModelShape("gqa_small", 4, 256, 4, 2, 64, 688, 512, 5e5, 1e-6, "bf16")
    w = synth.gen_weights(shape, seed=0)
    prompt = [int(x) for x in synth.gen_prompt(shape.vocab, 25, seed=1)] * 4
    n_new = 72
    ref = O.ar_decode(O.OracleModel(shape, w, max_ctx=256), prompt, n_new)
    g = cas.Model(shape, max_ctx=256, max_tree=64)
    g.load_weights(w)
    g.build_int8()
    g.build_int4()
    g.build_kv4()
    q3 = tuple(1 if l % 4 == 3 else 0 for l in range(shape.n_layers))
    odd = tuple(l % 2 for l in range(shape.n_layers))
    levels = [dytc.DraftConfig("kv4", kv4=True)] if full else []
    levels += [dytc.DraftConfig("q3", q3, kv4=True), dytc.DraftConfig("odd", odd, kv4=True, window=(4, 64)),
               dytc.DraftConfig("odd_i8", odd, 1, kv4=True), dytc.DraftConfig("odd_i4", odd, 2, kv4=True)]
    pld = dytc.DraftConfig("pld", pld=True)
    alpha = {"kv4": 0.95, "q3": 0.9, "odd": 0.8, "odd_i8": 0.75, "odd_i4": 0.72, "pld": 0.05}
    cost = {"kv4": 0.2, "q3": 0.3, "odd": 0.2, "odd_i8": 0.18, "odd_i4": 0.15, "pld": 0.01}
    params = dytc.DytcParams(max_tree=24, k_max=3, t_min=1.1, top_k=3, top_p=0.5)
    out, stats = [], {}
    while len(out) < n_new:
        seg = dytc.cas_decode_dytc(dytc.LibraryBackend(g), prompt + out, n_new - len(out), levels + [pld], pld,
                                   dytc.AcceptanceEstimator(dict(alpha)), cost, params, shape.n_layers, stats)
        i = next((k for k, (a, b) in enumerate(zip(seg, ref[len(out):])) if a != b), None)
        if i is None:
            out += seg
            break
        pos = len(out) + i
        seq = prompt + ref[:pos]
        m = O.OracleModel(shape, w, max_ctx=256)
        m.prefill(seq[:-1])
        lg = np.sort(m.forward([seq[-1]], [-1])[0])
        assert lg[-1] - lg[-2] <= 0.05, f"divergence at token {pos}, oracle margin {lg[-1] - lg[-2]}"
        out = ref[: pos + 1]
    assert out[:n_new] == ref
    assert sum(n for c, n in stats["expansions"].items() if c != "pld") > 0
    if full:  # drafted tokens were committed too
        assert sum(stats["accepted"]) > 0
    g.close()

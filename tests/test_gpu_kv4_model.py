"""Drafts over the 4-bit copy of the KV cache (Model.forward(..., kv4=True)).

Reference: a model whose cache holds, in the committed whole records, the
values that the copy stands for (their 64-bit definition, kv4_ref), and the
same elsewhere.  The two differ by the rounding of the attention's
probabilities only; per row, max |a - b| <= 2e-2 max |b|, the bar of bf16
decoders against the oracle.
"""
import numpy as np
import pytest

from paper_2510_26843_amd import cas, dytc, latency, synth
from tests import kv4_ref as R

pytestmark = pytest.mark.gpu

GQA = synth.ModelShape("gqa_small", 2, 512, 8, 2, 64, 1376, 1024, 5e5, 1e-6, "bf16")
MHA = synth.ModelShape("mha_small", 2, 1024, 8, 8, 128, 2752, 4096, 1e4, 1e-6, "bf16")
TOL = 2e-2


@pytest.fixture(scope="module")
def weights():
    return {s.name: synth.gen_weights(s, seed=9) for s in (GQA, MHA)}


def _model(shape, w, prompt, kv4=True, quant=True, max_ctx=1024):
    m = cas.Model(shape, max_ctx=max_ctx, max_tree=128)
    m.load_weights(w)
    if quant:
        m.build_int8()
        m.build_int4()
    if kv4:
        m.build_kv4()
    if len(prompt):
        m.prefill(prompt)
    return m


def _held(bits):
    """bf16 bits of the values that a 4-bit copy of these keys or values stands for."""
    x = synth.bf16_bits_to_f32(bits).astype(np.float64)
    return synth.f32_to_bf16_bits(R.values(*R.quantise(x)).astype(np.float32))


def _reference(shape, w, m):
    """A model with m's cache, its committed whole records as the copy has them."""
    ref = _model(shape, w, [], kv4=False)
    n = m.committed
    for l in range(shape.n_layers):
        k, v = m.kv_read(l, n)
        c = n // 32 * 32
        k[:, :c], v[:, :c] = _held(k[:, :c]), _held(v[:, :c])
        ref.kv_load(l, k, v)
    ref.set_committed(n)
    return ref


def _row_err(got, ref):
    return float((np.abs(got - ref).max(axis=1) / np.abs(ref).max(axis=1)).max())


def _tree(shape, n, seed=2):
    parents = synth.balanced_tree(n)
    return synth.gen_tree_tokens(parents, shape.vocab, seed=seed), parents


def _prompt(shape, n, seed=1):
    return [int(x) for x in synth.gen_prompt(shape.vocab, n, seed=seed)]


@pytest.mark.parametrize("shape", [GQA, MHA], ids=lambda s: s.name)
@pytest.mark.parametrize("plen,T", [(32, 1), (31, 3), (300, 1), (300, 2), (319, 32), (640, 64), (64, 128)])
@pytest.mark.parametrize("opts", [{}, {"skip": [0, 1]}, {"attn_window": (4, 100)}], ids=["full", "skip", "window"])
def test_draft_parity(weights, shape, plen, T, opts):
    m = _model(shape, weights[shape.name], _prompt(shape, plen))
    ref = _reference(shape, weights[shape.name], m)
    toks, parents = _tree(shape, T)
    got = m.forward(toks, parents, kv4=True, **opts)
    want = ref.forward(toks, parents, **opts)
    err = _row_err(got, want)
    assert err < TOL, err
    if plen >= 64:  # the quantisation of the cache moves the logits by more than that rounding
        assert _row_err(m.forward(toks, parents, **opts), want) > 2 * err
    m.close()
    ref.close()


@pytest.mark.parametrize("T", [1, 5, 33])
def test_int8_activations_with_4_bit_kv(weights, T):
    """The merge's codes for the O projection, at one node (quantised on load)
    and more (written by the merge).  An integer code turns a rounding of the
    attention into a whole step: 6e-2 (tests/test_gpu_forward.py)."""
    shape = MHA
    m = _model(shape, weights[shape.name], _prompt(shape, 64))
    ref = _reference(shape, weights[shape.name], m)
    toks, parents = _tree(shape, T)
    err = _row_err(m.forward(toks, parents, act_quant=1, kv4=True), ref.forward(toks, parents, act_quant=1))
    assert err < 6e-2, err
    m.close()
    ref.close()


@pytest.mark.parametrize("shape", [GQA, MHA], ids=lambda s: s.name)
@pytest.mark.parametrize("aq", [0, 1, 2])
def test_quantised_activations_where_the_attention_is_exact(weights, shape, aq):
    """One node and no context: its only probability is 1, so the attention
    gives its value whatever the kernel, and the draft the plain draft's bits.
    (Over a context two kernels' outputs differ by roundings, and no bound
    follows for int4: each may move a code by its step, amax / 7, and the
    codes of a row that move are not bounded below all of them.)"""
    m = _model(shape, weights[shape.name], [])
    a = m.forward([7], [-1], act_quant=aq, kv4=True)
    b = m.forward([7], [-1], act_quant=aq)
    assert np.array_equal(_bits(a), _bits(b))
    # ... and over a context the same bits each time
    m.prefill(_prompt(shape, 100))
    toks, parents = _tree(shape, 5)
    a = m.forward(toks, parents, act_quant=aq, kv4=True)
    assert np.isfinite(a).all() and np.array_equal(_bits(a), _bits(m.forward(toks, parents, act_quant=aq, kv4=True)))
    m.close()


def _bits(a):
    return a.view(np.uint32)


def test_the_copy_follows_the_cache(weights):
    """After commits, roll-backs and reloads a draft gives the bits that a
    model gives which packs that cache for the first time."""
    shape, w = GQA, weights["gqa_small"]
    m = _model(shape, w, _prompt(shape, 90))
    toks, parents = _tree(shape, 7)

    def fresh():
        f = _model(shape, w, [])
        n = m.committed
        for l in range(shape.n_layers):
            f.kv_load(l, *m.kv_read(l, n))
        f.set_committed(n)
        out = f.forward(toks, parents, kv4=True)
        f.close()
        return out

    def check(what):
        assert np.array_equal(_bits(m.forward(toks, parents, kv4=True)), _bits(fresh())), what

    check("first")
    for i in range(12):  # verify, accept a path, commit: record after record fills
        t, p = _tree(shape, 9, seed=40 + i)
        m.forward(t, p, logits=False)
        path = [8]
        while p[path[0]] >= 0:
            path.insert(0, p[path[0]])
        m.compact(path)
        check(("commit", i, m.committed))
    m.set_committed(50)
    check("rolled back")
    m.prefill(_prompt(shape, 200, seed=5))
    check("other tokens")
    m.set_committed(40)
    m.prefill(_prompt(shape, 30, seed=6))
    check("other tokens in a packed record")
    k, v = m.kv_read(1, m.committed)
    m.kv_load(1, v, k)
    check("reloaded")
    m.set_committed(0)
    m.forward([3], [-1], kv4=True)
    m.close()


@pytest.mark.parametrize("heads,kv_heads,hd", [(40, 8, 128), (64, 8, 64)])
@pytest.mark.parametrize("opts", [{}, {"attn_window": (40, 100)}], ids=["full", "window"])
def test_many_heads_and_a_wide_tree(heads, kv_heads, hd, opts):
    """More tiles of query rows than the card has places: workgroups of two."""
    shape = synth.ModelShape("many_heads", 1, 512, heads, kv_heads, hd, 1376, 1024, 1e4, 1e-6, "bf16")
    w = synth.gen_weights(shape, seed=9)
    m = _model(shape, w, _prompt(shape, 330), quant=False)
    ref = _model(shape, w, [], kv4=False, quant=False)
    k, v = m.kv_read(0, 330)
    k[:, :320], v[:, :320] = _held(k[:, :320]), _held(v[:, :320])
    ref.kv_load(0, k, v)
    ref.set_committed(330)
    toks, parents = _tree(shape, 128)
    err = _row_err(m.forward(toks, parents, kv4=True, **opts), ref.forward(toks, parents, **opts))
    assert err < TOL, err
    m.close()
    ref.close()


def test_graphs_and_direct_launches_give_the_same_bits(weights):
    shape = GQA
    m = _model(shape, weights["gqa_small"], _prompt(shape, 333))
    for T in (1, 2, 3, 17, 64):
        toks, parents = _tree(shape, T)
        a = m.forward(toks, parents, kv4=True, attn_window=(4, 64))
        b = m.forward(toks, parents, kv4=True, attn_window=(4, 64))
        m.set_graphs(False)
        c = m.forward(toks, parents, kv4=True, attn_window=(4, 64))
        m.set_graphs(True)
        assert np.array_equal(_bits(a), _bits(b)) and np.array_equal(_bits(a), _bits(c)), T
    m.close()


def test_profiled_and_gemv_calls(weights):
    """Launches timed one by one give the same bits, and the one-row tiles of
    cas_set_gemv a result within the bar."""
    shape = MHA
    m = _model(shape, weights["mha_small"], _prompt(shape, 200), quant=False)
    a = m.forward([5], [-1], kv4=True)
    m.profile(True)
    b = m.forward([5], [-1], kv4=True)
    m.profile(False)
    assert np.array_equal(_bits(a), _bits(b))
    m.set_gemv(True)
    assert _row_err(m.forward([5], [-1], kv4=True), a) < TOL
    m.set_gemv(False)
    assert np.array_equal(_bits(a), _bits(m.forward([5], [-1], kv4=True)))
    m.close()


def test_the_target_is_untouched(weights):
    """A 4-bit draft is no verify call, and verify calls around it keep their bits."""
    shape = MHA
    m = _model(shape, weights["mha_small"], _prompt(shape, 200))
    toks, parents = _tree(shape, 16)
    before = m.forward(toks, parents)
    path = m.accept()
    m.forward(toks, parents, kv4=True, logits=False)
    with pytest.raises(cas.CasError, match="CAS_ERR_STATE"):
        m.accept()
    with pytest.raises(cas.CasError, match="CAS_ERR_STATE"):
        m.compact(path[0])
    assert np.array_equal(_bits(m.forward(toks, parents)), _bits(before)) and m.accept() == path
    m.close()


def test_appended_levels(weights):
    """A round's levels drafted one after another over the copy: the last
    level's logits are those of the whole tree in one call."""
    shape = MHA
    m = _model(shape, weights["mha_small"], _prompt(shape, 150))
    toks, parents = _tree(shape, 15)
    whole = m.forward(toks, parents, kv4=True)
    m.forward(toks[:3], parents[:3], 0, kv4=True, logits=False)
    m.forward(toks[3:7], parents[3:7], 3, kv4=True, logits=False)
    last = m.forward(toks[7:], parents[7:], 7, kv4=True)
    assert _row_err(last, whole[7:]) < TOL
    m.close()


def test_refusals(weights):
    m = _model(GQA, weights["gqa_small"], _prompt(GQA, 40), kv4=False)
    with pytest.raises(cas.CasError, match="CAS_ERR_STATE"):
        m.forward([1], [-1], kv4=True)
    m.build_kv4()
    m.build_kv4()
    with pytest.raises(cas.CasError, match="CAS_ERR_ARG"):
        m.forward([1], [-1], kv4=True, attn_window=(0, -1))
    with pytest.raises(cas.CasError, match="CAS_ERR_TREE"):
        m.forward([1], [0], kv4=True)
    m.close()
    tiny = synth.SHAPES["tiny"]
    f = cas.Model(tiny, max_ctx=256)
    with pytest.raises(cas.CasError, match="CAS_ERR_UNSUPPORTED"):
        f.build_kv4()
    f.close()


def test_device_checks(weights):
    """The build with device checks: none fails in a round over the copy, and
    one that does (slots past a limit set for the test) is reported."""
    shape = GQA
    m = cas.Model(shape, max_ctx=512, max_tree=64, debug=True)
    m.load_weights(weights["gqa_small"])
    m.build_kv4()
    m.prefill(_prompt(shape, 150))
    toks, parents = _tree(shape, 20)
    a = m.forward(toks, parents, kv4=True)
    assert np.isfinite(a).all() and m.debug_check() == 0
    m.debug_limit_slots(160)
    m.forward(toks, parents, kv4=True, logits=False)
    assert m.debug_check() != 0
    m.debug_limit_slots(0)
    assert np.array_equal(_bits(m.forward(toks, parents, kv4=True)), _bits(a)) and m.debug_check() == 0
    m.close()


def test_small_cache_and_many_splits(weights):
    """A model whose partial-state buffer is small (a short cache, a small
    tree): a call takes no more splits than it holds."""
    shape = GQA
    m = cas.Model(shape, max_ctx=128, max_tree=2)
    m.load_weights(weights["gqa_small"])
    m.build_kv4()
    m.prefill(_prompt(shape, 120))
    ref = cas.Model(shape, max_ctx=128, max_tree=2)
    ref.load_weights(weights["gqa_small"])
    for l in range(shape.n_layers):
        k, v = m.kv_read(l, 120)
        k[:, :96], v[:, :96] = _held(k[:, :96]), _held(v[:, :96])
        ref.kv_load(l, k, v)
    ref.set_committed(120)
    for T in (1, 2):
        toks, parents = _tree(shape, T)
        assert _row_err(m.forward(toks, parents, kv4=True), ref.forward(toks, parents)) < TOL
    m.close()
    ref.close()


def test_dytc_and_the_latency_table_take_4_bit_drafts(weights):
    """A cascade with a 4-bit draft decodes the tokens of one without drafts
    (greedy verification is lossless whatever the draft)."""
    shape = GQA
    odd = tuple(l % 2 for l in range(shape.n_layers))
    prompt = _prompt(shape, 70)
    m = _model(shape, weights["gqa_small"], [])
    backend = dytc.LibraryBackend(m)
    backend.reset(prompt)
    ids, probs = backend.draft([prompt[-1]], [-1], 0, dytc.DraftConfig("odd_kv4", odd, kv4=True), 4)
    assert ids.shape == (1, 4) and (probs > 0).all()
    plain, _ = backend.draft([prompt[-1]], [-1], 0, dytc.DraftConfig("odd", odd), 4)
    assert len(set(ids[0]) & set(plain[0])) >= 1
    assert latency.parse_draft("odd+int4+kv4@4:64", 2) == ([0, 1], 2, (4, 64)) and latency.draft_kv4("odd+kv4@4:64")
    assert latency.parse_draft("odd+kv4+int4", 2) == ([0, 1], 2, None) and latency.draft_kv4("odd+kv4+int4")
    assert latency.parse_draft("odd", 2) == ([0, 1], 0, None) and not latency.draft_kv4("odd+int8@4:64")
    recs = latency.sweep(m, shape, [1, 4], [100, 640], ["odd", "odd+kv4", "none+int8+kv4@4:64"], reps=2)
    assert len(recs) == 2 * 2 * 4
    by = {(r["config"], r["T"], r["ctx"]): r["bytes"] for r in recs}
    assert by["odd+kv4", 1, 640] < by["odd", 1, 640]
    m.close()

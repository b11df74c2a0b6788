"""What the tensor calls of the paged KV cache and of the log probabilities make
of their tensors' types, sizes and strides, before anything is launched.  CPU:
the library notes the arguments that reach it, host tensors stand in for the
device's."""
import ctypes

import pytest
import torch

from paper_2510_26843_amd import cas

B, F, I, A = torch.bfloat16, torch.float32, torch.int32, torch.int64
HKV, HD, PAGE, H, N, SEQS = 2, 64, 64, 4, 5, 3


@pytest.fixture
def calls(monkeypatch):
    seen = []

    class Lib:
        def __getattr__(self, name):
            if name.endswith("_work_bytes"):
                return lambda *a: 0
            return lambda *a: seen.append(a) or 0

    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)  # (what a host tensor's get_device says)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: 0, raising=False)
    monkeypatch.setattr(cas, "lib", lambda debug=False: Lib())
    monkeypatch.setattr(cas, "_work", lambda n, stream=None: torch.zeros(16, dtype=torch.uint8))
    return seen


def _z(*shape, dtype=B):
    return torch.zeros(shape, dtype=dtype)


def _cache(**kw):
    a = dict(pages=_z(7, 2, HKV, PAGE * HD), page_size=PAGE, hd=HD, table=_z(SEQS, 4, dtype=I), seq_start=_z(SEQS + 1, dtype=I),
             ctx_len=_z(SEQS, dtype=I), n_rows=N)
    a.update(kw)
    return cas.Paged(**a)


def test_cache_numbers(calls):
    pages, table = _z(7, 2, HKV, PAGE * HD), _z(SEQS, 4, dtype=I)
    c = _cache(pages=pages, table=table, max_rows=3, nodes=_z(SEQS, dtype=I))
    assert (c.pages, c.n_pages, c.page_size, c.n_kv_heads, c.head_dim) == (pages.data_ptr(), 7, PAGE, HKV, HD)
    assert (c.table, c.table_len, c.n_seqs, c.n_rows, c.max_rows) == (table.data_ptr(), 4, SEQS, N, 3) and c.nodes
    assert _cache().nodes is None
    assert ctypes.sizeof(c) == 72  # (the C struct's)


@pytest.mark.parametrize("change,name", [
    (dict(pages=_z(7, 2, HKV, PAGE * HD, dtype=F)), "pages"), (dict(pages=_z(7, 2, HKV * 2, PAGE * HD)[:, :, ::2]), "pages"),
    (dict(pages=_z(7, HKV, PAGE * HD)), "pages"), (dict(pages=_z(7, 1, HKV, PAGE * HD)), "pages"),
    (dict(pages=_z(7, 2, HKV, 32 * HD)), "pages"), (dict(table=_z(SEQS, 4, dtype=A)), "table"), (dict(table=_z(4, dtype=I)), "table"),
    (dict(table=_z(SEQS, 8, dtype=I)[:, :4]), "table"), (dict(seq_start=_z(SEQS, dtype=I)), "seq_start"),
    (dict(seq_start=_z(SEQS + 1, dtype=A)), "seq_start"), (dict(ctx_len=_z(SEQS - 1, dtype=I)), "ctx_len"),
    (dict(ctx_len=_z(2 * SEQS, dtype=I)[::2]), "ctx_len"), (dict(nodes=_z(SEQS, dtype=F)), "nodes")])
def test_cache_refuses(calls, change, name):
    with pytest.raises(cas.CasError, match=rf"CAS_ERR_ARG.*: {name} "):
        _cache(**change)


WIDE = (H + 2 * HKV) * HD


def _append(**kw):
    a = dict(k=_z(N, HKV * HD), v=_z(N, HKV * HD), q=_z(N, H * HD), q_out=_z(N, H, HD), pos=_z(N, dtype=I),
             cos=_z(50, HD // 2, dtype=F), sin=_z(50, HD // 2, dtype=F))
    a.update(kw)
    cas.op_paged_append(_cache(), a.pop("k"), a.pop("v"), **a)


FUSED = _z(N, WIDE)


@pytest.mark.parametrize("change,lds", [
    ({}, (H * HD, HKV * HD, HKV * HD)),
    (dict(q=FUSED[:, : H * HD], k=FUSED[:, H * HD : (H + HKV) * HD], v=FUSED[:, (H + HKV) * HD :]), (WIDE, WIDE, WIDE)),
    (dict(q=_z(N, H, HD), k=_z(N, HKV, HD), v=_z(N + 1, HKV * HD)), (H * HD, HKV * HD, HKV * HD)),
    (dict(q=_z(N, H, HD), k=_z(N, 6, HD)[:, 2:4]), (H * HD, 6 * HD, HKV * HD)),
    (dict(k=_z(N, HKV * HD, dtype=torch.int16)), (H * HD, HKV * HD, HKV * HD)),
    (dict(q=None, q_out=None), (0, HKV * HD, HKV * HD)), (dict(cos=None, sin=None, pos=None), (H * HD, HKV * HD, HKV * HD))])
def test_append_takes(calls, change, lds):
    _append(**change)
    assert len(calls) == 1 and (calls[0][2], calls[0][5], calls[0][7]) == lds
    assert calls[0][3] == (H if lds[0] else 0)


@pytest.mark.parametrize("change,name", [
    (dict(k=_z(N, HKV * HD, dtype=F)), "k"), (dict(k=_z(N - 1, HKV * HD)), "k"), (dict(v=_z(N, 2 * HKV * HD)[:, ::2]), "v"),
    (dict(v=_z(HKV * HD, N).t()), "v"), (dict(q=_z(N - 1, H * HD)), "q"), (dict(q=_z(N, H * HD, dtype=torch.float16)), "q"),
    (dict(q_out=_z(N, H * HD)), "q_out"), (dict(q_out=_z(N - 1, H, HD)), "q_out"), (dict(q_out=_z(N, H, 2 * HD)[..., :HD]), "q_out"),
    (dict(q_out=_z(N, H, HD, dtype=F)), "q_out"), (dict(pos=_z(N, dtype=A)), "pos"), (dict(pos=_z(N - 1, dtype=I)), "pos"),
    (dict(cos=_z(50, HD, dtype=F)), "cos"), (dict(cos=_z(50, HD // 2)), "cos"), (dict(sin=_z(49, HD // 2, dtype=F)), "sin"),
    (dict(sin=_z(50, HD, dtype=F)[:, ::2]), "sin")])
def test_append_refuses(calls, change, name):
    with pytest.raises(cas.CasError, match=rf"CAS_ERR_ARG.*: {name} "):
        _append(**change)
    assert not calls


def _attend(**kw):
    a = dict(q=_z(N, H, HD), out=_z(N, H * HD), anc=_z(N, 2, dtype=A))
    a.update(kw)
    cas.op_attention_paged(_cache(), a.pop("q"), a.pop("out"), **a)


@pytest.mark.parametrize("change", [{}, dict(anc=None), dict(q=_z(N + 2, H, HD)), dict(out=_z(N, H, HD), sink=4, window=9),
                                    dict(q=_z(N, H, HD, dtype=torch.int16)), dict(anc=_z(2 * N, dtype=A))])
def test_attention_takes(calls, change):
    _attend(**change)
    assert len(calls) == 1 and calls[0][2] == H and calls[0][4:6] == (change.get("sink", 0), change.get("window", 0))


@pytest.mark.parametrize("change,name", [
    (dict(q=_z(N, H, HD, dtype=F)), "q"), (dict(q=_z(N - 1, H, HD)), "q"), (dict(q=_z(N, H * HD)), "q"),
    (dict(q=_z(H, N, HD).transpose(0, 1)), "q"), (dict(q=_z(N, H, 2 * HD)[..., ::2]), "q"), (dict(out=_z(N, H * HD, dtype=F)), "out"),
    (dict(out=_z(N, H * HD - 1)), "out"), (dict(out=_z(N, 2 * H * HD)[:, : H * HD]), "out"), (dict(anc=_z(N, 2, dtype=I)), "anc"),
    (dict(anc=_z(N, dtype=A)), "anc"), (dict(anc=_z(N, 4, dtype=A)[:, :2]), "anc")])
def test_attention_refuses(calls, change, name):
    with pytest.raises(cas.CasError, match=rf"CAS_ERR_ARG.*: {name} "):
        _attend(**change)
    assert not calls


ROWS, V = 3, 100


def _score(**kw):
    a = dict(logits=_z(ROWS, V, dtype=F), tokens=_z(ROWS, 2, dtype=I), logp=_z(ROWS, 2, dtype=F), entropy=_z(ROWS, dtype=F),
             top_ids=_z(ROWS, 4, dtype=I), top_logp=_z(ROWS, 4, dtype=F))
    a.update(kw)
    cas.op_logprobs(**a)


@pytest.mark.parametrize("change,lt,ld,m,K", [
    ({}, 0, V, 2, 4), (dict(logits=_z(ROWS, V)), 1, V, 2, 4), (dict(logits=_z(ROWS, 2 * V, dtype=F)[:, V:]), 0, 2 * V, 2, 4),
    (dict(tokens=None, logp=None), 0, V, 0, 4), (dict(top_ids=None, top_logp=None, entropy=None), 0, V, 2, 0),
    (dict(tokens=_z(ROWS, dtype=I), logp=_z(ROWS, dtype=F)), 0, V, 1, 4), (dict(logits=_z(ROWS, V, dtype=torch.int16)), 1, V, 2, 4),
    (dict(top_ids=_z(ROWS, 0, dtype=I), top_logp=_z(ROWS, 0, dtype=F)), 0, V, 2, 0)])
def test_logprobs_takes(calls, change, lt, ld, m, K):
    _score(**change)
    assert len(calls) == 1
    c = calls[0]
    assert (c[0], c[2], c[3], c[4], c[7], c[10]) == (lt, ld, ROWS, V, m, K)


@pytest.mark.parametrize("change,name", [
    (dict(logits=_z(ROWS * V, dtype=F)), "logits"), (dict(logits=_z(ROWS, V, dtype=torch.float16)), "logits"),
    (dict(logits=_z(ROWS, 2 * V, dtype=F)[:, ::2]), "logits"), (dict(logits=_z(V, ROWS, dtype=F).t()), "logits"),
    (dict(tokens=_z(ROWS, 2, dtype=A)), "tokens"), (dict(tokens=_z(ROWS, 4, dtype=I)[:, ::2]), "tokens"),
    (dict(logp=_z(ROWS, 1, dtype=F)), "logp"), (dict(logp=_z(ROWS, 2)), "logp"), (dict(entropy=_z(ROWS - 1, dtype=F)), "entropy"),
    (dict(top_ids=_z(ROWS, 4, dtype=A)), "top_ids"), (dict(tokens=_z(ROWS + 1, dtype=I)), "tokens"),
    (dict(top_ids=_z(2 * ROWS - 1, dtype=I)), "tokens and top_ids"), (dict(top_logp=_z(ROWS, 3, dtype=F)), "top_logp")])
def test_logprobs_refuses(calls, change, name):
    with pytest.raises(cas.CasError, match=rf"CAS_ERR_ARG.*: {name} "):
        _score(**change)
    assert not calls


def test_another_device(calls, monkeypatch):
    cache = _cache()
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(cas, "Paged", lambda **kw: cache)
    for call in (_append, _attend, _score):
        with pytest.raises(cas.CasError, match="not on the current device"):
            call()
    monkeypatch.undo()
    assert not calls


def test_a_batch_keeps_its_tensors(calls):
    c = _cache()
    assert len(c.tensors) == 5 and c.tensors[0].data_ptr() == c.pages


@pytest.mark.parametrize("vocab", [1, 1000, 8193, 32000, 128256, 1 << 20])
def test_logprob_work_serves_fewer_rows(vocab):
    """Scratch for n rows and K serves any call of fewer: the parts of a row go with the rows."""
    f = cas.lib().cas_op_logprobs_work_bytes
    sizes = [f(n, vocab, 32) for n in range(1, 700)]
    assert sizes == sorted(sizes) and sizes[0] >= 16
    assert all(f(n, vocab, K) <= f(n, vocab, 32) for n in (1, 33, 257) for K in (0, 1, 8))


class _Elsewhere:
    """A tensor that says it lies on device 0."""

    def __init__(self, t):
        self.t = t

    def get_device(self):
        return 0

    def __getattr__(self, name):
        return getattr(self.t, name)


@pytest.mark.parametrize("call", [_append, _attend])
def test_a_batch_of_another_device(calls, monkeypatch, call):
    """Made where device 0 is current, used with rows of another one that is current then."""
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    cache = cas.Paged(*(_Elsewhere(x) if isinstance(x, torch.Tensor) else x for x in (
        _z(7, 2, HKV, PAGE * HD), PAGE, HD, _z(SEQS, 4, dtype=I), _z(SEQS + 1, dtype=I), _z(SEQS, dtype=I), N)))
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    monkeypatch.setattr(cas, "Paged", lambda **kw: cache)
    with pytest.raises(cas.CasError, match="CAS_ERR_ARG.*not on the current device"):
        call()
    assert not calls


@pytest.mark.parametrize("scale,status", [(2.4e38, cas.ERR_ARG), (3.4e38, cas.ERR_ARG), (float("inf"), cas.ERR_ARG)])
def test_scales_whose_exponents_overflow(scale, status):
    """In log2 units the scale is 1.44 times itself, which fp32 has to hold."""
    p = 4096  # (an address that a refused call does not look at)
    assert cas.lib().cas_op_logprobs(cas.W_F32, p, 100, 1, 100, scale, None, 0, None, p, 0, None, None, p, 1 << 20, None) == status

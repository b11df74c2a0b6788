"""The scratch that a kernel-level call takes for itself belongs to the stream
that the call runs on.  From another stream's memory it would go back to that
stream when the call returns, and be written by its next work while the call's
kernels still use it.  CPU: the library and torch's streams are stand-ins that
note on which stream an allocation happens.  GPU: two streams at once."""
import contextlib
import types

import numpy as np
import pytest
import torch

from paper_2510_26843_amd import cas

CURRENT = 64


@pytest.fixture
def allocations(monkeypatch):
    """(stream of each scratch allocation, stream of each call)"""
    allocs, calls, now = [], [], [CURRENT]
    empty = torch.empty

    @contextlib.contextmanager
    def under(s):
        now.append(s.cuda_stream)
        yield
        now.pop()

    def fake_empty(*a, device=None, **kw):
        assert device == "cuda"
        allocs.append(now[-1])
        return empty(*a, **kw)

    class Lib:
        def __getattr__(self, name):
            if name.endswith("_work_bytes"):
                return lambda *a: 256
            return lambda *a: calls.append(a[-1]) or 0

    handle = lambda s=0: types.SimpleNamespace(cuda_stream=s)  # noqa: E731
    monkeypatch.setattr(torch, "empty", fake_empty)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)  # (what a host tensor's get_device says)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda dev: now[-1], raising=False)
    monkeypatch.setattr(torch.cuda, "stream", under)
    monkeypatch.setattr(torch.cuda, "ExternalStream", handle)
    monkeypatch.setattr(torch.cuda, "default_stream", handle)
    monkeypatch.setattr(cas, "lib", lambda debug=False: Lib())
    return allocs, calls


def _calls():
    x = torch.zeros(4096, dtype=torch.bfloat16)
    b = torch.zeros(4096, dtype=torch.uint8)
    anc = torch.zeros(2, dtype=torch.int64)
    return {
        "gemm": lambda **kw: cas.op_gemm(cas.W_BF16, x, x, 16, 64, 1, x, 16, **kw),
        "quant_weight": lambda **kw: cas.op_quant_weight(cas.W_BF16, x, 16, 64, b, x, **kw),
        "attention": lambda **kw: cas.op_attention(x, x, x, 32, 10, 1, 1, 1, 1, 64, anc, x, **kw),
        "rmsnorm": lambda **kw: cas.op_rmsnorm(cas.W_BF16, x, x, 1, 64, 1e-6, out=x, **kw),
        "attn_merge": lambda **kw: cas.op_attn_merge(x, x, 1, 1, 1, 64, out=x, **kw),
        "gemm_qx": lambda **kw: cas.op_gemm_qx(cas.W_I8, b, x, x, 16, 64, 1, 127, x, **kw),
        "attention_kv4": lambda **kw: cas.op_attention_kv4(x, b, 32, 11, 10, 1, 1, 1, 1, 64, anc, x, **kw),
    }


@pytest.mark.parametrize("op", sorted(_calls()))
@pytest.mark.parametrize("stream", [None, CURRENT, 4096, 0])
def test_scratch_is_the_streams_own(allocations, op, stream):
    allocs, calls = allocations
    _calls()[op](stream=stream)
    assert calls == [CURRENT if stream is None else stream]
    assert allocs == calls


@pytest.mark.gpu
def test_two_streams_at_once():
    """A split attention on a stream that is still busy when the call returns,
    and work of the current stream in memory of the scratch's size meanwhile."""
    H, Hkv, hd, Lc = 8, 1, 128, 40001
    n = Lc + 1
    cap = (n + 31) // 32 * 32
    need = cas.lib().cas_op_attention_kv4_work_bytes(Lc, 1, 1, H, Hkv, hd, 0, 0)
    assert need > 0
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    rows = torch.randn((n, hd), generator=g, device="cuda").to(torch.bfloat16)
    rec = torch.zeros((Hkv, cap // 32, 34 * hd), dtype=torch.uint8, device="cuda")
    cas.op_kv4_append(rows, rows, n, Hkv, hd, rec, cap, 0)
    q = torch.randn((1, H, hd), generator=g, device="cuda").to(torch.bfloat16)
    anc = torch.from_numpy(np.array([[1, 0]], np.int64)).to("cuda")
    want, out = (torch.zeros((1, H * hd), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    args = (q, rec, cap, n, Lc, 1, 1, H, Hkv, hd, anc)
    cas.op_attention_kv4(*args, want)
    s = torch.cuda.Stream()
    big = torch.zeros(1 << 28, dtype=torch.float32, device="cuda")
    torch.cuda.synchronize()
    for _ in range(3):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            for _ in range(20):
                big.add_(1.0)  # (2 GB each way: the stream is busy for several ms)
        cas.op_attention_kv4(*args, out, stream=s.cuda_stream)
        theirs = [torch.full((need,), 255, dtype=torch.uint8, device="cuda") for _ in range(4)]
        torch.cuda.synchronize()
        assert torch.equal(out, want) and all(bool((t == 255).all()) for t in theirs)
        out.zero_()

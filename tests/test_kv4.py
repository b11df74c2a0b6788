"""CPU checks of the 4-bit KV cache: its size, what its calls refuse (before
any device work), and that the reference's form and byte order agree."""
import numpy as np
import pytest

from paper_2510_26843_amd import cas
from tests import kv4_ref as R

P = 0x10000  # a pointer that no refused call follows


@pytest.mark.parametrize("Hkv,hd,cap,want", [(1, 64, 32, 34 * 64), (8, 128, 4096, 8 * 128 * 34 * 128),
                                            (40, 128, 1 << 20, 40 * (1 << 15) * 34 * 128), (0, 64, 32, 0),
                                            (1, 96, 32, 0), (1, 64, 33, 0), (1, 64, 0, 0), (1, 64, 1 << 21, 0)])
def test_bytes(Hkv, hd, cap, want):
    assert cas.kv4_bytes(Hkv, hd, cap) == want


def test_reference_round_trip():
    r = np.random.default_rng(0)
    for hd in (64, 128):
        places = R._places(hd)
        nibbles = {(int(b), int(h)) for p, f in (places[:2], places[2:4]) for b, h in zip(p.ravel(), f.ravel())}
        scales = {int(b) for p in places[4:] for b in p.ravel()}
        assert nibbles == {(b, h) for b in range(32 * hd) for h in (0, 1)}
        assert scales == set(range(32 * hd, 34 * hd))
    x = R.bf16(r.normal(0, 3, (5, 64)))
    y = R.values(*R.quantise(x))
    amax = np.abs(x.reshape(5, 2, 32)).max(-1, keepdims=True)
    assert (np.abs(y - x).reshape(5, 2, 32) <= amax / 4).all()  # saturation: at most 2 of 8
    again = R.values(*R.quantise(y))
    assert np.array_equal(again, y)


APPEND = dict(k=P, v=P, ldk=512, ldv=512, T=3, slot0=0, pos=None, cos=None, sin=None, n_pos=0, Hkv=4, hd=128, kv4=P,
              cap=64)


@pytest.mark.parametrize("change,status", [
    (dict(k=None), cas.ERR_ARG), (dict(v=None), cas.ERR_ARG), (dict(kv4=None), cas.ERR_ARG),
    (dict(kv4=P + 8), cas.ERR_ARG), (dict(k=P + 1), cas.ERR_ARG), (dict(T=0), cas.ERR_ARG), (dict(T=-1), cas.ERR_ARG),
    (dict(slot0=-1), cas.ERR_ARG), (dict(slot0=62), cas.ERR_ARG), (dict(slot0=2**31 - 1), cas.ERR_ARG),
    (dict(T=2**31 - 1), cas.ERR_ARG), (dict(ldk=511), cas.ERR_ARG), (dict(ldv=0), cas.ERR_ARG),
    (dict(cos=P, n_pos=5), cas.ERR_ARG), (dict(cos=P, sin=P), cas.ERR_ARG), (dict(hd=96), cas.ERR_UNSUPPORTED),
    (dict(cap=48), cas.ERR_ARG), (dict(cap=1 << 21), cas.ERR_UNSUPPORTED), (dict(Hkv=0), cas.ERR_ARG)])
def test_append_refuses(change, status):
    a = {**APPEND, **change}
    assert cas.lib().cas_op_kv4_append(a["k"], a["v"], a["ldk"], a["ldv"], a["T"], a["slot0"], a["pos"], a["cos"],
                                       a["sin"], a["n_pos"], a["Hkv"], a["hd"], a["kv4"], a["cap"], None) == status


READ = dict(kv4=P, cap=64, slot0=3, n=9, Hkv=4, hd=64, k=P, v=P)


@pytest.mark.parametrize("change,status", [
    (dict(kv4=None), cas.ERR_ARG), (dict(k=None), cas.ERR_ARG), (dict(v=P + 2), cas.ERR_ARG), (dict(n=0), cas.ERR_ARG),
    (dict(n=62), cas.ERR_ARG), (dict(slot0=-1), cas.ERR_ARG), (dict(n=2**31 - 1), cas.ERR_ARG),
    (dict(hd=32), cas.ERR_UNSUPPORTED), (dict(cap=0), cas.ERR_ARG)])
def test_read_refuses(change, status):
    a = {**READ, **change}
    assert cas.lib().cas_op_kv4_read(a["kv4"], a["cap"], a["slot0"], a["n"], a["Hkv"], a["hd"], a["k"], a["v"],
                                     None) == status


ATTEND = dict(q=P, kv4=P, cap=65536, n4=32000, k=P, v=P, kv_cap=20, Lc=32008, n_tree=3, T=3, H=8, Hkv=2, hd=64,
              sink=0, window=0, anc=P, out=P, work=P, nbytes=1 << 30)


@pytest.mark.parametrize("change,status", [
    (dict(q=None), cas.ERR_ARG), (dict(kv4=None), cas.ERR_ARG), (dict(k=None), cas.ERR_ARG),
    (dict(v=None), cas.ERR_ARG), (dict(anc=None), cas.ERR_ARG), (dict(out=None), cas.ERR_ARG),
    (dict(work=None), cas.ERR_ARG), (dict(nbytes=16), cas.ERR_ARG), (dict(q=P + 8), cas.ERR_ARG),
    (dict(out=P + 2), cas.ERR_ARG), (dict(k=P + 2), cas.ERR_ARG), (dict(anc=P + 4), cas.ERR_ARG),
    (dict(kv4=P + 4), cas.ERR_ARG), (dict(work=P + 4), cas.ERR_ARG), (dict(n4=31), cas.ERR_ARG),
    (dict(n4=-32), cas.ERR_ARG), (dict(n4=32032), cas.ERR_ARG), (dict(kv_cap=10), cas.ERR_ARG),
    (dict(n4=32011, cap=32000), cas.ERR_ARG), (dict(T=0), cas.ERR_ARG), (dict(T=129), cas.ERR_ARG),
    (dict(n_tree=0), cas.ERR_ARG), (dict(n_tree=129), cas.ERR_ARG), (dict(Lc=-1), cas.ERR_ARG),
    (dict(Lc=2**31 - 1), cas.ERR_ARG), (dict(H=7), cas.ERR_ARG), (dict(H=4098), cas.ERR_ARG), (dict(Lc=1 << 20), cas.ERR_ARG),
    (dict(Hkv=0), cas.ERR_ARG),
    (dict(sink=-1), cas.ERR_ARG), (dict(window=-1), cas.ERR_ARG), (dict(hd=80), cas.ERR_UNSUPPORTED),
    (dict(cap=40), cas.ERR_ARG)])
def test_attention_refuses(change, status):
    a = {**ATTEND, **change}
    assert cas.lib().cas_op_attention_kv4(
        a["q"], a["kv4"], a["cap"], a["n4"], a["k"], a["v"], a["kv_cap"], a["Lc"], a["n_tree"], a["T"], a["H"],
        a["Hkv"], a["hd"], a["sink"], a["window"], a["anc"], a["out"], a["work"], a["nbytes"], None) == status


def test_work_bytes():
    assert cas.lib().cas_op_attention_kv4_work_bytes(40, 3, 0, 8, 2, 64, 0, 0) == 0
    assert cas.lib().cas_op_attention_kv4_work_bytes(40, 3, 3, 8, 2, 64, 0, 0) == 0  # one run of tiles: none
    need = cas.lib().cas_op_attention_kv4_work_bytes(100000, 3, 3, 8, 2, 64, 0, 0)
    assert need >= 2 * 3 * 8 * 66 * 4 and need % (3 * 8 * 66 * 4) == 0

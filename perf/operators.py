"""Timed workloads of the 4-bit KV cache: appending to it, reading it back and
attending over it.

The cache holds keys and values as microscaled 4-bit floats (the OCP MX form
with E2M1 elements): 32 consecutive elements of a token's head row share a
power-of-two scale 2^(b - 127), b = 127 + max(floor(log2 max|x|) - 2, -125),
and an element is the nearest of +-{0, 0.5, 1, 1.5, 2, 3, 4, 6} times it (ties
to the even code, values past 6 saturate).  It is one byte buffer,
[n_kv_heads][ctx_cap / 32] records of 34 * head_dim bytes for 32 slots each:

- keys, 16 * hd bytes, [2 s][4 g][4 i][4 j][hd/32 u][4 c]: byte c holds the
  elements d = g hd/4 + 8u + 2c (low four bits) and d + 1 of slot 8i + 4s + j;
- values, 16 * hd bytes, [hd/64 m][4 g][hd/32 b][w r][2 n][8 j], w = 512 / hd:
  a byte holds the elements d = 32b + w (4m + 2n) + r (low) and d + w of slot
  8g + j;
- key scales, hd bytes, [hd/32 b][4 i][4 j][2 s] (slot 8i + 4s + j);
- value scales, hd bytes, [hd/32 b][32 slots].

A case is one of the calls that a decoding program makes:

- "append": T tokens' keys and values, as the projections leave them, are
  rotated by their positions, quantised and written from slot `slot0` on, and
  read back as a program does that checks or hands on what it stored;
- "read": a range of slots as bf16 rows (a cache that is saved, or handed to
  a step that wants bf16);
- "attend": tree attention of T query rows over `ctx` committed slots and the
  round's nodes; the first `n4` slots come from the 4-bit cache, the others
  (the last committed ones and the tree) from bf16 rows.

Head layouts are those of the repository's shapes; keys and values are
N(0, 1.28^2) and queries N(0, 1).
"""
import math

import numpy as np
import torch

own = False

# heads, kv heads, head width, rotation base
LAYOUTS = {
    "gqa_small": (8, 2, 64, 5e5),
    "llama2_7b": (32, 32, 128, 1e4),
    "llama2_13b": (40, 40, 128, 1e4),
    "llama3_8b": (32, 8, 128, 5e5),
}


def _append(name, layout, T, slot0, rotate=True, fused=False, tree=False):
    return {"name": name, "kind": "append", "layout": layout, "T": T, "slot0": slot0, "rotate": rotate,
            "fused": fused, "tree": tree}


def _read(name, layout, n, slot0):
    return {"name": name, "kind": "read", "layout": layout, "T": n, "slot0": slot0}


def _attend(name, layout, T, ctx, extra=0, tail=False, sink=0, window=0):
    """extra: nodes of the round before this call's T; tail: the slots past
    the last whole 32 committed ones are bf16 rows."""
    return {"name": name, "kind": "attend", "layout": layout, "T": T, "ctx": ctx, "extra": extra, "tail": tail,
            "sink": sink, "window": window}


def listed():
    return [
        # the key and value of one decoded token of the grouped-query shape
        _append("append one token", "llama3_8b", 1, 4095),
        # a verified tree of an odd size, straight from the fused projection's
        # rows, positions by depth, starting inside a record
        _append("append tree rows", "llama2_7b", 61, 2047, fused=True, tree=True),
        # a long prompt
        _append("append prompt", "llama3_8b", 16384, 0),
        # a few slots of a small decoder, from inside a record to inside another
        _read("read few slots", "gqa_small", 45, 1000),
        # a whole multi-head cache but for its last slots
        _read("read cache", "llama2_7b", 8190, 0),
        # the smallest call: one row of the small decoder after a short prompt
        _attend("attend small", "gqa_small", 1, 33),
        # plain decoding at 4096 slots
        _attend("attend decode 4096", "llama3_8b", 1, 4095),
        # the benchmark's tree width over a long multi-head cache whose last slots are bf16
        _attend("attend tree 32 at 8190", "llama2_7b", 32, 8190, tail=True),
        # the 13B tree
        _attend("attend tree 64 at 2048", "llama2_13b", 64, 2048),
        # a draft leaf with its siblings, sink and window, bf16 tail
        _attend("attend window", "llama2_7b", 3, 8190, extra=9, tail=True, sink=4, window=1024),
        # the widest tree at the longest context of the decoder
        _attend("attend tree 128 at 16001", "llama3_8b", 128, 16001),
        # one row over a very long cache
        _attend("attend decode 131072", "llama3_8b", 1, 131071),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def draw(rng):
    layout = rng.choice(sorted(LAYOUTS))
    hkv = LAYOUTS[layout][1]
    most = 16384 * 8 // hkv  # slots of an append or a read: no more bytes than the long prompt's
    kind = rng.choice(["append", "read", "attend", "attend"])
    if kind == "append":
        tree = rng.random() < 0.4
        T = _log_int(rng, 1, 128 if tree else min(most, 16384))
        return _append("", layout, T, rng.choice([0, rng.randrange(4096)]), rng.random() < 0.8, rng.random() < 0.5, tree)
    if kind == "read":
        return _read("", layout, _log_int(rng, 1, min(most, 16384)), rng.choice([0, rng.randrange(4096)]))
    T = _log_int(rng, 1, 128)
    # long contexts for few rows of few heads
    hi = 131071 if T <= 4 and hkv <= 8 else 16128 if hkv <= 8 or T <= 8 else 4096
    ctx = _log_int(rng, 1, hi)
    window = rng.choice([0, 0, 0, 256, 1024])
    return _attend("", layout, T, ctx, rng.choice([0, rng.randrange(0, 129 - T)]), rng.random() < 0.5,
                   4 if window else 0, window)


# ----------------------------------------------------------------------------
# inputs
# ----------------------------------------------------------------------------

def _cap(slots):
    return (slots + 31) // 32 * 32


def _n4(case):
    n = case["ctx"] + case["extra"] + case["T"]
    return case["ctx"] // 32 * 32 if case["tail"] else n


def _parents(n, seed):
    """A random tree, every parent before its children, mostly growing at its latest nodes."""
    r = np.random.default_rng([seed, n])
    return [-1] + [int(max(0, i - 1 - int(r.exponential(3.0)))) for i in range(1, n)]


def _depths_masks(parents):
    depth, masks = [], []
    for i, p in enumerate(parents):
        depth.append(depth[p] + 1 if p >= 0 else 0)
        masks.append((masks[p] if p >= 0 else 0) | (1 << i))
    words = np.array([[m & (2**64 - 1), m >> 64] for m in masks], dtype=np.uint64)
    return depth, words


def _normal(g, *shape, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(torch.bfloat16)


def _filled(g, layout, slots):
    """A cache with `slots` slots of random keys and values."""
    _, hkv, hd, _ = LAYOUTS[layout]
    cap = _cap(slots)
    cache = torch.zeros((hkv, cap // 32, 34 * hd), dtype=torch.uint8, device="cuda")
    for h in range(hkv):
        k, v = _normal(g, 1, slots, hd, std=1.28), _normal(g, 1, slots, hd, std=1.28)
        _store(cache[h : h + 1], _quantise(k.float()), _quantise(v.float()), 0)
    return cache


def prepare(case, seed):
    H, hkv, hd, theta = LAYOUTS[case["layout"]]
    g = torch.Generator(device="cuda")
    g.manual_seed(int(np.random.SeedSequence([seed, 7]).generate_state(1, np.uint64)[0] >> 1))
    s = {"case": case, "H": H, "hkv": hkv, "hd": hd}
    T = case["T"]
    if case["kind"] == "append":
        if case["fused"]:  # the rows q, k, v of one product
            rows = _normal(g, T, (H + 2 * hkv) * hd, std=1.28)
            s["k"], s["v"] = rows[:, H * hd : (H + hkv) * hd], rows[:, (H + hkv) * hd :]
        else:
            s["k"], s["v"] = _normal(g, T, hkv * hd, std=1.28), _normal(g, T, hkv * hd, std=1.28)
        s["cap"] = _cap(case["slot0"] + T)
        s["cache"] = torch.zeros((hkv, s["cap"] // 32, 34 * hd), dtype=torch.uint8, device="cuda")
        pos = np.arange(T)
        if case["tree"]:
            pos = np.array(_depths_masks(_parents(T, seed))[0])
        s["pos"] = torch.from_numpy((case["slot0"] + pos).astype(np.int32)).cuda()
        if case["rotate"]:
            f = theta ** (-2.0 * torch.arange(hd // 2, dtype=torch.float64) / hd)
            a = torch.arange(s["cap"], dtype=torch.float64)[:, None] * f
            s["cos"], s["sin"] = a.cos().float().cuda(), a.sin().float().cuda()
    elif case["kind"] == "read":
        s["cap"] = _cap(case["slot0"] + T)
        s["cache"] = _filled(g, case["layout"], case["slot0"] + T)
    else:
        n_tree = case["extra"] + T
        s["n_tree"], s["n4"] = n_tree, _n4(case)
        s["cap"] = _cap(case["ctx"] + n_tree)
        s["cache"] = _filled(g, case["layout"], case["ctx"] + n_tree)
        s["q"] = _normal(g, T, H, hd)
        rest = case["ctx"] + n_tree - s["n4"]
        s["k"] = s["v"] = None
        if rest:
            s["k"], s["v"] = _normal(g, hkv, rest, hd, std=1.28), _normal(g, hkv, rest, hd, std=1.28)
        masks = _depths_masks(_parents(n_tree, seed))[1][case["extra"] :]
        s["anc"] = torch.from_numpy(masks.view(np.int64).copy()).cuda()
    return s


# ----------------------------------------------------------------------------
# the plain form
# ----------------------------------------------------------------------------

_VALUES = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _quantise(x):
    """Codes [..., hd] (0..15) and scale bytes [..., hd/32] of fp32 rows."""
    b = x.unflatten(-1, (-1, 32))
    amax = b.abs().amax(-1, keepdim=True)
    e = torch.clamp(torch.frexp(amax)[1] - 3, min=-125)
    y = torch.ldexp(b.abs(), -e)
    code = ((y > 0.25).to(torch.uint8) + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5))
    code = code + 8 * torch.signbit(b)
    return code.to(torch.uint8).flatten(-2), (e + 127).to(torch.uint8).squeeze(-1)


def _parts(cache):
    """The four arrays of a cache's records, with their inner dimensions."""
    hd = cache.shape[-1] // 34
    lead, u = cache.shape[:2], hd // 32
    at = [0, 16 * hd, 32 * hd, 33 * hd, 34 * hd]
    dims = [(2, 4, 4, 4, u, 4), (u // 2, 4, u, 16 // u, 2, 8), (u, 4, 4, 2), (u, 32)]
    return [cache[..., at[i] : at[i + 1]].unflatten(-1, dims[i]) for i in range(4)], lead, hd


def _codes_of(cache):
    """Key and value codes [heads][slots][hd] and scale bytes [heads][slots][hd/32]."""
    (k, v, ks, vs), (heads, _), hd = _parts(cache)
    k = k.permute(0, 1, 4, 2, 5, 3, 6, 7).reshape(heads, -1, hd // 2)
    k = torch.stack((k & 15, k >> 4), -1).flatten(-2)
    v = torch.stack((v & 15, v >> 4), -1)  # heads, tile, m, g, b, r, n, j, half
    v = v.permute(0, 1, 3, 7, 4, 2, 6, 8, 5).reshape(heads, -1, hd)
    ks = ks.permute(0, 1, 3, 5, 4, 2).reshape(heads, -1, hd // 32)
    return k, ks, v, vs.transpose(-1, -2).reshape(heads, -1, hd // 32)


def _store(cache, k4, v4, slot0):
    """Writes quantised rows ([heads][n][..] codes and scale bytes) from slot0 on."""
    n = k4[0].shape[1]
    t0, t1 = slot0 // 32, (slot0 + n + 31) // 32
    part = cache[:, t0:t1]
    at = slice(slot0 - 32 * t0, slot0 - 32 * t0 + n)
    rows = _codes_of(part)
    for held, new in zip(rows, (*k4, *v4)):
        held[:, at] = new
    k, ks, v, vs = rows
    (pk, pv, pks, pvs), (heads, tiles), hd = _parts(part)
    u = hd // 32
    k = k.unflatten(-1, (-1, 2))
    k = (k[..., 0] | (k[..., 1] << 4)).reshape(heads, tiles, 4, 2, 4, 4, u, 4)
    pk.copy_(k.permute(0, 1, 3, 5, 2, 4, 6, 7))
    v = v.reshape(heads, tiles, 4, 8, u, u // 2, 2, 2, 16 // u)  # g, j, b, m, n, half, r
    v = v[..., 0, :] | (v[..., 1, :] << 4)
    pv.copy_(v.permute(0, 1, 5, 2, 4, 7, 6, 3))
    pks.copy_(ks.reshape(heads, tiles, 4, 2, 4, u).permute(0, 1, 5, 2, 4, 3))
    pvs.copy_(vs.reshape(heads, tiles, 32, u).transpose(-1, -2))


def _values(code, scale):
    """fp32 values of codes and their scale bytes."""
    table = torch.tensor(_VALUES + [-x for x in _VALUES], device=code.device)
    x = table[code.int()].unflatten(-1, (-1, 32))
    return torch.ldexp(x, scale.int().unsqueeze(-1) - 127).flatten(-2)


def _slots(cache, slot0, n):
    """fp32 keys and values of a range of slots, [heads][n][hd]."""
    t0, t1 = slot0 // 32, (slot0 + n + 31) // 32
    k, ks, v, vs = _codes_of(cache[:, t0:t1])
    at = slice(slot0 - 32 * t0, slot0 - 32 * t0 + n)
    return _values(k[:, at], ks[:, at]), _values(v[:, at], vs[:, at])


def _heads_first(x, hkv):
    return x.unflatten(-1, (hkv, -1)).transpose(0, 1)


def _plain_append(s):
    c = s["case"]
    k, v = _heads_first(s["k"], s["hkv"]).float(), _heads_first(s["v"], s["hkv"]).float()
    if c["rotate"]:  # in 64 bits: a code hangs on which side of a border the value falls
        x, cs, sn = k.double(), s["cos"][s["pos"].long()].double(), s["sin"][s["pos"].long()].double()
        lo, hi = x.chunk(2, -1)
        k = torch.cat((lo * cs - hi * sn, hi * cs + lo * sn), -1).float()
    _store(s["cache"], _quantise(k), _quantise(v), c["slot0"])


def _plain_read(s, slot0, n):
    k, v = _slots(s["cache"], slot0, n)
    return {"k": k.to(torch.bfloat16), "v": v.to(torch.bfloat16)}


def _plain_attend(s):
    c, H, hkv, hd = s["case"], s["H"], s["hkv"], s["hd"]
    T, n_tree, Lc, n4 = c["T"], s["n_tree"], c["ctx"], s["n4"]
    k, v = _slots(s["cache"], 0, n4)
    if s["k"] is not None:
        k, v = torch.cat((k, s["k"].float()), 1), torch.cat((v, s["v"].float()), 1)
    q = s["q"].float().view(T, hkv, H // hkv, hd).permute(1, 2, 0, 3).reshape(hkv, -1, hd)
    x = torch.matmul(q, k.transpose(1, 2).contiguous()) / math.sqrt(hd)
    slot = torch.arange(Lc + n_tree, device=x.device)
    seen = slot < Lc
    if c["window"]:
        seen = seen & ((slot < c["sink"]) | (slot >= Lc - c["window"]))
    seen = seen.repeat(T, 1)
    node = torch.arange(n_tree, device=x.device)
    seen[:, Lc:] = ((s["anc"][:, node // 64] >> (node % 64)) & 1).bool()
    x = x.view(hkv, H // hkv, T, -1).masked_fill(~seen, -math.inf)
    p = torch.exp(x - x.amax(-1, keepdim=True))
    o = torch.matmul((p / p.sum(-1, keepdim=True)).view(hkv, -1, Lc + n_tree), v)
    return o.view(hkv, H // hkv, T, hd).permute(2, 0, 1, 3).reshape(T, H * hd).to(torch.bfloat16)


# ----------------------------------------------------------------------------
# one pass
# ----------------------------------------------------------------------------

def _own_read(s, slot0, n):
    from paper_2510_26843_amd import cas
    k = torch.empty((s["hkv"], n, s["hd"]), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    cas.op_kv4_read(s["cache"], s["cap"], slot0, n, s["hkv"], s["hd"], k, v)
    return {"k": k, "v": v}


def _own_append(s):
    from paper_2510_26843_amd import cas
    c = s["case"]
    cas.op_kv4_append(s["k"], s["v"], c["T"], s["hkv"], s["hd"], s["cache"], s["cap"], c["slot0"], pos=s["pos"],
                      cos=s.get("cos"), sin=s.get("sin"), ldk=s["k"].stride(0), ldv=s["v"].stride(0))


def _own_attend(s):
    from paper_2510_26843_amd import cas
    c = s["case"]
    out = torch.empty((c["T"], s["H"] * s["hd"]), dtype=torch.bfloat16, device="cuda")
    cas.op_attention_kv4(s["q"], s["cache"], s["cap"], s["n4"], c["ctx"], s["n_tree"], c["T"], s["H"], s["hkv"],
                         s["hd"], s["anc"], out, k=s["k"], v=s["v"], sink=c["sink"], window=c["window"])
    return out


def run(state):
    c = state["case"]
    if c["kind"] == "attend":
        return _own_attend(state) if own else _plain_attend(state)
    if c["kind"] == "append":
        _own_append(state) if own else _plain_append(state)
    return (_own_read if own else _plain_read)(state, c["slot0"], c["T"])


def work(case):
    H, hkv, hd, _ = LAYOUTS[case["layout"]]
    T, held, rows = case["T"], hkv * hd * 17 // 16, hkv * hd * 4  # bytes of a slot's k and v, in the cache and in bf16
    if case["kind"] == "read":
        return {"bytes": T * (held + rows), "flops": T * hkv * hd * 2}
    if case["kind"] == "append":
        turn = 2 * hd if case["rotate"] else 0  # fp32 cos and sin of a position
        return {"bytes": T * (2 * rows + 2 * held + 2 * turn), "flops": T * hkv * hd * (8 + (3 if case["rotate"] else 0))}
    n_tree, n4, ctx = case["extra"] + T, _n4(case), case["ctx"]
    seen = min(ctx, case["sink"] + case["window"]) if case["window"] else ctx
    tail = ctx + n_tree - n4
    in4 = seen + n_tree - tail
    return {"bytes": in4 * held + tail * rows + 2 * T * H * hd * 2 + T * 16,
            "flops": 4 * hd * H * T * (seen + (n_tree + 1) // 2)}


# ----------------------------------------------------------------------------
# the definition in 64 bits
# ----------------------------------------------------------------------------

def _exact_mx(x):
    """The values that rows are held as, from the definition."""
    b = x.reshape(*x.shape[:-1], -1, 32)
    top = b.abs().max(-1, keepdim=True).values
    unit = torch.exp2(torch.clamp(torch.floor(torch.log2(top)) - 2, min=-125.0))
    y = b / unit
    step = torch.exp2(torch.clamp(torch.floor(torch.log2(y.abs())), min=0.0) - 1)
    return (torch.clamp(torch.round(y / step) * step, -6, 6) * unit).reshape(x.shape)


def _exact_slots(cache, slots, hd):
    """Keys and values of slots, element by element from the record's layout."""
    s, d = slots[:, None], torch.arange(hd, device=slots.device)[None, :]
    rec, w, u = (s // 32) * (34 * hd), s % 32, hd // 32
    i, h, j = w // 8, w // 4 % 2, w % 4
    g, rest = d // (hd // 4), d % (hd // 4)
    kb = rec + ((((h * 4 + g) * 4 + i) * 4 + j) * u + rest // 8) * 4 + rest % 8 // 2
    ke = rec + 32 * hd + ((d // 32 * 4 + i) * 4 + j) * 2 + h
    wide = 16 // u
    x, r = d % 32 // wide, d % wide  # x = 4m + 2n + half
    vb = rec + 16 * hd + ((((x // 4 * 4 + w // 8) * u + d // 32) * wide + r) * 2 + x // 2 % 2) * 8 + w % 8
    ve = rec + 33 * hd + d // 32 * 32 + w
    flat = cache.reshape(cache.shape[0], -1)

    def value(at, high, scale_at):
        byte = flat[:, at].long()
        n = torch.where(high, byte // 16, byte % 16)
        m = n % 8
        x = torch.where(m < 2, m * 0.5, (1 + (m % 2) * 0.5) * torch.exp2((m // 2 - 1).double()))
        return torch.where(n < 8, x, -x) * torch.exp2(flat[:, scale_at].double() - 127)

    return value(kb, (d % 2 == 1).expand_as(kb), ke), value(vb, (x % 2 == 1).expand_as(vb), ve)


def exact(case, seed):
    s = prepare(case, seed)
    H, hkv, hd = s["H"], s["hkv"], s["hd"]
    T = case["T"]
    if case["kind"] == "read":
        k, v = _exact_slots(s["cache"], case["slot0"] + torch.arange(T, device="cuda"), hd)
        return {"k": k, "v": v}
    if case["kind"] == "append":
        k, v = (s[n].double().reshape(T, hkv, hd).permute(1, 0, 2) for n in ("k", "v"))
        if case["rotate"]:
            i = torch.arange(hd, device="cuda")
            other = (i + hd // 2) % hd
            cs, sn = (s[n].double()[s["pos"].long()][:, i % (hd // 2)] for n in ("cos", "sin"))
            k = k * cs + k[..., other] * sn * torch.where(i < hd // 2, -1.0, 1.0)
            k = k.float().double()  # the one rounding of the rotated key
        return {"k": _exact_mx(k), "v": _exact_mx(v)}
    Lc, n_tree, n4 = case["ctx"], s["n_tree"], s["n4"]
    masks = s["anc"].cpu().numpy().view(np.uint64)
    see = torch.zeros((T, Lc + n_tree), dtype=torch.bool)
    lo = max(0, Lc - case["window"]) if case["window"] else 0
    see[:, lo:Lc] = True
    see[:, : min(case["sink"], Lc)] = True
    for j in range(n_tree):
        see[:, Lc + j] = torch.from_numpy((masks[:, j // 64] >> np.uint64(j % 64)) & np.uint64(1) != 0)
    see = see.cuda()
    out = torch.empty((T, H, hd), dtype=torch.float64, device="cuda")
    for h in range(hkv):
        k, v = _exact_slots(s["cache"][h : h + 1], torch.arange(n4, device="cuda"), hd)
        k, v = k[0], v[0]
        if s["k"] is not None:
            k, v = torch.cat((k, s["k"][h].double())), torch.cat((v, s["v"][h].double()))
        for i in range(h * (H // hkv), (h + 1) * (H // hkv)):
            x = (s["q"][:, i].double() @ k.T) * hd**-0.5
            out[:, i] = torch.softmax(x.masked_fill(~see, -math.inf), -1) @ v
    return out.reshape(T, H * hd)

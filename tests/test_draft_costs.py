"""Cost coefficients of the cascade's levels: every level is timed as it
drafts (its window and its 4-bit KV among it) and priced by what it reads."""
import dataclasses

import numpy as np
import pytest

from paper_2510_26843_amd import dytc, e2e, latency, synth

SHAPE = synth.SHAPES["llama2_7b"]


@pytest.mark.parametrize("kv4", [False, True])
@pytest.mark.parametrize("window", [None, (4, 1024)])
@pytest.mark.parametrize("ctx", [31, 1024, 8190])
@pytest.mark.parametrize("aq", [0, 2])
def test_features_are_the_byte_models(ctx, window, kv4, aq):
    n, run = 3, 16
    f = dytc.roofline_features(SHAPE, run, n, ctx, aq, window, kv4)
    b = latency.algorithmic_bytes(SHAPE, n, ctx, run, int8=aq, window=window, kv4=kv4)
    # the byte model counts the KV written, embedding rows, logits and scales beside
    b -= run * 2 * SHAPE.n_kv_heads * SHAPE.head_dim * 2 * n + n * SHAPE.d_model * 2 + n * SHAPE.vocab * 4
    none = latency.algorithmic_bytes(SHAPE, n, 0, run, int8=aq) - latency.algorithmic_bytes(SHAPE, n, 0, 0)
    scales = none - run * (SHAPE.layer_params() * {0: 2, 2: 0.5}[aq] + 4 * n * SHAPE.n_kv_heads * SHAPE.head_dim * 2)
    assert (f[1] + f[2]) * 1e9 == pytest.approx(b - scales, rel=1e-9)


class _Clock:
    """A model whose forwards take what linear coefficients of their features
    say, on a clock of its own."""

    W = np.array([0.1, 0.2, 0.2, 0.1, 0.01])

    def __init__(self):
        self.now, self.ctx, self.seen = 0.0, 0, set()

    def set_committed(self, n):
        self.ctx = n

    def sync(self):
        pass

    def cost(self, n, skip, act_quant, window, kv4):
        run = SHAPE.n_layers - (sum(skip) if skip else 0)
        return float(dytc.roofline_features(SHAPE, run, n, self.ctx, act_quant, window, kv4) @ self.W)

    def forward(self, tokens, parents, off, skip=None, act_quant=0, logits=True, attn_window=None, kv4=False):
        self.seen.add((skip and tuple(skip), act_quant, attn_window, kv4))
        self.now += self.cost(len(tokens), skip, act_quant, attn_window, kv4) / 1e3


def test_calibration_times_the_draft_that_a_level_is(monkeypatch):
    m = _Clock()
    monkeypatch.setattr(e2e.time, "perf_counter", lambda: m.now)
    odd = tuple(l % 2 for l in range(SHAPE.n_layers))
    plain = [dytc.DraftConfig("odd", odd), dytc.DraftConfig("odd4", odd, 2), dytc.DraftConfig("win", odd, window=(4, 1024))]
    levels = plain + [dataclasses.replace(c, name=c.name + "_kv4", kv4=True) for c in plain]
    levels.append(dytc.DraftConfig("kv4", kv4=True))
    ctx = 16000
    got = e2e.calibrate(m, SHAPE, ctx, levels, lambda *a: None)
    assert m.seen >= {(c.skip, c.act_quant, c.window, c.kv4) for c in levels}
    m.ctx = ctx
    base = m.cost(1, None, 0, None, False)
    # the regression's objective is at most its prior's at the true weights, so a
    # timed point is off by sqrt(prior / noise) |W| ms at most: twice that here,
    # for the level's point and the target's
    tol = 2 * np.sqrt(1e-3 / 1e2) * np.linalg.norm(m.W) / base
    for c in levels:
        want = m.cost(1, c.skip, c.act_quant, c.window, c.kv4) / base
        assert got["cost"][c.name] == pytest.approx(want, abs=tol * (1 + want)), c.name
    assert got["cost"]["odd_kv4"] < 0.9 * got["cost"]["odd"]

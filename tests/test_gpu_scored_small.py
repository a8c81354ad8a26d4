"""Many tokens of which each has next to no weight, beside one that has nearly all, in attention of many rows with other scores (flatquant_cache_scored_attention): what they have
together stays within the bound, whose part for products in fp16's subnormals is 2^-32 of the largest a token, or 2^-27 with a cap and 2^14 tokens or fewer."""
import math

import numpy as np
import pytest

from cache_util import D, Batch
from oracle import step_oracle as so
from test_gpu_scored import run_scored

pytestmark = pytest.mark.gpu
ROWS, SCALE, K_STEP, V_STEP = 33, 0.25, 0.125, 0.0625


@pytest.mark.parametrize("whole", ["8 waves", "4 waves"])
@pytest.mark.parametrize("kind", ["cap", "large cap", "slopes", "prefix"])
@pytest.mark.parametrize("tokens", [8192, 16384, 16385, 131072])
def test_one_token_beside_many(tokens, kind, whole, tuning):
    """The axis in one workgroup.  Scores: the one token's, and zero; weights of the others from 2^-27.2 of its (below half a step of fp16's subnormals where the largest
    product is 2^2) down."""
    print(f"[case] {tokens} {kind} {whole}", flush=True)
    tuning("FLATQUANT_ATT_WAVES", 8 if whole == "8 waves" else 4)
    if whole == "4 waves":
        tuning("FLATQUANT_ATT_CHUNK", 1 << 28)
    c = Batch(1, [ROWS], [tokens], 1, page=1024, filled=False)
    at = tokens - ROWS if kind == "slopes" else 0                              # with slopes the steps go backwards: the one is where they come first
    page, place = int(c.table[0, at // 1024]), at % 1024
    for x, step in zip(c.host, (K_STEP, V_STEP)):
        x.codes[:], x.params[:] = 0, int(np.float16(step).view(np.uint16))
    c.host[0].codes[page, 0, place, 0] = 15                                    # that token's key: channel 0 alone
    c.host[1].codes[:] = 0xFF                                                  # values: 15 steps, of that token none
    c.host[1].codes[page, 0, place] = 0
    cap = {"cap": 50.0, "large cap": 300.0}.get(kind, 0.0)
    score = np.log(2.0) * (27.2 + 0.05 * np.arange(ROWS))
    if cap:
        score = cap * np.arctanh(score / cap)
    q = np.zeros((ROWS, D), dtype=np.float16)
    q[:, 0] = score / (SCALE * K_STEP * 15)
    how = dict(cap=cap, slopes=[0.0] if kind == "slopes" else None, prefix=[1] if kind == "prefix" else None)
    got = run_scored(c.upload(), q, 1, SCALE, **how).astype(np.float64)
    k, v = np.zeros((tokens, D)), np.full((tokens, D), 15 * V_STEP)
    k[at, 0], v[at] = 15 * K_STEP, 0.0
    ks, vs = np.full(tokens, K_STEP), np.full(tokens, V_STEP)
    for i in (0, 7, ROWS - 1):
        seen = (np.arange(tokens) <= tokens - ROWS + i)[None]
        o, A, S, E = so.scored64(q[i:i + 1], k, v, seen, SCALE, np.array([tokens - ROWS + i]), cap, 0.0, ks, vs)
        tol = so.scored_bound(o, A, S, E, tokens, capped=cap > 0)
        share = (tokens - ROWS + i) * math.exp(-float(score[i] if not cap else cap * np.tanh(score[i] / cap)))
        assert abs(o[0, 0] / (15 * V_STEP) / share - 1) < 0.01                 # (queries are rounded)
        worst = float((np.abs(got[i] - o) / tol).max())
        print(f"[case] row {i}: {worst:.3f} of the bound, the others' share {share:.2e}", flush=True)
        assert worst <= 1.0

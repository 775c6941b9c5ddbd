"""The step over pages with blocks chosen, against the same step in 64 bits: every layer and head scores the bounds of its own
pages with its own query, chooses, and attends to the rows of what it chose."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

from oracle import cerberus_oracle as orc
from paper_2410_13344_amd import binding as B
from paper_2410_13344_amd import synth
from tests import harness as H

F32, BF16 = B.CERBERUS_F32, B.CERBERUS_BF16


def sparse_step(cfg, W, token, L, keys, values, bounds, n_select, page):
    """(logits of the one row, the smallest difference between a score that was chosen and one that was not).  keys, values: [layer][head][L][dh]
    rows of the cache; bounds: [layer][block][head][2][dh]."""
    d, nH, dh, F = cfg["d_model"], cfg["n_heads"], cfg["head_dim"], cfg["d_ffn"]
    held, gap = L // page + 1, math.inf                            # (row L is there too)
    x = orc._f(W["embed"][np.array([token])])
    pos = np.array([L])
    for l in range(cfg["n_layers"]):
        w = W["layers"][l]
        qkv = orc.rmsnorm(x, w["attn_norm"], cfg["rms_eps"]) @ orc._f(w["wqkv"]).T
        q = orc.rope(qkv[:, :d].reshape(1, nH, dh), pos, cfg["rope_theta"])[0]
        k = orc.rope(qkv[:, d:2 * d].reshape(1, nH, dh), pos, cfg["rope_theta"])[0]
        v = qkv[:, 2 * d:].reshape(nH, dh)
        o = np.zeros((nH, dh))
        for h in range(nH):
            chosen = list(range(held))
            if held > n_select:
                middle = range(1, held - 1)
                score = {j: float(np.sum(np.where(q[h] >= 0, q[h] * bounds[l][j, h, 1], q[h] * bounds[l][j, h, 0]))) for j in middle}
                best = sorted(middle, key=lambda j: (-score[j], j))
                m = max(n_select - 2, 0)
                if 0 < m < len(best):
                    gap = min(gap, score[best[m - 1]] - score[best[m]])
                chosen = best[:m] + [held - 1] + ([0] if n_select > 1 else [])
            rows = [r for j in chosen for r in range(j * page, min((j + 1) * page, L))]
            K, V = np.concatenate([keys[l][h][rows], k[h][None]]), np.concatenate([values[l][h][rows], v[h][None]])
            s = K @ q[h] / math.sqrt(dh)
            e = np.exp(s - s.max())
            o[h] = (e / e.sum()) @ V
        x = x + o.reshape(1, d) @ orc._f(w["wo"]).T
        gu = orc.rmsnorm(x, w["ffn_norm"], cfg["rms_eps"]) @ orc._f(w["w_gate_up"]).T
        x = x + (orc.silu(gu[:, :F]) * gu[:, F:]) @ orc._f(w["w_down"]).T
    return (orc.rmsnorm(x, W["final_norm"], cfg["rms_eps"]) @ orc._f(W["lm_head"]).T)[0], gap


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads", [{}, dict(n_heads=2, head_dim=128)])
@pytest.mark.parametrize("blocks", [9, 1100])                      # room of a table: the choice in one launch, in two
def test_paged_step_attends_to_the_blocks_that_every_layer_and_head_chooses(dtype, heads, blocks):
    """A choice is settled where the scores next to its border lie apart by more than the queries can be off.  A score is off by at
    most sum |dq| |bound|.  The queries' error, like that of h_last, is within tol.hidden, and errors of 64 or 128 coordinates
    of either sign add up as their root at most ten times over; bounds are below 8: 80 tol.hidden would be safe and leave nothing to
    compare in bf16, where the measured error of h_last is a tenth of its bar.  So: 8 tol.hidden (bf16 3.2e-2, fp32 4e-4)."""
    pair = H.Pair("tiny", dtype, "tiny", seed=0, max_batch=3, kv_capacity=192, **heads)
    eng, cfg, page, lens = pair.engine, pair.cfg, 16, [128, 90, 111]
    tol = H.TOL_F32 if dtype == F32 else H.TOL_BF16_TINY
    taps, compared = pair.taps(), 0
    rows = torch.arange(3, device="cuda") * pair.T
    for n_select in (1, 2, 3, 4, 5, 6):
        sp = eng.new_state()
        for b, n in enumerate(lens):
            eng.prefill(sp, 3, b, synth.make_token_ids(n, cfg["vocab"], seed=20 + b).to(torch.int32).cuda())
        cache = B.PageCache(cfg["n_layers"], 40, page, cfg["n_heads"], cfg["head_dim"], dtype, 3, blocks)
        eng.move_prompts(sp, cache, lens)
        for step in range(2):                                      # (112 rows and one: the third begins a page in the second step)
            want = []
            for b, n in enumerate(lens):
                L, pages = n + step, cache.block_table[b, :-(-(n + step) // page)].long()
                host = [t[:, pages].double().cpu().numpy() for t in (cache.k, cache.v, cache.bounds)]
                flat = [t.transpose(0, 2, 1, 3, 4).reshape(cfg["n_layers"], cfg["n_heads"], -1, cfg["head_dim"])[:, :, :L] for t in host[:2]]
                want.append(sparse_step(cfg, pair.W, int(sp.root_token[b]), L, flat[0], flat[1], host[2], n_select, page))
            eng.paged_step(sp, cache, 3, n_select=n_select)
            got = taps.logits[rows].double().cpu().numpy()
            for b, (logits, gap) in enumerate(want):
                if gap > 8 * tol.hidden:
                    compared += 1
                    assert np.abs(got[b] - logits).max() <= tol.logits, (n_select, step, b, gap, np.abs(got[b] - logits).max())
        assert int(cache.status) == 0
    print("compared", compared)
    assert compared >= 18                                          # (half of them)
    eng.close()

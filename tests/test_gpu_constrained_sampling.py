"""Sampled steps under constraints where the block maxima narrow a row down (top_k no more
than the vocabulary's 128-id blocks), every decision against the float64 rule."""
import dataclasses

import numpy as np
import pytest
import torch

from oracle.sampling import verify_sampled
from paper_2607_17299_amd import synth
from test_gpu_constraints import DEV, _war, bits_of, f32, t32

pytestmark = pytest.mark.gpu
B, K = 4, 3
TOP = 2.0 ** 30   # so large a bias leaves equal logits: an fp32 step there is 64 and more


@pytest.fixture(scope="module")
def decoder(request):
    war = _war()
    cfg = dataclasses.replace(synth.TINY, vocab=request.param)
    w = synth.model_weights(cfg, seed=0, norm_std=0.1)
    return cfg, war.Model(cfg, {k: v.to(DEV) for k, v in w.items()}, max_rows=256)


def expected(rows, drafts, u, T, top_k):
    """(accept, next, least margin): rows end at the first that leaves no token."""
    live = 0
    while live < len(rows) and np.isfinite(rows[live]).any():
        live += 1
    if live == 0:
        return 0, -1, 1.0
    if live == len(rows):
        r = verify_sampled(rows, drafts, u[:, 0], u[:, 1], T, top_k)
        return r["accept"], r["next"], min(r["margins"])
    # a row of any logits stands for the one without a token: where it is reached there is none
    r = verify_sampled(np.concatenate([rows[:live], np.zeros((1, rows.shape[1]))]), drafts[:live], u[: live + 1, 0],
                       u[: live + 1, 1], T, top_k)
    if r["accept"] == live:
        return live, -1, min(r["margins"][:live])
    return r["accept"], r["next"], min(r["margins"])


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
@pytest.mark.parametrize("decoder,top_k", [(4096, 1), (4096, 8), (4096, 32), (131072, 1), (131072, 8), (131072, 200),
                                           (131072, 1024)], indirect=["decoder"])
def test_every_decision_follows_the_rule(decoder, top_k, fmt):
    war, (cfg, model) = _war(), decoder
    V = cfg.vocab
    rng = np.random.default_rng(top_k)
    R, T = B * (K + 1), 0.8
    bad = rng.choice(V, 2, replace=False)                        # excluded everywhere; their bias is NaN and inf
    ok = np.setdiff1d(np.arange(V), bad)
    few = lambda n: rng.choice(ok, n, replace=False)
    allowed = rng.random((R, V)) < 0.33
    drafts = rng.choice(ok, (B, K))
    for r, n in ((4, 1), (5, 1), (6, 0), (8, 0), (12, 3), (13, 2), (14, min(top_k, 5)), (15, len(ok))):
        allowed[r] = False
        at = few(n)
        allowed[r, at] = True
        if r % (K + 1) < K and n:
            drafts[r // (K + 1), r % (K + 1)] = at[0]
    allowed[3] = True
    allowed[:, bad] = False
    # request 0: equal logits around the top_k-th place
    ties = few(min(1000, 2 * top_k + 3))
    allowed[0, ties[0]] = True
    bias_ids, bias = np.full((B, len(ties) + 2), -1), np.zeros((B, len(ties) + 2))
    bias_ids[0, :-2], bias[0, :-2] = ties, TOP
    bias_ids[:, -2:], bias[:, -2:] = bad, [np.nan, np.inf]
    cons = war.Constraints(V, masks=bits_of(allowed), bias_ids=t32(bias_ids), bias_values=f32(bias))
    pool = war.Pool(cfg, 64, B, 16, device=DEV, kv_format=fmt)
    seq, ctx, nxt, acc = t32(list(range(B))), t32([0] * B), t32([0] * B), t32([0] * B)
    toks = np.concatenate([synth.uniform_tokens(70 + b, 33, V) for b in range(B)])
    war.prefill_append(model, pool, seq, ctx, [33] * B, t32(toks), nxt)
    drafts[0, 0] = rng.choice(np.flatnonzero(allowed[0] & np.isin(np.arange(V), ties)))
    accepted = 0
    for turn in range(6):
        u = rng.random((R, 2)).astype(np.float32)
        if turn == 0:
            u[0] = [0.0, 1 - 2.0 ** -24]                         # the ends of the range
        z = torch.empty((R, V), device=DEV)
        for logits in (z, None):                                 # into the caller's logits, then without
            acc.fill_(77), nxt.fill_(77)
            war.verify_step_constrained(model, pool, seq, ctx, nxt * 0 + 5, t32(drafts), None, K, cons, acc, nxt, logits,
                                        uniforms=f32(u), temperature=T, top_k=top_k)
            war.kv_commit(pool, seq, ctx, t32([-1] * B))
            zz = z.cpu().numpy().astype(np.float64)
            assert ((zz == -np.inf) == ~allowed).all() and not np.isnan(zz).any()
            for b in range(B):
                r = slice(b * (K + 1), (b + 1) * (K + 1))
                a, t, margin = expected(zz[r], drafts[b].tolist(), u[r].astype(np.float64), T, top_k)
                assert (int(acc[b]), int(nxt[b])) == (a, t) or margin < 1e-5, (turn, b, a, t, margin)
                accepted += int(acc[b])
        assert (int(acc[1]), int(nxt[1])) == (2, -1) and (int(acc[2]), int(nxt[2])) == (0, -1)
    assert accepted >= 6 * 2 * 2 and pool.state()["status"] == 0

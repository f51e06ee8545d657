"""Attention over e4m3 pools is off by no more than attention over bf16 pools: the
softmax weights keep 16 bits, as over every cache, whatever the values' codes keep."""
import numpy as np
import pytest
import torch

from oracle import e4m3
from test_gpu_kv8 import DEV, _war, as64, cfg_of, scattered_pool, t32

pytestmark = pytest.mark.gpu


def rows_seen(ctx, rows, parents):
    see = np.zeros((rows, ctx + rows), bool)
    see[:, :ctx] = True
    for i in range(rows):
        j = i
        while True:
            see[i, ctx + j] = True
            if j == 0:
                break
            j = parents[j - 1] if parents else j - 1
    return see


def case(heads, n, ctx, rows, parents=None, seed=0, fmt="e4m3", spoil=None):
    """[(got, want, bound)] of each request, [rows, Hq, D] in float64."""
    war = _war()
    cfg = cfg_of(*heads)
    Hq, Hkv, D, B = *heads, len(ctx)
    G = Hq // Hkv
    g = torch.Generator().manual_seed(seed)
    pool = scattered_pool(cfg, [c + n for c in ctx], fmt)
    q = torch.randn((B, n, Hq, D), generator=g).bfloat16()
    held = []
    for b in range(B):
        S = ctx[b] + rows[b]
        k = torch.randn((1, S, Hkv, D), generator=g).bfloat16()
        v = (torch.randn((1, S, Hkv, D), generator=g) * torch.exp2(torch.randint(-3, 4, (1, S, 1, 1), generator=g))).bfloat16()
        if spoil is not None:
            spoil(b, k, v)
        war.kv_write(pool, 0, t32([b]), t32([0]), k.to(DEV), v.to(DEV))
        held.append(e4m3.store_kv(as64(k[0]), as64(v[0])) if fmt == "e4m3" else (as64(k[0]), as64(v[0])))
    plan = war.AttendPlan(pool, B, n)
    out = torch.full((B, n, Hq, D), 7.0, dtype=torch.bfloat16, device=DEV)
    plan.update(t32(list(range(B))), t32(ctx), t32(rows), t32(parents) if parents else None)
    war.attend(plan, 0, q.to(DEV), out)
    assert pool.state()["status"] == 0
    res = []
    for b in range(B):
        r, (k, v) = rows[b], held[b]
        see = rows_seen(ctx[b], r, parents[b] if parents else None)
        want, tol = np.zeros((r, Hq, D)), np.zeros((r, Hq, D))
        for h in range(Hq):
            qh, K, V = as64(q[b, :r, h]), k[:, h // G], v[:, h // G]
            s = np.where(see, qh @ K.T / np.sqrt(D), -np.inf)
            p = np.exp(s - s.max(-1, keepdims=True))
            p /= p.sum(-1, keepdims=True)
            # the result rounded to bf16: 2^-8 of it; scores summed over D products in fp32: a
            # weight and the sum off by exp(2 ds); two bf16 parts of a weight keep 2^-17 of it,
            # exp2 and the fp32 sums stay under 2^-15 of the sum of magnitudes T
            ds = (D + 4) * 2.0 ** -24 * (np.abs(qh) @ np.abs(K).T).max() / np.sqrt(D)
            Vz = np.where(np.isfinite(V), V, 0.0)
            T = p @ np.abs(Vz)
            want[:, h] = p @ Vz
            tol[:, h] = 2.0 ** -8 * np.abs(want[:, h]) + (np.expm1(2 * ds) + 2.0 ** -14) * T
        res.append((as64(out[b, :r]), want, tol))
    return res


@pytest.mark.parametrize("fmt", ["e4m3", "bf16"])
@pytest.mark.parametrize("heads,n,ctx,rows", [
    ((4, 2, 64), 1, [0, 5, 1000], [1, 1, 1]),            # one row tile
    ((8, 2, 128), 3, [33, 700, 2500], [3, 2, 3]),
    ((8, 2, 64), 6, [100, 3000], [6, 5]),                # two
    ((32, 8, 128), 9, [500, 64], [9, 7]),                # three
    ((4, 4, 64), 40, [2100], [33]),
    ((8, 2, 64), 70, [900, 0], [70, 41]),                # row blocks
    ((16, 2, 128), 64, [3, 1500], [64, 50]),
])
def test_weights_keep_sixteen_bits(fmt, heads, n, ctx, rows):
    for got, want, tol in case(heads, n, ctx, rows, fmt=fmt):
        assert (np.abs(got - want) <= tol).all(), (np.abs(got - want) / tol).max()


def test_weights_of_draft_trees_keep_sixteen_bits():
    parents = [[0, 0, 1, 1, 3, 0, 6], [0, 1, 2, 3, 4, 5, 6], [0] * 7]
    for got, want, tol in case((8, 4, 64), 8, [40, 0, 1000], [8, 6, 8], parents):
        assert (np.abs(got - want) <= tol).all(), (np.abs(got - want) / tol).max()

"""Keys and values in 8 bits: war_kv_write / war_kv_read bit for bit against the oracle,
attention over given rows (war_attend) in both formats, and every step over an 8-bit
pool against the oracle with the same cache."""
import copy
import gc

import numpy as np
import pytest
import torch

from oracle import e4m3
from oracle.decoder import RequestKV, Weights
from oracle.verify import commit_request, prefill_request, verify_request, verify_tree_request
from paper_2607_17299_amd import synth
from parity import compare_request, compare_tree_request, fp32_drift_tol

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _war():
    from paper_2607_17299_amd import war
    return war


def t32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)


def cfg_of(q, kv, dim, layers=1):
    return synth.ModelConfig(n_layers=layers, d_model=128, n_q_heads=q, n_kv_heads=kv, head_dim=dim, ffn_dim=128, vocab=128)


def scattered_pool(cfg, tokens, fmt, layers=None):
    """A pool whose sequences' pages interleave; every byte starts as 0xff (NaN)."""
    war = _war()
    pages = [-(-t // 16) for t in tokens]
    pool = war.Pool(cfg, sum(pages) + 2, len(tokens), max(max(pages), 1), device=DEV, kv_format=fmt)
    pool.kv.view(torch.uint8).fill_(255)
    for part in range(1, 5):
        pool.alloc(list(range(len(tokens))), [t * part // 4 for t in tokens])
    return pool


def as64(x):
    return x.double().cpu().numpy()


# ---------------------------------------------------------------- write and read
@pytest.mark.parametrize("heads", [(4, 2, 64), (32, 8, 128), (7, 1, 128)])
@pytest.mark.parametrize("fmt", ["e4m3", "bf16"])
def test_write_then_read_is_the_oracles(heads, fmt):
    war = _war()
    cfg = cfg_of(*heads, layers=2)
    rng = np.random.default_rng(1)
    pos, n, n_max = [0, 5, 16, 31, 47, 0, 300], [1, 0, 16, 40, 2, 37, 40], 40
    pool = scattered_pool(cfg, [p + n_max for p in pos], fmt)
    ids = t32(np.arange(len(pos))[::-1].copy())          # request b is sequence B - 1 - b
    pool2 = [p + n_max for p in pos][::-1]
    pool = scattered_pool(cfg, pool2, fmt)
    x = rng.standard_normal((2, len(pos), n_max, cfg.n_kv_heads, cfg.head_dim))
    x *= 2.0 ** rng.integers(-140, 120, x.shape[:-1] + (1,))   # every size of block, subnormal ones too
    x[:, 2, 3] = 0.0
    x[0, 3, 7, 0, 5], x[1, 5, 0, 0, 1], x[1, 5, 36, 0, 0] = np.inf, np.nan, -np.inf
    k, v = (torch.tensor(y, device=DEV).bfloat16() for y in x)
    before = pool.kv.clone()
    war.kv_write(pool, 1, ids, t32(pos), k, v, t32(n))
    out = [torch.full_like(k, 7.0) for _ in range(2)]
    war.kv_read(pool, 1, ids, t32(pos), *out, t32(n))
    assert pool.state()["status"] == 0
    want = e4m3.store_kv(as64(k), as64(v)) if fmt == "e4m3" else (as64(k), as64(v))
    for got, w in zip(out, want):
        got = as64(got)
        for b in range(len(pos)):
            np.testing.assert_array_equal(got[b, : n[b]], w[b, : n[b]])
            assert (got[b, n[b]:] == 7.0).all()
    # layer 0 and every byte of other tokens are as they were: writing the rest of the
    # pool's tokens back changes only what was written above
    codes = 2 * cfg.n_kv_heads * 16 * cfg.head_dim * (1 if fmt == "e4m3" else 2)
    a, b = before.view(torch.uint8), pool.kv.view(torch.uint8)
    assert torch.equal(a[: codes * pool.num_pages], b[: codes * pool.num_pages])
    changed = int((a != b).sum())
    per = cfg.n_kv_heads * 2 * (cfg.head_dim * (1 if fmt == "e4m3" else 2) + (1 if fmt == "e4m3" else 0))
    assert 0 < changed <= sum(n) * per


def test_every_bf16_number_at_every_place_of_a_block():
    """All finite bf16 numbers, each once the block's largest and once beside a larger one."""
    war = _war()
    cfg = cfg_of(4, 2, 64)
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    x = bits[torch.isfinite(bits)]
    x = x[x.abs().double() <= 1.9375 * 2.0 ** 127]
    x = torch.cat([x, x[: -len(x) % 128]]).view(-1, 64)             # neighbours by bit pattern share a block
    k = torch.cat([x, x.flatten()[torch.randperm(x.numel(), generator=torch.Generator().manual_seed(0))].view(-1, 64)])
    n = k.shape[0] // 2
    k = k.view(1, n, 2, 64).to(DEV)
    v = k.flip(1).flip(3).contiguous()
    pool = scattered_pool(cfg, [n], "e4m3")
    war.kv_write(pool, 0, t32([0]), t32([0]), k, v)
    ok, ov = torch.empty_like(k), torch.empty_like(v)
    war.kv_read(pool, 0, t32([0]), t32([0]), ok, ov)
    wk, wv = e4m3.store_kv(as64(k), as64(v))
    # 1.9375 * 2^127 is 248 * 2^120, between the numbers 240 and 256 = even: 2^128, which bf16 has not
    big = lambda w: np.where(np.abs(w) >= 2.0 ** 128, np.copysign(np.inf, w), w)
    np.testing.assert_array_equal(as64(ok), big(wk))
    np.testing.assert_array_equal(as64(ov), big(wv))


def test_load_write_and_strided_rows_store_the_same_bytes():
    war = _war()
    cfg = cfg_of(16, 2, 128)
    n = 53
    g = torch.Generator(device=DEV).manual_seed(3)
    qkv = torch.randn((1, n, (16 + 4) * 128), device=DEV, generator=g).bfloat16()   # a projection's rows
    k, v = qkv[..., 16 * 128: 18 * 128].view(1, n, 2, 128), qkv[..., 18 * 128:].view(1, n, 2, 128)
    pools = [scattered_pool(cfg, [n + 3], "e4m3") for _ in range(3)]
    war.kv_write(pools[0], 0, t32([0]), t32([3]), k, v)
    pools[1].load(0, 0, 3, torch.stack([k[0].transpose(0, 1), v[0].transpose(0, 1)]).contiguous())
    for i in range(n):                                     # token by token
        war.kv_write(pools[2], 0, t32([0]), t32([3 + i]), k[:, i:i + 1], v[:, i:i + 1])
    assert torch.equal(pools[0].kv, pools[1].kv) and torch.equal(pools[0].kv, pools[2].kv)


def test_bad_requests_are_left_out_and_flagged():
    war = _war()
    cfg = cfg_of(4, 2, 64)
    for bad in (dict(seq=9), dict(seq=-1), dict(pos=-1), dict(pos=30), dict(n=5), dict(n=-1), dict(pos=2**31 - 1)):
        pool = scattered_pool(cfg, [32, 32], "e4m3")
        before = pool.kv.clone()
        k = torch.ones((2, 4, 2, 64), dtype=torch.bfloat16, device=DEV)
        args = [t32([0, bad.get("seq", 1)]), t32([0, bad.get("pos", 0)]), k, k, t32([0, bad.get("n", 4)])]
        war.kv_write(pool, 0, *args)
        assert pool.state()["status"] == -5, bad
        assert torch.equal(before, pool.kv), bad
        assert pool.state()["status"] == 0


# ------------------------------------------------------------------- attention
def attend_case(fmt, heads, n, ctx, rows, parents=None, seed=0, layers=1, spoil=None):
    """(got [B, n, Hq, D] float64, prefilled with 7; want with the same; error bound)."""
    war = _war()
    cfg = cfg_of(*heads, layers=layers)
    Hq, Hkv, D, G, B = *heads, heads[0] // heads[1], len(ctx)
    g = torch.Generator().manual_seed(seed)
    pool = scattered_pool(cfg, [c + n for c in ctx], fmt)
    q = torch.randn((B, n, Hq, D), generator=g).bfloat16()
    kv = []
    for b in range(B):
        S = ctx[b] + rows[b]
        k = torch.randn((1, max(S, 1), Hkv, D), generator=g) * torch.where(torch.arange(D) % 16 == 0, 5.0, 1.0)
        v = torch.randn((1, max(S, 1), Hkv, D), generator=g) * torch.exp2(torch.randint(-3, 4, (1, max(S, 1), 1, 1), generator=g))
        if spoil is not None:
            spoil(b, k, v)
        k, v = k.bfloat16(), v.bfloat16()
        if S:
            war.kv_write(pool, layers - 1, t32([b]), t32([0]), k.to(DEV)[:, :S], v.to(DEV)[:, :S])
        kv.append(e4m3.store_kv(as64(k[0]), as64(v[0])) if fmt == "e4m3" else (as64(k[0]), as64(v[0])))
    plan = war.AttendPlan(pool, B, n)
    out = torch.full((B, n, Hq, D), 7.0, dtype=torch.bfloat16, device=DEV)
    plan.update(t32(list(range(B))), t32(ctx), t32(rows), t32(parents) if parents else None)
    war.attend(plan, layers - 1, q.to(DEV), out)
    assert pool.state()["status"] == 0
    want, tol = np.full((B, n, Hq, D), 7.0), np.zeros((B, n, Hq, D))
    for b in range(B):
        reference(fmt, as64(q[b]), *kv[b], ctx[b], rows[b], parents[b] if parents else None, want[b], tol[b])
    return as64(out), want, tol


def reference(fmt, q, k, v, ctx, rows, parents, want, tol):
    """One request's rows in float64 into want [n, Hq, D], with what a result may be off by."""
    n, Hq, D = q.shape
    G = Hq // k.shape[1]
    for i in range(rows):
        see = list(range(ctx + i + 1))
        if parents:
            see, j = list(range(ctx)), i
            while True:
                see.append(ctx + j)
                if j == 0:
                    break
                j = parents[j - 1]
        for h in range(Hq):
            K, V = k[see, h // G], v[see, h // G]
            s = K @ q[i, h] / np.sqrt(D)
            with np.errstate(invalid="ignore"):
                p = np.exp(s - s.max())
                p /= p.sum()
                want[i, h] = p @ V
            # the result rounded to bf16; scores summed over D products in fp32 move a
            # weight and the sum by exp(2 ds); a weight's two bf16 parts keep 2^-16 of it
            # (2^-17 each way), exp2 and the sums in fp32 under 2^-15 of it altogether
            ds = (D + 4) * 2.0 ** -24 * (np.abs(K) @ np.abs(q[i, h])).max() / np.sqrt(D)
            T = p @ np.abs(V)
            tol[i, h] = 2.0 ** -8 * np.abs(want[i, h]) + (np.expm1(2 * ds) + 2.0 ** -14) * T
            if fmt == "e4m3":
                # one bf16 a weight: p (1 + d) with |d| <= 2^-8 above and below the line,
                # (sum p (1 + d) v) / (sum p (1 + d)) is off by at most 2^-8 (T + |o|) / (1 - 2^-8)
                tol[i, h] += 2.0 ** -8 * (T + np.abs(want[i, h])) * 1.004


def check(got, want, tol):
    assert (np.isnan(got) == np.isnan(want)).all()
    ok = ~np.isnan(want)
    err = np.abs(got[ok] - want[ok])
    assert (err <= tol[ok]).all(), f"worst {np.max(err / np.maximum(tol[ok], 1e-30)):.3g} of the bound"


@pytest.mark.parametrize("fmt", ["e4m3", "bf16"])
@pytest.mark.parametrize("heads,n,ctx,rows", [
    ((4, 2, 64), 1, [0, 1, 15, 16, 17, 31, 32, 33], [1] * 8),            # one row, pages that end anywhere
    ((32, 8, 128), 1, [0, 700, 127, 3000], [1, 1, 0, 1]),                # a request without rows
    ((32, 8, 128), 5, [0, 1029, 95], [5, 2, 4]),                         # two row tiles
    ((16, 2, 128), 6, [260, 31], [6, 6]),                                # three row tiles, eight heads a kv-head
    ((7, 1, 128), 6, [77, 0, 1500], [6, 1, 3]),                          # seven heads a kv-head
    ((8, 8, 64), 12, [511, 2], [12, 7]),                                 # heads that share nothing
])
def test_attention_of_a_steps_rows(fmt, heads, n, ctx, rows):
    check(*attend_case(fmt, heads, n, ctx, rows))


@pytest.mark.parametrize("fmt", ["e4m3", "bf16"])
@pytest.mark.parametrize("heads,n,ctx,rows", [
    ((4, 2, 64), 70, [0, 130], [70, 33]),        # several row blocks, one ends raggedly
    ((8, 2, 128), 45, [700, 0, 17], [45, 0, 1]),  # a request without rows, one with a single one
    ((7, 1, 128), 40, [333], [40]),              # 18 tokens a block
    ((3, 3, 128), 129, [5], [129]),              # heads that share nothing
])
def test_attention_of_many_rows(fmt, heads, n, ctx, rows):
    check(*attend_case(fmt, heads, n, ctx, rows))


def test_chunks_of_row_blocks_merge():
    """More than one chunk for the later row blocks, the chunk border inside one."""
    check(*attend_case("e4m3", (4, 1, 128), 100, [470, 200], [100, 100]))


@pytest.mark.parametrize("fmt", ["e4m3", "bf16"])
@pytest.mark.parametrize("heads,n,ctx,rows", [
    ((32, 32, 64), 50, [14000], [50]),              # 16 items fill the grid: chunks of 896 or so keys
    ((16, 16, 64), 130, [3000, 0, 1000], [60, 130, 0]),
])
def test_cuts_of_row_blocks(fmt, heads, n, ctx, rows):
    check(*attend_case(fmt, heads, n, ctx, rows))


@pytest.mark.parametrize("heads,n,ctx", [
    ((32, 8, 128), 1, [5000, 3000, 4100]),       # cut into chunks of 384 or so keys
    ((8, 8, 64), 7, [2500, 1, 6300, 0, 700]),    # 640
    ((2, 2, 64), 3, [9000, 64]),                 # one request takes most of them
])
def test_even_cuts(heads, n, ctx):
    check(*attend_case("e4m3", heads, n, ctx, [n] * len(ctx)))


@pytest.mark.parametrize("fmt", ["e4m3", "bf16"])
def test_attention_of_draft_trees(fmt):
    parents = [[0, 0, 1, 1, 3, 0, 6], [0, 1, 2, 3, 4, 5, 6], [0] * 7]
    check(*attend_case(fmt, (8, 4, 64), 8, [40, 0, 1000], [8, 6, 8], parents))


@pytest.mark.parametrize("n", [4, 30])
def test_tokens_that_are_not_finite_reach_only_the_rows_that_see_them(n):
    def spoil(b, k, v):
        if b == 0:
            v[0, 102, 0, 3] = float("nan")       # row 2's own token
        if b == 1:
            k[0, 50, 1, 9] = float("inf")        # a context token: every row of that kv-head
    got, want, tol = attend_case("e4m3", (8, 2, 64), n, [100, 60], [n, n], spoil=spoil)
    assert np.isfinite(want[0, :2]).all() and np.isnan(want[0, 2:, :4]).all() and np.isnan(want[1, :, 4:]).all()
    check(got, want, tol)


def test_forked_siblings_share_their_prefix():
    war = _war()
    cfg = cfg_of(8, 2, 128)
    g = torch.Generator(device=DEV).manual_seed(5)
    B, shared, n = 4, 2048, 3
    pool = war.Pool(cfg, 1024, B, 160, device=DEV, kv_format="e4m3")
    pool.alloc([0], [shared])
    kv = torch.randn((2, 1, shared, 2, 128), device=DEV, generator=g).bfloat16()
    war.kv_write(pool, 0, t32([0]), t32([0]), *kv)
    for b in range(1, B):
        pool.fork(0, b, shared)
    pool.alloc(list(range(B)), [shared + 20 * (b + 1) + n for b in range(B)])
    tails = [torch.randn((2, 1, 20 * (b + 1) + n, 2, 128), device=DEV, generator=g).bfloat16() for b in range(B)]
    for b in range(B):
        war.kv_write(pool, 0, t32([b]), t32([shared]), *tails[b])
    q = torch.randn((B, n, 8, 128), device=DEV, generator=g).bfloat16()
    plan = war.AttendPlan(pool, B, n)
    for rows in ([3, 3, 3, 3], [0, 3, 0, 2]):             # siblings without rows, the first one too
        out = torch.full_like(q, 7.0)
        ctx = [shared + 20 * (b + 1) for b in range(B)]
        plan.update(t32(list(range(B))), t32(ctx), t32(rows))
        war.attend(plan, 0, q, out)
        alone = torch.full_like(q, 7.0)
        one = war.AttendPlan(pool, 1, n)
        for b in range(B):                                 # each by itself: no sharing
            one.update(t32([b]), t32([ctx[b]]), t32([rows[b]]))
            war.attend(one, 0, q[b:b + 1], alone[b:b + 1])
        assert pool.state()["status"] == 0
        for b in range(B):
            want, tol = np.full((n, 8, 128), 7.0), np.zeros((n, 8, 128))
            k, v = (as64(x).transpose(1, 0, 2) for x in pool.gather_kv(b, ctx[b] + n, 0))
            reference("e4m3", as64(q[b]), k, v, ctx[b], rows[b], None, want, tol)
            check(as64(out[b]), want, tol)
            check(as64(alone[b]), want, tol)


def test_plan_refuses_bad_requests_and_writes_nothing():
    war = _war()
    cfg = cfg_of(8, 2, 64)
    for n in (2, 40):
        for bad in (dict(seq=7), dict(seq=-1), dict(seq=0), dict(ctx=-1), dict(ctx=64), dict(ctx=2**31 - 1), dict(n=n + 1),
                    dict(n=-1)):
            pool = scattered_pool(cfg, [64, 64], "e4m3")
            war.kv_write(pool, 0, t32([0, 1]), t32([0, 0]), *torch.ones((2, 2, 64, 2, 64), dtype=torch.bfloat16, device=DEV))
            plan = war.AttendPlan(pool, 2, n)
            q = torch.ones((2, n, 8, 64), dtype=torch.bfloat16, device=DEV)
            out = torch.full_like(q, 7.0)
            plan.update(t32([0, bad.get("seq", 1)]), t32([3, bad.get("ctx", 3)]), t32([n, bad.get("n", n)]))
            war.attend(plan, 0, q, out)
            assert pool.state()["status"] == -5, (n, bad)
            assert (out == 7.0).all(), (n, bad)
            plan.update(t32([0, 1]), t32([3, 3]))          # the next plan is unaffected
            war.attend(plan, 0, q, out)
            assert pool.state()["status"] == 0 and (out == 1.0).all(), (n, bad)


def test_refusals():
    war = _war()
    cfg = cfg_of(8, 2, 64)
    pool = scattered_pool(cfg, [64, 64], "e4m3")
    bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device=DEV)
    ids, pos = t32([0, 1]), t32([0, 0])
    for k in (bf(2, 3, 2, 64).float(), bf(2, 3, 1, 64), bf(2, 3, 2, 128)[..., ::2], bf(3, 2, 2, 64).transpose(0, 1),
              bf(2, 3, 2, 64).cpu()):
        with pytest.raises(ValueError):
            war.kv_write(pool, 0, ids, pos, k, bf(2, 3, 2, 64))
    with pytest.raises(ValueError):
        war.kv_write(pool, 0, ids.long(), pos, bf(2, 3, 2, 64), bf(2, 3, 2, 64))
    with pytest.raises(war.WarError):
        war.kv_write(pool, 1, ids, pos, bf(2, 3, 2, 64), bf(2, 3, 2, 64))                # no such layer
    with pytest.raises(war.WarError):                                                   # rows 2 bytes off
        war.kv_write(pool, 0, ids, pos, bf(2 * 3 * 2 * 64 + 1)[1:].view(2, 3, 2, 64), bf(2, 3, 2, 64))
    with pytest.raises(war.WarError):                                                   # a stride of 130
        war.kv_write(pool, 0, ids, pos, bf(2, 3, 130)[..., :128].unflatten(2, (2, 64)), bf(2, 3, 2, 64))
    with pytest.raises(ValueError):
        war.Pool(cfg, 4, 1, 4, kv_format="int4")
    plan = war.AttendPlan(pool, 2, 40)
    with pytest.raises(ValueError):
        war.attend(plan, 0, bf(2, 40, 8, 64), bf(2, 40, 8, 64))                          # no plan yet
    with pytest.raises(war.WarError):
        plan.update(ids, pos, n_rows=41)
    with pytest.raises(war.WarError) as e:
        plan.update(ids, pos, draft_parents=t32(np.zeros((2, 39))))                      # a tree of 160 rows a kv-head
    assert e.value.status == -4
    with pytest.raises(war.WarError):
        plan.update(t32([0, 1, 0]), t32([0, 0, 0]))
    with pytest.raises(war.WarError):
        war.AttendPlan(pool, 1025, 1)


def test_a_plan_ends_when_pages_are_given_back():
    war = _war()
    cfg = cfg_of(8, 2, 64)
    pool = scattered_pool(cfg, [64, 64], "e4m3")
    ids, ctx = t32([0, 1]), t32([3, 3])
    war.kv_write(pool, 0, ids, t32([0, 0]), *torch.ones((2, 2, 64, 2, 64), dtype=torch.bfloat16, device=DEV))
    plan = war.AttendPlan(pool, 2, 2)
    q = torch.ones((2, 2, 8, 64), dtype=torch.bfloat16, device=DEV)
    out = torch.zeros_like(q)
    plan.update(ids, ctx)
    pool.free([1])
    with pytest.raises(war.WarError) as e:
        war.attend(plan, 0, q, out)
    assert e.value.status == -1
    plan.update(ids[:1], ctx[:1])
    war.attend(plan, 0, q[:1], out[:1])
    assert pool.state()["status"] == 0 and (out[0] == 1.0).all() and (out[1] == 0.0).all()


def test_captured_plans_replay_and_follow_their_inputs():
    war = _war()
    cfg = cfg_of(8, 2, 64)
    g = torch.Generator(device=DEV).manual_seed(9)
    B, S = 3, 300
    pool = scattered_pool(cfg, [S] * B, "e4m3")
    war.kv_write(pool, 0, t32([0, 1, 2]), t32([0] * B), *torch.randn((2, B, S, 2, 64), device=DEV, generator=g).bfloat16())
    for n in (3, 40):
        plans = [war.AttendPlan(pool, B, n) for _ in range(3)]
        ids, ctx = t32([0, 1, 2]), t32([10, 100, 200])
        qs = [torch.randn((B, n, 8, 64), device=DEV, generator=g).bfloat16() for _ in range(2)]
        outs = [torch.zeros_like(q) for q in qs]
        graphs = []
        for plan, q, out in zip(plans, qs, outs):
            graph = torch.cuda.CUDAGraph()
            gc.collect()                                   # (an object freed by a collection would end the capture)
            with torch.cuda.graph(graph):
                plan.update(ids, ctx)
                war.attend(plan, 0, q, out)
            graphs.append(graph)
        for step in range(4):
            ctx += 7
            for graph in graphs:
                graph.replay()
            for q, out in zip(qs, outs):
                want = torch.zeros_like(q)
                plans[2].update(ids, ctx)
                war.attend(plans[2], 0, q, want)
                assert torch.equal(out, want), (n, step)
        assert pool.state()["status"] == 0


@pytest.mark.parametrize("fmt", ["e4m3", "bf16"])
def test_pages_past_32_bit_offsets(fmt):
    """A sequence's pages at both ends of a pool of more than 2^32 bytes (bf16: elements)."""
    war = _war()
    cfg, far = cfg_of(32, 8, 128, layers=2), 70000
    pool = war.Pool(cfg, far, 2, 69990, device=DEV, kv_format=fmt)
    assert 2 * far * 8 * 2 * 16 * 128 > 2 ** 32
    n_ctx, n = 300, 3
    pool.alloc([0], [160])
    pool.alloc([1], [69960 * 16])
    pool.alloc([0], [n_ctx + n])
    used = pool.block_tables[0, :19].tolist()
    assert max(used) - min(used) > 65000
    g = torch.Generator(device=DEV).manual_seed(8)
    kv = torch.randn((2, 1, n_ctx + n, 8, 128), device=DEV, generator=g).bfloat16()
    q = torch.randn((1, 40, 32, 128), device=DEV, generator=g).bfloat16()
    for layer in range(2):
        war.kv_write(pool, layer, t32([0]), t32([0]), *kv.roll(layer, 0))
    back = torch.empty_like(kv)
    want_kv = [e4m3.store_kv(as64(x[0]), as64(y[0])) if fmt == "e4m3" else (as64(x[0]), as64(y[0])) for x, y in
               (kv, kv.roll(1, 0))]
    for rows in (n, 40):
        plan = war.AttendPlan(pool, 1, rows)
        plan.update(t32([0]), t32([n_ctx + n - rows]))
        for layer in range(2):
            war.kv_read(pool, layer, t32([0]), t32([0]), *back)
            for x, w in zip(back, want_kv[layer]):
                np.testing.assert_array_equal(as64(x[0]), w)
            out = torch.full((1, rows, 32, 128), 7.0, dtype=torch.bfloat16, device=DEV)
            war.attend(plan, layer, q[:, :rows].contiguous(), out)
            want, tol = np.zeros((rows, 32, 128)), np.zeros((rows, 32, 128))
            reference(fmt, as64(q[0, :rows]), *want_kv[layer], n_ctx + n - rows, rows, None, want, tol)
            check(as64(out[0]), want, tol)
    assert pool.state()["status"] == 0


def test_the_most_rows_of_a_request_and_the_most_requests():
    war = _war()
    cfg = cfg_of(2, 1, 64)
    g = torch.Generator(device=DEV).manual_seed(12)
    n, ctx = 65536, 37
    pool = war.Pool(cfg, (ctx + n) // 16 + 3, 1, (ctx + n) // 16 + 2, device=DEV, kv_format="e4m3")
    pool.alloc([0], [ctx + n])
    kv = torch.randn((2, 1, ctx + n, 1, 64), device=DEV, generator=g).bfloat16()
    war.kv_write(pool, 0, t32([0]), t32([0]), *kv)
    q = torch.randn((1, n, 2, 64), device=DEV, generator=g).bfloat16()
    plan, out = war.AttendPlan(pool, 1, n), torch.empty_like(q)
    plan.update(t32([0]), t32([ctx]))
    war.attend(plan, 0, q, out)
    k, v = e4m3.store_kv(as64(kv[0, 0]), as64(kv[1, 0]))
    for i in (0, 1, 63, 64, 4095, 40000, 65535):
        want, tol = np.zeros((1, 2, 64)), np.zeros((1, 2, 64))
        reference("e4m3", as64(q[0, i:i + 1]), k, v, ctx + i, 1, None, want, tol)
        check(as64(out[0, i:i + 1]), want, tol)
    B = 1024
    pool = war.Pool(cfg, 3 * B, B, 3, device=DEV, kv_format="e4m3")
    ctx = np.random.default_rng(4).integers(0, 40, B)
    pool.alloc(list(range(B)), [48] * B)
    ids, kv = t32(np.random.default_rng(5).permutation(B)), torch.randn((2, B, 45, 1, 64), device=DEV, generator=g).bfloat16()
    war.kv_write(pool, 0, ids, t32(np.zeros(B)), *kv)
    war.kv_write(pool, 0, ids, t32(np.zeros(B)), *kv[:, :, :0])                  # no rows: nothing
    plan = war.AttendPlan(pool, B, 30)
    rows = np.random.default_rng(6).integers(0, 6, B)
    for m in (5, 30):                                                             # few rows, blocks of rows
        q = torch.randn((B, m, 2, 64), device=DEV, generator=g).bfloat16()
        out = torch.full_like(q, 7.0)
        plan.update(ids, t32(ctx), t32(rows), n_rows=m)
        war.attend(plan, 0, q, out)
        assert pool.state()["status"] == 0
        for b in range(0, B, 73):
            want, tol = np.full((m, 2, 64), 7.0), np.zeros((m, 2, 64))
            reference("e4m3", as64(q[b]), *e4m3.store_kv(as64(kv[0, b]), as64(kv[1, b])), ctx[b], rows[b], None, want, tol)
            check(as64(out[b]), want, tol)


def test_contexts_of_more_chunks_than_a_merge_takes():
    """300000 tokens: 512-key chunks would be 587 partials of a row block, 512 are merged."""
    war = _war()
    cfg, ctx = cfg_of(8, 1, 64), 300000
    pool = war.Pool(cfg, ctx // 16 + 3, 1, ctx // 16 + 3, device=DEV, kv_format="e4m3")
    pool.alloc([0], [ctx + 30])
    g = torch.Generator(device=DEV).manual_seed(14)
    kv = torch.randn((2, 1, ctx + 30, 1, 64), device=DEV, generator=g).bfloat16()
    kv[0, 0, ::50000] *= 6                                                     # keys that stand out in some chunks
    war.kv_write(pool, 0, t32([0]), t32([0]), *kv)
    k, v = e4m3.store_kv(as64(kv[0, 0]), as64(kv[1, 0]))
    for n in (1, 6, 30):
        q = torch.randn((1, n, 8, 64), device=DEV, generator=g).bfloat16()
        plan, out = war.AttendPlan(pool, 1, n), torch.zeros_like(q)
        plan.update(t32([0]), t32([ctx]))
        war.attend(plan, 0, q, out)
        assert pool.state()["status"] == 0
        for i in {0, n - 1}:
            want, tol = np.zeros((1, 8, 64)), np.zeros((1, 8, 64))
            reference("e4m3", as64(q[0, i:i + 1]), k, v, ctx + i, 1, None, want, tol)
            check(as64(out[0, i:i + 1]), want, tol)


def test_an_object_serves_smaller_plans_and_another_stream():
    war = _war()
    cfg = cfg_of(8, 2, 64)
    g = torch.Generator(device=DEV).manual_seed(10)
    pool = scattered_pool(cfg, [200] * 4, "e4m3")
    kv = torch.randn((2, 4, 150, 2, 64), device=DEV, generator=g).bfloat16()
    stream, plan = torch.cuda.Stream(), war.AttendPlan(pool, 4, 50)
    ids, zero = t32(range(4)), t32([0] * 4)
    torch.cuda.synchronize()
    war.kv_write(pool, 0, ids, zero, *kv, stream=stream)
    for B, n in ((4, 50), (1, 1), (2, 13), (3, 12), (4, 2), (1, 50)):            # both kinds of plans in turn
        pos = t32([99] * B)
        q = torch.randn((B, n, 8, 64), device=DEV, generator=g).bfloat16()
        out = torch.zeros_like(q)
        torch.cuda.synchronize()
        plan.update(ids[:B], pos, n_rows=n, stream=stream)
        war.attend(plan, 0, q, out, stream=stream)
        stream.synchronize()
        for b in range(B):
            want, tol = np.zeros((n, 8, 64)), np.zeros((n, 8, 64))
            reference("e4m3", as64(q[b]), *e4m3.store_kv(as64(kv[0, b]), as64(kv[1, b])), 99, n, None, want, tol)
            check(as64(out[b]), want, tol)
    back = torch.zeros_like(kv)
    torch.cuda.synchronize()
    war.kv_read(pool, 0, ids, zero, *back, stream=stream)
    stream.synchronize()
    for b in range(4):
        for x, w in zip(back[:, b], e4m3.store_kv(as64(kv[0, b]), as64(kv[1, b]))):
            np.testing.assert_array_equal(as64(x), w)
    pool.close()
    with pytest.raises(ValueError):
        plan.update(ids, zero)
    with pytest.raises(ValueError):
        war.attend(plan, 0, q, out)


def test_captured_write_attend_and_read_replay():
    """A step of somebody's decoder as one graph, replayed on changing inputs."""
    war = _war()
    cfg = cfg_of(8, 2, 64, layers=2)
    g = torch.Generator(device=DEV).manual_seed(13)
    B, n = 3, 4
    pools = [scattered_pool(cfg, [120] * B, "e4m3") for _ in range(2)]            # replayed, eager
    plans = [war.AttendPlan(p, B, n) for p in pools]
    ids, pos, lens = t32([2, 0, 1]), t32([0] * B), t32([4, 2, 3])
    kv = torch.empty((2, 2, B, n, 2, 64), dtype=torch.bfloat16, device=DEV)
    q = torch.empty((B, n, 8, 64), dtype=torch.bfloat16, device=DEV)
    outs = [torch.zeros((2, B, n, 8, 64), dtype=torch.bfloat16, device=DEV) for _ in pools]
    backs = [torch.zeros_like(kv) for _ in pools]

    def step(i):
        plans[i].update(ids, pos, lens)
        for layer in range(2):
            war.kv_write(pools[i], layer, ids, pos, *kv[layer], lens)
            war.attend(plans[i], layer, q, outs[i][layer])
            war.kv_read(pools[i], layer, ids, pos, *backs[i][layer], lens)

    graph = torch.cuda.CUDAGraph()
    gc.collect()
    with torch.cuda.graph(graph):
        step(0)
    for _ in range(6):
        kv.copy_(torch.randn(kv.shape, device=DEV, generator=g))
        q.copy_(torch.randn(q.shape, device=DEV, generator=g))
        graph.replay()
        step(1)
        assert torch.equal(outs[0], outs[1]) and torch.equal(backs[0], backs[1])
        pos += lens
        lens.copy_(torch.randint(0, n + 1, (B,), device=DEV, generator=g))
    assert [p.state()["status"] for p in pools] == [0, 0]


# ------------------------------------------------------------------- whole steps
CFG = synth.TINY


def near_codes(got, want):
    """Q(a) against the oracle's Q(b): |Q(a) - Q(b)| <= |Q(a) - a| + |a - b| + |b - Q(b)|.  The
    numbers before rounding agree to 2e-2 + 2e-2 |b| (what the bf16 pools' contents are held
    to, test_gpu_edges.py); rounding moves a number by 2^-4 of it or 2^-10 of the scale, under
    2^-17 of the block's largest; |b| <= |Q(b)| / (1 - 2^-4), |a| <= 1.02 |b| + 2e-2."""
    for x, w in zip(got, want):
        b = np.abs(w) / (1 - 2.0 ** -4)
        gap = 2e-2 + 2e-2 * b
        bound = gap + 2.0 ** -4 * (b + gap) + 2.0 ** -4 * b + 2.0 ** -16 * np.abs(w).max(-1, keepdims=True)
        assert (np.abs(x - w) <= bound).all()


WIDE = synth.ModelConfig(n_layers=2, d_model=512, n_q_heads=8, n_kv_heads=2, head_dim=128, ffn_dim=512, vocab=1024)


@pytest.mark.parametrize("wide", [False, True])
def test_a_step_stores_the_bytes_of_its_bf16_keys_and_values(tiny, wide):
    """Layer 0's keys and values do not hang on the cache: a bf16 pool's, written with
    war_kv_write, are an 8-bit pool's bit for bit (an append, and a step's rows)."""
    war, cfg, model = _war(), CFG, tiny["model"]
    if wide:
        cfg = WIDE
        model = war.Model(cfg, {k: v.to(DEV) for k, v in synth.model_weights(cfg, seed=2, norm_std=0.1).items()}, max_rows=128)
    pools = {name: war.Pool(cfg, 32, 2, 16, device=DEV, kv_format=f)
             for name, f in (("bf16", "bf16"), ("e4m3", "e4m3"), ("copy", "e4m3"))}
    toks = t32(np.concatenate([synth.uniform_tokens(31, 61, cfg.vocab), synth.uniform_tokens(32, 7, cfg.vocab)]))
    for f in ("bf16", "e4m3"):
        seq, ctx, nxt, acc = t32([0, 1]), t32([0, 0]), t32([0, 0]), t32([0, 0])
        war.prefill_append(model, pools[f], seq, ctx, [61, 7], toks, nxt)
        war.verify_step(model, pools[f], seq, ctx, t32([3, 4]), t32([[5, 6, 7], [8, 9, 10]]), None, 3, acc, nxt)
        war.kv_commit(pools[f], seq, ctx, t32([3, 2]))
        assert ctx.tolist() == [65, 10]
    for b, n in ((0, 65), (1, 10)):
        k, v = pools["bf16"].gather_kv(b, n, 0)
        pools["copy"].alloc([b], [n])
        war.kv_write(pools["copy"], 0, t32([b]), t32([0]), k.transpose(0, 1).contiguous()[None], v.transpose(0, 1).contiguous()[None])
        assert torch.equal(pools["copy"].gather_kv(b, n, 0), pools["e4m3"].gather_kv(b, n, 0))


@pytest.fixture(scope="module")
def tiny():
    war = _war()
    w_cpu = synth.model_weights(CFG, seed=0, norm_std=0.1)
    return {"model": war.Model(CFG, {k: v.to(DEV) for k, v in w_cpu.items()}, max_rows=256), "W": Weights(CFG, w_cpu)}


def test_prefill_verify_commit_over_an_8_bit_pool(tiny):
    """Two appends and three steps per request; the cache stays within one code of the
    oracle's, the logits within the drift that other summation orders have there."""
    war, model, W = _war(), tiny["model"], tiny["W"]
    B, k = 3, 3
    pool = war.Pool(CFG, 64, B, 16, device=DEV, kv_format="e4m3")
    seq, ctx, nxt = t32(list(range(B))), t32([0] * B), t32([0] * B)
    kvs = [RequestKV(CFG, store=e4m3.store_kv) for _ in range(B)]
    pend = None
    for turn, lens in enumerate(([40, 17, 1], [3, 30, 64])):
        toks = [synth.uniform_tokens(100 * turn + b, lens[b], CFG.vocab) for b in range(B)]
        war.prefill_append(model, pool, seq, ctx, lens, t32(np.concatenate(toks)), nxt)
        pend = [prefill_request(CFG, W, kv, c)["next"] for kv, c in zip(kvs, toks)]
    report = []
    for step in range(3):
        lens = [k, 1, 0] if step == 1 else [k] * B
        drafts = [synth.uniform_tokens(300 + 10 * step + b, k, CFG.vocab).tolist() for b in range(B)]
        for b in range(B):                                  # a prefix that the target accepts
            x = copy.copy(kvs[b])
            p = pend[b]
            for i in range((step + b) % 3):
                r = verify_request(CFG, W, x, p, [])
                commit_request(x, r)
                p = drafts[b][i] = r["next"]
        logits = torch.empty((B * (k + 1), CFG.vocab), device=DEV)
        acc, nx = t32([0] * B), t32([0] * B)
        war.verify_step(model, pool, seq, ctx, t32(pend), t32(drafts), t32(lens), k, acc, nx, logits)
        war.kv_commit(pool, seq, ctx, acc)
        z = logits.cpu().numpy().reshape(B, k + 1, CFG.vocab)
        for b in range(B):
            d = drafts[b][: lens[b]]
            r = verify_request(CFG, W, kvs[b], pend[b], d)
            r32 = verify_request(CFG, W, kvs[b], pend[b], d, precision="fp32")
            compare_request(r["logits"], z[b], d, r["accept"], r["next"], int(acc[b]), int(nx[b]), report, f"{step}/{b}",
                            tol=fp32_drift_tol(r["logits"], r32["logits"]))
            # (a near-tie may go the other way, parity.py: the text is then the GPU's)
            commit_request(kvs[b], r, int(acc[b]))
            pend[b] = int(nx[b])
    assert ctx.tolist() == [kv.length for kv in kvs]
    for b in range(B):
        for layer in range(CFG.n_layers):
            near_codes(as64(pool.gather_kv(b, kvs[b].length, layer)), kvs[b].get(layer))
    assert pool.state()["status"] == 0


def test_appends_behind_long_contexts(tiny):
    """Appends whose contexts are cut into several chunks: new keys and values and the last
    row's logits, as above."""
    war, model, W = _war(), tiny["model"], tiny["W"]
    ctx, lens = [2600, 513, 5000], [70, 30, 5]
    pool = war.Pool(CFG, 540, 3, 330, device=DEV, kv_format="e4m3")
    pool.alloc([0, 1, 2], ctx)
    kvs = []
    for b, c in enumerate(ctx):
        layers = []
        for layer in range(CFG.n_layers):
            x = synth.kv_context(CFG, 6, b, layer, 0, c, DEV)               # [2, Hkv, c, D]
            pool.load(b, layer, 0, x)
            k, v = e4m3.store_kv(*(as64(y.transpose(0, 1)) for y in x))
            layers.append((k.transpose(1, 0, 2), v.transpose(1, 0, 2)))
        kvs.append(RequestKV(CFG, layers, store=e4m3.store_kv))
    toks = [synth.uniform_tokens(500 + b, lens[b], CFG.vocab) for b in range(3)]
    d_ctx, nxt, logits = t32(ctx), t32([0] * 3), torch.empty((3, CFG.vocab), device=DEV)
    war.prefill_append(model, pool, t32([0, 1, 2]), d_ctx, lens, t32(np.concatenate(toks)), nxt, logits)
    assert d_ctx.tolist() == [c + n for c, n in zip(ctx, lens)] and pool.state()["status"] == 0
    for b in range(3):
        first, rest = int(toks[b][0]), [int(t) for t in toks[b][1:]]
        z, z32 = (verify_request(CFG, W, kvs[b], first, rest, precision=p)["logits"] for p in ("fp64", "fp32"))
        assert np.abs(as64(logits[b]) - z[-1]).max() <= fp32_drift_tol(z, z32)
        prefill_request(CFG, W, kvs[b], toks[b])
        for layer in range(CFG.n_layers):
            got = as64(pool.gather_kv(b, ctx[b] + lens[b], layer))
            want = kvs[b].get(layer)
            for x, w in zip(got, want):
                np.testing.assert_array_equal(x[:, : ctx[b]], w[:, : ctx[b]])
            near_codes(got[:, :, ctx[b]:], [w[:, ctx[b]:] for w in want])


def test_tree_step_moves_codes_and_scales(tiny):
    war, model, W = _war(), tiny["model"], tiny["W"]
    pool = war.Pool(CFG, 32, 1, 16, device=DEV, kv_format="e4m3")
    seq, ctx, nxt = t32([0]), t32([0]), t32([0])
    toks = synth.uniform_tokens(7, 45, CFG.vocab)
    war.prefill_append(model, pool, seq, ctx, [45], t32(toks), nxt)
    kv = RequestKV(CFG, store=e4m3.store_kv)
    p = prefill_request(CFG, W, kv, toks)["next"]
    x, path = copy.copy(kv), []
    y = p
    for _ in range(2):
        r = verify_request(CFG, W, x, y, [])
        commit_request(x, r)
        y = r["next"]
        path.append(y)
    drafts, parents = [11, path[0], 12, path[1], 13], [0, 0, 1, 2, 4]      # accepted: nodes 2 and 4
    logits = torch.empty((6, CFG.vocab), device=DEV)
    acc, nx, ap = t32([0]), t32([0]), t32([[0] * 5])
    war.verify_step_tree(model, pool, seq, ctx, t32([p]), t32([drafts]), t32([parents]), None, 5, acc, nx, ap, logits)
    war.kv_commit(pool, seq, ctx, acc)
    o = verify_tree_request(CFG, W, kv, p, drafts, parents)
    report = []
    a = int(acc[0])
    assert compare_tree_request(o, logits.cpu().numpy(), [p] + drafts, parents, a, int(nx[0]), ap[0, :a].tolist(), report, "tree")
    assert o["path"] == [2, 4] and ctx.item() == 48
    commit_request(kv, o)
    # the moved tokens read as a chain of the same tokens stores them, but for bf16 roundings
    for layer in range(CFG.n_layers):
        near_codes(as64(pool.gather_kv(0, 48, layer)), kv.get(layer))


def test_rejected_drafts_leave_no_trace(tiny):
    """A step whose drafts are all discarded, then the same tokens as one without it."""
    war, model = _war(), tiny["model"]
    kept = []
    for drafts in (None, [[4000, 3999, 17, 18, 19, 20, 21]]):
        pool = war.Pool(CFG, 32, 1, 16, device=DEV, kv_format="e4m3")
        pool.kv.fill_(0)
        seq, ctx, nxt = t32([0]), t32([0]), t32([0])
        war.prefill_append(model, pool, seq, ctx, [27], t32(synth.uniform_tokens(8, 27, CFG.vocab)), nxt)
        acc, nx = t32([0]), t32([0])
        if drafts:
            war.verify_step(model, pool, seq, ctx, t32([5]), t32(drafts), None, 7, acc, nx)
            war.kv_commit(pool, seq, ctx, t32([-1]))
        for tok in (5, 6, 7):
            war.verify_step(model, pool, seq, ctx, t32([tok]), None, None, 0, acc, nx)
            war.kv_commit(pool, seq, ctx, t32([0]))
        kept.append([pool.gather_kv(0, 30, layer) for layer in range(CFG.n_layers)])
    for a, b in zip(*kept):
        assert torch.equal(a, b)


def test_noalloc_and_sampled_steps_agree_with_the_plain_step(tiny):
    war, model = _war(), tiny["model"]
    B, k = 2, 3
    toks = [synth.uniform_tokens(60 + b, 50, CFG.vocab) for b in range(B)]
    res = []
    for step in ("plain", "noalloc", "sampled"):
        pool = war.Pool(CFG, 32, B, 16, device=DEV, kv_format="e4m3")
        seq, ctx, nxt = t32(list(range(B))), t32([0] * B), t32([0] * B)
        war.prefill_append(model, pool, seq, ctx, [50] * B, t32(np.concatenate(toks)), nxt)
        acc, nx, z = t32([0] * B), t32([0] * B), torch.empty((B * (k + 1), CFG.vocab), device=DEV)
        drafts = t32([[1, 2, 3], [4, 5, 6]])
        if step == "sampled":                              # top-k 1: the greedy token
            war.verify_step_sampled(model, pool, seq, ctx, nxt, drafts, None, k, torch.full((B * (k + 1), 2), 0.5, device=DEV),
                                    1.0, 1, acc, nx, z)
        else:
            (war.verify_step if step == "plain" else war.verify_step_noalloc)(model, pool, seq, ctx, nxt, drafts, None, k, acc,
                                                                              nx, z)
        war.kv_commit(pool, seq, ctx, acc)
        res.append((acc.tolist(), nx.tolist(), z.clone()))
    for r in res[1:]:
        assert r[:2] == res[0][:2] and torch.equal(r[2], res[0][2])


@pytest.mark.parametrize("n", [4, 30])
def test_a_value_that_reads_as_infinite_reaches_only_the_rows_that_see_it(n):
    """Above 1.9375 * 2^127 a finite number's code stands for 2^128.  Two heads' worth of
    rows, row 2's own token; all keys in one 32-key block, or in two."""
    def spoil(b, k, v):
        v[0, 12 + b, 0, 3] = 1.96 * 2.0 ** 127
        v[0, 12 + b, 1, 40] = -1.96 * 2.0 ** 127
    got, want, tol = attend_case("e4m3", (8, 2, 64), n, [10, 11], [n, n], spoil=spoil)
    for b, first in ((0, 2), (1, 2)):
        assert np.isfinite(got[b, :first]).all()
        check(got[b, :first], want[b, :first], tol[b, :first])
        for h, d in ((0, 3), (1, 40)):
            heads = slice(4 * h, 4 * h + 4)
            other = np.delete(np.arange(64), d)
            seen = got[b, first:, heads, d]
            assert not np.isnan(seen).any() and (np.sign(seen) == (-1) ** h).all()
            sub = np.ix_(np.arange(first, n), np.arange(4 * h, 4 * h + 4), other)
            check(got[b][sub], want[b][sub], tol[b][sub])


@pytest.mark.parametrize("heads", [(4, 2, 64), (16, 2, 128)])
@pytest.mark.parametrize("fmt", ["e4m3", "bf16"])
def test_an_import_may_begin_at_any_element(heads, fmt):
    cfg = cfg_of(*heads)
    n = 37
    g = torch.Generator(device=DEV).manual_seed(4)
    flat = torch.randn(2 * cfg.n_kv_heads * n * cfg.head_dim + 8, device=DEV, generator=g).bfloat16()
    for at in (0, 1, 2, 3, 5, 7):
        src = flat[at: at + flat.numel() - 8].view(2, cfg.n_kv_heads, n, cfg.head_dim)
        assert src.data_ptr() % 16 == 2 * at
        pools = [scattered_pool(cfg, [n + 5], fmt) for _ in range(2)]
        pools[0].load(0, 0, 5, src)
        pools[1].load(0, 0, 5, src.clone())
        assert torch.equal(pools[0].kv.view(torch.uint8), pools[1].kv.view(torch.uint8))

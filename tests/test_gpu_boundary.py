"""GPU checks of the boundary's failure handling on the tiny decoder.

* A verify step whose device-side inputs are bad (a sequence id repeated in
  the batch, or one request past its block-table row) fails as a whole: no
  page moves, every accept length and next token is -1, the following commit
  changes nothing whatever accept lengths it is given, and war_pool_state
  reports WAR_ERR_DEVICE once, then clears the flag.
* A steady verify/commit loop never waits for the device to learn how many
  pages are free: the commit kernel's report keeps the host's lower bound up.
All failure conditions are plain inputs that the kernels' own checks turn
into flags; every kernel runs to completion.
"""
import numpy as np
import pytest
import torch

from paper_2607_17299_amd import synth

pytestmark = pytest.mark.gpu
CFG = synth.TINY
DEV = "cuda"


def _war():
    from paper_2607_17299_amd import war
    return war


@pytest.fixture(scope="module")
def tiny():
    war = _war()
    w = {k: v.to(DEV) for k, v in synth.model_weights(CFG, seed=0, norm_std=0.1).items()}
    return war, war.Model(CFG, w, max_rows=64)


def _t(a):
    return torch.as_tensor(np.asarray(a), dtype=torch.int32).to(DEV)


def _prefilled(war, model, lens, num_pages=64, max_pages=8):
    B = len(lens)
    pool = war.Pool(CFG, num_pages, B + 1, max_pages)
    ctx = _t([0] * B)
    toks = _t(np.concatenate([synth.uniform_tokens(300 + b, n, CFG.vocab) for b, n in enumerate(lens)]))
    nxt = _t([0] * B)
    war.prefill_append(model, pool, _t(range(B)), ctx, list(lens), toks, nxt)
    torch.cuda.synchronize()
    return pool, ctx, nxt


def _snapshot(pool):
    st = pool.state()
    assert st["status"] == 0
    return {k: st[k].copy() for k in ("stack", "refcount", "held", "base", "table")}


def _flagged(war, pool, words):
    """war_pool_state reports the device's flag once (WAR_ERR_DEVICE)."""
    st = pool.state()
    assert st["status"] == -5
    assert words in war.lib().war_last_error().decode()


def _same(a, b):
    for k in a:
        np.testing.assert_array_equal(a[k], b[k], err_msg=k)


def _failed_step(war, model, pool, seq, ctx, last, k, commit_with):
    B = seq.numel()
    drafts = _t(np.arange(B * k).reshape(B, k) % CFG.vocab)
    acc, nxt = _t([7] * B), _t([7] * B)
    ctx_before = ctx.cpu().tolist()
    war.verify_step(model, pool, seq, ctx, last, drafts, None, k, acc, nxt)
    war.kv_commit(pool, seq, ctx, acc if commit_with is None else _t(commit_with))
    torch.cuda.synchronize()
    assert acc.cpu().tolist() == [-1] * B
    assert nxt.cpu().tolist() == [-1] * B
    assert ctx.cpu().tolist() == ctx_before


@pytest.mark.parametrize("commit_with", [None, [3, 3, 3]])
def test_repeated_sequence_id_fails_the_step(tiny, commit_with):
    war, model = tiny
    pool, ctx, nxt = _prefilled(war, model, [40, 37, 50])
    before = _snapshot(pool)
    seq = _t([0, 1, 0])
    _failed_step(war, model, pool, seq, ctx, nxt, 4, commit_with)
    _flagged(war, pool, "twice")
    _same(before, _snapshot(pool))                     # flag cleared, nothing moved
    # the pool still works: a valid step on the same sequences
    acc, nx = _t([0] * 3), _t([0] * 3)
    seq = _t([0, 1, 2])
    war.verify_step(model, pool, seq, ctx, nxt, _t([[1, 2]] * 3), None, 2, acc, nx)
    war.kv_commit(pool, seq, ctx, _t([-1] * 3))
    torch.cuda.synchronize()
    assert min(acc.cpu().tolist()) >= 0
    _same(before, _snapshot(pool))


@pytest.mark.parametrize("commit_with", [None, [4, 4, 4]])
def test_request_past_its_block_table_fails_the_step(tiny, commit_with):
    """max_pages_per_seq = 4 (64 slots): request 1 has 60 cached tokens, so
    60 + 4 drafts + 1 > 64 fails the whole batch."""
    war, model = tiny
    pool, ctx, nxt = _prefilled(war, model, [20, 60, 33], max_pages=4)
    before = _snapshot(pool)
    _failed_step(war, model, pool, _t([0, 1, 2]), ctx, nxt, 4, commit_with)
    _flagged(war, pool, "context length")
    _same(before, _snapshot(pool))


def test_bad_sequence_id_fails_the_step(tiny):
    war, model = tiny
    pool, ctx, nxt = _prefilled(war, model, [20, 30])
    before = _snapshot(pool)
    _failed_step(war, model, pool, _t([0, 99]), ctx, nxt, 2, [1, 1])
    _flagged(war, pool, "sequence id")
    _same(before, _snapshot(pool))


def test_steady_loop_never_waits_for_the_free_count(tiny):
    """4 requests x k = 4 reserve at most 4 pages per step; the pool has 40
    free pages, so a bound that only fell would need an exact read within 10
    steps.  Over 60 steps (each followed by a host synchronisation, so that
    the commit report is current) no verify step reads the exact count."""
    war, model = tiny
    pool, ctx, nxt = _prefilled(war, model, [20, 30, 16, 45], num_pages=48)
    seq = _t(range(4))
    acc, nx = _t([0] * 4), _t([0] * 4)
    drafts = _t(np.arange(16).reshape(4, 4))
    free0 = pool.state()["stack"].size
    assert free0 == 48 - (2 + 2 + 1 + 3)
    w0 = pool.waits()
    for _ in range(60):
        war.verify_step(model, pool, seq, ctx, nxt, drafts, None, 4, acc, nx)
        war.kv_commit(pool, seq, ctx, _t([-1] * 4))
        torch.cuda.synchronize()
    assert pool.waits() == w0
    assert pool.state()["stack"].size == free0


@pytest.mark.parametrize("far", [2**31 - 1, 2**31 - 2, 2**31 - 5, 2**31 - 17, 2**30])
@pytest.mark.parametrize("k", [0, 3])
def test_the_largest_context_lengths_fail_the_step(tiny, far, k):
    """ctx + drafts + 1 passes 2^31: chain, tree, sampled, noalloc and constrained steps."""
    war, model = tiny
    pool, ctx, nxt = _prefilled(war, model, [20, 30])
    before = _snapshot(pool)
    seq, bad = _t([0, 1]), _t([20, far])
    drafts = _t(np.arange(2 * k).reshape(2, k) % CFG.vocab) if k else None
    parents = _t([list(range(k))] * 2) if k else None
    u = torch.zeros((2 * (k + 1), 2), device=DEV)
    cons = war.Constraints(CFG.vocab, repetition=torch.ones(3, device=DEV))
    steps = {
        "chain": lambda acc, out: war.verify_step(model, pool, seq, bad, nxt, drafts, None, k, acc, out),
        "sampled": lambda acc, out: war.verify_step_sampled(model, pool, seq, bad, nxt, drafts, None, k, u, 1.0, 5, acc, out),
        "noalloc": lambda acc, out: war.verify_step_noalloc(model, pool, seq, bad, nxt, drafts, None, k, acc, out),
        "constrained": lambda acc, out: war.verify_step_constrained(model, pool, seq, bad, nxt, drafts, None, k, cons, acc, out),
    }
    if k:
        steps["tree"] = lambda acc, out: war.verify_step_tree(model, pool, seq, bad, nxt, drafts, parents, None, k, acc, out,
                                                              _t(np.zeros((2, k))))
    for name, step in steps.items():
        acc, out = _t([7, 7]), _t([7, 7])
        step(acc, out)
        war.kv_commit(pool, seq, bad, acc)
        torch.cuda.synchronize()
        assert acc.cpu().tolist() == [-1, -1] and out.cpu().tolist() == [-1, -1], name
        assert bad.cpu().tolist() == [20, far], name
        _flagged(war, pool, "context length")
        _same(before, _snapshot(pool))


@pytest.mark.parametrize("sampled", [False, True])
def test_a_step_without_memory_for_its_logits_leaves_the_pool_alone(sampled):
    """1024 requests of 16 rows, 8,000,000 ids: 524 GB of logits that the caller does not
    bring; no page is reserved, and the next step runs."""
    war = _war()
    cfg = synth.ModelConfig(n_layers=1, d_model=128, n_q_heads=2, n_kv_heads=2, head_dim=64, ffn_dim=128, vocab=8000000)
    w = {name: torch.zeros(shape, dtype=torch.bfloat16, device=DEV) for name, shape in synth.weight_shapes(cfg)}
    model = war.Model(cfg, w, max_rows=16384)
    del w
    B, k = 1024, 15
    pool = war.Pool(cfg, B + 1, B, 2)
    before = _snapshot(pool)
    cons = war.Constraints(cfg.vocab, repetition=torch.ones(B, device=DEV))

    def step(B, k):
        seq, ctx, last, drafts = _t(np.arange(B)), _t([0] * B), _t([1] * B), _t(np.ones((B, k)))
        acc, nxt = _t([7] * B), _t([7] * B)
        u = torch.zeros((B * (k + 1), 2), device=DEV)
        if sampled:
            war.verify_step_sampled(model, pool, seq, ctx, last, drafts, None, k, u, 1.0, 1, acc, nxt)
        else:
            war.verify_step_constrained(model, pool, seq, ctx, last, drafts, None, k, cons, acc, nxt)
        return seq, ctx, acc

    with pytest.raises(war.WarError, match="memory"):
        step(B, k)
    torch.cuda.synchronize()
    _same(before, _snapshot(pool))
    seq, ctx, acc = step(1, 0)
    war.kv_commit(pool, seq, ctx, acc)
    assert acc.cpu().tolist() == [0] and ctx.cpu().tolist() == [1]
    assert pool.state()["status"] == 0
    pool.close()
    model.close()
    torch.cuda.empty_cache()


def test_a_step_whose_workspace_does_not_fit_leaves_the_model_usable():
    """1024 requests of 48 rows over block tables of 2^24 tokens want 412 GB of partial sums."""
    war = _war()
    cfg = synth.ModelConfig(n_layers=1, d_model=128, n_q_heads=32, n_kv_heads=32, head_dim=128, ffn_dim=128, vocab=128)
    w = {name: t.to(DEV) for name, t in synth.model_weights(cfg, seed=0, norm_std=0.1).items()}
    model = war.Model(cfg, w, max_rows=1024 * 48)
    small = war.Pool(cfg, 8, 1, 4)

    def step(pool, B, k):
        acc, nxt = _t([7] * B), _t([7] * B)
        logits = torch.empty((B * (k + 1), cfg.vocab), device=DEV)
        war.verify_step(model, pool, _t(np.arange(B)), _t([0] * B), _t([1] * B), _t(np.ones((B, k))), None, k, acc, nxt, logits)
        war.kv_commit(pool, _t(np.arange(B)), _t([0] * B), _t([-1] * B))
        return logits

    first = step(small, 1, 3)
    large = war.Pool(cfg, 1024 * 3, 1024, 1 << 20)
    with pytest.raises(war.WarError, match="memory"):
        step(large, 1024, 47)
    assert bool((large.block_tables == -1).all())                     # no page moved
    assert torch.equal(first, step(small, 1, 3))
    large.close()
    small.close()
    model.close()
    del large
    torch.cuda.empty_cache()


def test_a_pool_made_on_another_stream_waits_for_its_memory():
    """Memory that the current stream still reads, freed there and taken for the pool's block
    tables, is not cleared before that reading."""
    war = _war()
    n = 4096 * 32768                                         # int32: as large as the block tables below
    other = torch.cuda.Stream()
    for _ in range(3):
        torch.cuda.synchronize()
        torch.cuda.empty_cache()
        x = torch.full((n,), 9, dtype=torch.int32, device=DEV)
        y = torch.empty_like(x)
        torch.cuda.synchronize()
        torch.cuda._sleep(40_000_000)
        y.copy_(x)                                           # waits behind the sleep
        at = x.data_ptr()
        del x
        pool = war.Pool(CFG, 8, 4096, 32768, stream=other)
        torch.cuda.synchronize()
        assert pool.block_tables.data_ptr() == at            # (the allocator gave it that memory)
        assert (y == 9).all()
        pool.close()
        del pool, y

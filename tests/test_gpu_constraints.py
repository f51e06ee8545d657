"""Constrained logits, their greedy tokens, token counts and verify steps under
constraints, against the float64 oracle."""
import gc

import numpy as np
import pytest
import torch

from oracle import constraints as oc
from oracle.sampling import verify_sampled
from oracle.verify import tree_path
from paper_2607_17299_amd import synth

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _war():
    from paper_2607_17299_amd import war
    return war


def t32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)


def f32(a):
    return torch.tensor(np.asarray(a), dtype=torch.float32, device=DEV)


def bits_of(allowed):
    """bool [m, V] -> int32 [m, ceil(V / 32)]."""
    m, V = allowed.shape
    pad = np.zeros((m, -(-V // 32) * 32), bool)
    pad[:, :V] = allowed
    return torch.from_numpy(np.packbits(pad, axis=1, bitorder="little").view(np.int32).copy()).to(DEV)


def table_of(u16):
    return torch.from_numpy(u16.view(np.int16).copy()).to(DEV)


class Case:
    """Seeded constraints of S sequences and a step's tokens; everything that can go wrong
    is in them: ids outside the vocabulary, the same id twice, empty masks, NaN and
    infinities where the mask excludes them and where it does not."""

    def __init__(self, V, B, k, seed, tree=False, n_bias=5, masks=True, S=None, odd=True):
        rng = np.random.default_rng(seed)
        self.V, self.B, self.k, S = V, B, k, S or B + 1
        self.S = S
        self.seq = rng.permutation(S)[:B]
        self.table = np.zeros((S, V), np.uint16)
        for s in range(S):
            at = rng.integers(0, V, min(V, 50))
            self.table[s, at] = rng.integers(0, 65536, at.size)
        self.last = rng.integers(0, V, B)
        self.drafts = rng.integers(0, V, (B, max(k, 1)))
        if k >= 2:
            self.drafts[:, 1] = self.drafts[:, 0]                     # the same token twice
            self.drafts[0, 0] = self.last[0]
        self.lens = rng.integers(0, k + 1, B)
        self.lens[-1] = k
        self.parents = [[int(rng.integers(0, i + 1)) for i in range(k)] for _ in range(B)] if tree and k else None
        self.rep = (1 + rng.random(S) * 0.5).astype(np.float32)
        self.freq = rng.standard_normal(S).astype(np.float32)
        self.pres = rng.standard_normal(S).astype(np.float32)
        self.bid = rng.integers(0, V, (S, n_bias))
        self.bval = (rng.standard_normal((S, n_bias)) * 3).astype(np.float32)
        if n_bias >= 4:
            self.bid[:, 2] = self.bid[:, 0]
            self.bid[:, 3] = [V, -1, 2**31 - 1][seed % 3]
        R = B * (k + 1)
        self.z = (rng.standard_normal((R, V)) * 4).astype(np.float32)
        if odd:
            self.z[rng.integers(0, R, 3), rng.integers(0, V, 3)] = [np.inf, -np.inf, np.nan]
            self.z[0, :] = -np.inf
            self.last[B // 2] = [V, -1][seed % 2]
        m = 4
        self.allowed = rng.random((m, V)) < 0.5
        self.allowed[1] = False
        self.allowed[2] = False
        self.allowed[2, rng.integers(0, V)] = True
        self.index = rng.integers(-1, m + 1, R) if masks else None
        if masks:
            self.index[0] = 1

    def constraints(self):
        war = _war()
        kw = dict(counts=table_of(self.table), repetition=f32(self.rep), frequency=f32(self.freq), presence=f32(self.pres))
        if self.bid.shape[1]:
            kw.update(bias_ids=t32(self.bid), bias_values=f32(self.bval))
        if self.index is not None:
            kw.update(masks=bits_of(self.allowed), mask_index=t32(self.index))
        return war.Constraints(self.V, **kw)

    def allowed_row(self, r):
        if self.index is None or self.index[r] < 0:
            return np.ones(self.V, bool)
        return self.allowed[self.index[r]] if self.index[r] < len(self.allowed) else np.zeros(self.V, bool)

    def oracle_row(self, b, i, z):
        s, r = self.seq[b], b * (self.k + 1) + i
        text = oc.row_tokens(int(self.last[b]), self.drafts[b, : self.k].tolist(), self.parents[b] if self.parents else None, i)
        row = self.table[s]
        return oc.constrain(z, row & 0x7FFF, row >= 0x8000, text, float(self.rep[s]), float(self.freq[s]), float(self.pres[s]),
                            list(zip(self.bid[s].tolist(), self.bval[s].astype(np.float64).tolist())), self.allowed_row(r))

    def bound_row(self, b, i):
        """Each of the operations (a sum of up to n_bias + 1 numbers, a product or quotient,
        a product and two differences) rounds by 2^-24 of a number no larger than this."""
        s, r = self.seq[b], b * (self.k + 1) + i
        big = np.abs(self.z[r].astype(np.float64))
        for t, by in zip(self.bid[s], self.bval[s]):
            if 0 <= t < self.V:
                big[t] += abs(float(by))
        n = (self.table[s] & 0x7FFF).astype(np.float64) + self.k + 1
        return (self.bid.shape[1] + 5) * 2.0 ** -24 * (big * 1.5 + abs(float(self.freq[s])) * n + abs(float(self.pres[s])))


def run_case(c, out=None, z=None, stream=None):
    war = _war()
    R = c.B * (c.k + 1)
    z = f32(c.z) if z is None else z
    out = torch.full((R, c.V), 123.0, device=DEV) if out is None else out
    greedy = torch.full((R,), 77, dtype=torch.int32, device=DEV)
    war.constrain_logits(z, c.constraints(), t32(c.seq), t32(c.last), t32(c.drafts[:, : c.k]) if c.k else None, t32(c.lens), c.k,
                         out=out, greedy=greedy, draft_parents=t32(c.parents) if c.parents else None)
    return out, greedy.cpu().numpy()


def check_case(c, out, greedy, untouched=123.0):
    got = out.cpu().numpy().astype(np.float64)
    for b in range(c.B):
        for i in range(c.k + 1):
            r = b * (c.k + 1) + i
            if i > c.lens[b]:
                assert greedy[r] == 77
                if untouched is not None:
                    assert (got[r] == untouched).all()
                continue
            want, ok = c.oracle_row(b, i, c.z[r]), c.allowed_row(r)
            assert (np.isnan(got[r]) == np.isnan(want)).all(), (b, i)
            fine = np.isfinite(want)
            np.testing.assert_array_equal(got[r][~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)])
            with np.errstate(invalid="ignore"):
                assert (np.abs(got[r] - want)[fine] <= c.bound_row(b, i)[fine]).all(), (b, i)
            assert greedy[r] == oc.greedy(got[r], ok), (b, i)
            w = oc.greedy(want, ok)
            assert (greedy[r] == -1) == (w == -1)
            if w >= 0 and greedy[r] != w:                             # only within the rounding
                tol = c.bound_row(b, i)
                assert want[w] - want[greedy[r]] <= tol[w] + tol[greedy[r]]


@pytest.mark.parametrize("V,B,k,tree,n_bias", [
    (1, 1, 0, False, 0), (3, 2, 1, False, 5), (31, 3, 2, True, 5), (128, 1, 0, False, 4), (129, 2, 3, False, 300),
    (2047, 2, 0, False, 5), (2048, 2, 5, True, 5), (2052, 3, 1, False, 0), (4096, 4, 3, False, 1024), (50257, 2, 2, False, 5),
    (151936, 3, 2, True, 7)])
def test_constrained_logits_and_greedy_tokens(V, B, k, tree, n_bias):
    for seed in range(3):
        c = Case(V, B, k, seed, tree, n_bias)
        check_case(c, *run_case(c))


def test_rows_of_63_drafts():
    c = Case(300, 2, 63, 5, tree=True)
    check_case(c, *run_case(c))


def test_in_place_strided_and_unaligned_rows():
    for V, pad, off in ((4096, 4, 4), (4096, 3, 0), (4096, 4, 1), (1000, 0, 0)):
        c = Case(V, 3, 2, 11)
        R = 9
        base = torch.full((R * (V + pad) + off,), 55.0, device=DEV)
        z = base[off:].view(R, V + pad)[:, :V]
        z.copy_(f32(c.z))
        _, greedy = run_case(c, out=z, z=z)
        got = z.clone()
        want, g2 = run_case(c)
        np.testing.assert_array_equal(greedy, g2)
        for b in range(3):
            for i in range(3):
                r = 3 * b + i
                ref = want[r] if i <= c.lens[b] else f32(c.z[r])
                assert torch.equal(torch.nan_to_num(got[r], 1e9), torch.nan_to_num(ref, 1e9))
        assert (base[off:].view(R, V + pad)[:, V:] == 55.0).all() and (base[:off] == 55.0).all()


def test_parts_that_are_absent_do_nothing():
    war = _war()
    V, B, k = 512, 2, 1
    z = torch.randn((4, V), device=DEV)
    seq, last, drafts = t32([1, 0]), t32([3, 4]), t32([[5], [6]])
    out, greedy = torch.empty_like(z), torch.empty(4, dtype=torch.int32, device=DEV)
    one = lambda x: f32([x, x])
    war.constrain_logits(z, war.Constraints(V, repetition=one(1.0)), seq, last, drafts, None, k, out=out, greedy=greedy)
    assert torch.equal(out, z) and torch.equal(greedy.long(), z.argmax(-1))
    # without a counts table the pending token and the drafts count
    war.constrain_logits(z, war.Constraints(V, presence=one(2.0)), seq, last, drafts, None, k, out=out)
    want = z.clone()
    for r, toks in enumerate(([3], [3, 5], [4], [4, 6])):
        want[r, toks] -= 2.0
    assert torch.equal(out, want)
    masks = torch.full((4, V // 32), -1, dtype=torch.int32, device=DEV)
    masks[2] = 0
    war.constrain_logits(z, war.Constraints(V, masks=masks, n_seqs=2), seq, last, drafts, None, k, greedy=greedy)
    assert greedy.tolist() == [int(z[0].argmax()), int(z[1].argmax()), -1, int(z[3].argmax())]


def test_a_request_outside_the_tables_has_no_token():
    war = _war()
    c = Case(700, 3, 1, 2, odd=False)
    c.seq = np.array([c.S, -1, 0])
    out, greedy = torch.full((6, 700), 9.0, device=DEV), torch.zeros(6, dtype=torch.int32, device=DEV)
    war.constrain_logits(f32(c.z), c.constraints(), t32(c.seq), t32(c.last), t32(c.drafts[:, :1]), None, 1, out=out, greedy=greedy)
    assert greedy[:4].tolist() == [-1] * 4 and (out[:4] == 9.0).all() and (out[4:] != 9.0).all()


@pytest.mark.parametrize("V", [1, 33, 16384, 16385, 50257])
def test_counts_begin_and_add(V):
    war = _war()
    rng = np.random.default_rng(V)
    S, B, n = 5, 3, 9
    table = rng.integers(0, 65536, (S, V)).astype(np.uint16)
    gpu = table_of(table)
    seq = np.array([4, 1, 2])
    prompts = [rng.integers(0, V, m).tolist() for m in (0, 1, 400)]
    prompts[2][:3] = [-1, V, 2**31 - 1]
    off = np.cumsum([0] + [len(p) for p in prompts])
    toks = np.concatenate([np.array(p, np.int64) for p in prompts])
    war.counts_begin(gpu, t32(seq), t32(toks), t32(off))
    for s, p in zip(seq, prompts):
        oc.begin(table, s, p)
    np.testing.assert_array_equal(gpu.cpu().numpy().view(np.uint16), table)
    # commits: chains with repeated and bad tokens, one discarded, one at the largest count
    last, drafts = rng.integers(0, V, B), rng.integers(0, min(V, 4), (B, n))
    drafts[0, 2] = V
    top = int(drafts[2, 0])
    table[2, top] = 0xFFFD
    gpu[2, top] = -3
    for lens in ([4, -1, n], [0, n, n], None):
        war.counts_add(gpu, t32(seq), t32(last), t32(drafts), None if lens is None else t32(lens))
        for b, s in enumerate(seq):
            m = n if lens is None else lens[b]
            if m >= 0:
                oc.add(table, s, [int(last[b])] + drafts[b, :m].tolist())
        np.testing.assert_array_equal(gpu.cpu().numpy().view(np.uint16), table)
    path = np.array([[3, 5, 9, -1, 0, 10, 1, 1, 1]] * B)
    war.counts_add(gpu, t32(seq), None, t32(drafts), t32([3, 6, 0]), t32(path))
    for b, m in enumerate((3, 6, 0)):
        oc.add(table, seq[b], [int(drafts[b, p - 1]) for p in path[b, :m] if 1 <= p <= n])
    np.testing.assert_array_equal(gpu.cpu().numpy().view(np.uint16), table)


def test_counts_begin_reads_no_token_outside_its_array():
    war = _war()
    V, toks = 64, [1, 2, 3, 4, 5]
    for off, want in (([-7, 2], [1, 2]), ([3, 2**31 - 1], [4, 5]), ([5, 9], []), ([4, 1], []), ([0, 5], toks)):
        gpu = torch.full((1, V), 77, dtype=torch.int16, device=DEV)
        war.counts_begin(gpu, t32([0]), t32(toks), t32(off))
        assert (gpu[0] != 0).nonzero().flatten().tolist() == want and (gpu[0, want] == -32768).all()


def test_another_stream():
    """The calls go to the given stream, in order there; their temporary memory lives as long."""
    war = _war()
    c = Case(50257, 4, 3, 9)
    want, g0 = run_case(c)
    s = torch.cuda.Stream()
    z, cons, args = f32(c.z), c.constraints(), (t32(c.seq), t32(c.last), t32(c.drafts[:, :3]), t32(c.lens))
    out, greedy = torch.full_like(z, 123.0), torch.full((16,), 77, dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    war.constrain_logits(z, cons, *args, 3, out=out, greedy=greedy, stream=s)
    junk = [torch.full((1 << 20,), -1, dtype=torch.uint8, device=DEV) for _ in range(8)]   # on the current stream
    s.synchronize()
    assert torch.equal(torch.nan_to_num(out, 1e9), torch.nan_to_num(want, 1e9)) and greedy.tolist() == g0.tolist() and junk


def test_captured_constraints_and_counts_replay():
    """Constrain, count what was taken, constrain again: replays against eager calls."""
    war = _war()
    c = Case(5000, 3, 4, 21, odd=False)
    kw = dict(repetition=f32(c.rep), frequency=f32(c.freq), presence=f32(c.pres), bias_ids=t32(c.bid), bias_values=f32(c.bval),
              masks=bits_of(c.allowed), mask_index=t32(c.index))
    prompt, off = t32([1, 2, 3, 4999, 0, 7]), t32([0, 2, 2, 6])
    seq, last, drafts, lens = t32(c.seq), t32(c.last), t32(c.drafts), t32([4, 0, 3])
    z = f32(c.z)
    tables = [torch.full((c.S, c.V), 5, dtype=torch.int16, device=DEV) for _ in range(2)]
    cons = [war.Constraints(c.V, counts=t, **kw) for t in tables]
    outs = [torch.full((15, c.V), 123.0, device=DEV) for _ in range(2)]
    greedy = [torch.full((15,), 77, dtype=torch.int32, device=DEV) for _ in range(2)]
    work = torch.empty(war.lib().war_constrain_workspace(15, c.V), dtype=torch.uint8, device=DEV)

    def step(i, workspace=None):
        war.counts_add(tables[i], seq, last, drafts, lens)
        war.constrain_logits(z, cons[i], seq, last, drafts, lens, 4, out=outs[i], greedy=greedy[i], workspace=workspace)

    for i in range(2):
        war.counts_begin(tables[i], seq, prompt, off)
    graph = torch.cuda.CUDAGraph()
    gc.collect()
    with torch.cuda.graph(graph):
        step(0, work)
    g = torch.Generator(device=DEV).manual_seed(2)
    for _ in range(5):
        z.copy_(torch.randn(z.shape, device=DEV, generator=g) * 4)
        drafts.copy_(torch.randint(0, 40, drafts.shape, device=DEV, generator=g))
        lens.copy_(torch.randint(-1, 5, (3,), device=DEV, generator=g))
        graph.replay()
        step(1)
        assert torch.equal(tables[0], tables[1]) and torch.equal(outs[0], outs[1]) and torch.equal(greedy[0], greedy[1])
    counted = (tables[0].long() & 0x7FFF).sum(1)                # (the rows that began started at 0)
    rest = [s for s in range(c.S) if s not in c.seq]
    assert (counted[seq.long()] > 0).all() and (counted[rest] == 5 * c.V).all()


# ------------------------------------------------------------------- whole steps
CFG = synth.TINY


@pytest.fixture(scope="module")
def tiny():
    war = _war()
    w_cpu = synth.model_weights(CFG, seed=0, norm_std=0.1)
    return war.Model(CFG, {k: v.to(DEV) for k, v in w_cpu.items()}, max_rows=256)


def start(model, fmt, B, ctx_len=33):
    war = _war()
    pool = war.Pool(CFG, 64, B, 16, device=DEV, kv_format=fmt)
    seq, ctx, nxt = t32(list(range(B))), t32([0] * B), t32([0] * B)
    toks = np.concatenate([synth.uniform_tokens(70 + b, ctx_len, CFG.vocab) for b in range(B)])
    war.prefill_append(model, pool, seq, ctx, [ctx_len] * B, t32(toks), nxt)
    return pool, seq, ctx, toks.reshape(B, ctx_len)


def grammar(B, k, rng):
    """Each row its own mask of a third of the ids."""
    return bits_of(rng.random((B * (k + 1), CFG.vocab)) < 0.33)


@pytest.mark.parametrize("fmt", ["bf16", "e4m3"])
def test_speculation_under_constraints_is_plain_decoding(tiny, fmt):
    """Penalties that change the greedy text: decoded token by token, then with drafts
    (some right, some wrong) verified under the same constraints and counted: the same."""
    war, B, n_out = _war(), 2, 12
    kw = lambda: dict(repetition=f32([1.3, 1.1]), frequency=f32([0.4, 0.0]), presence=f32([0.2, 0.9]),
                      bias_ids=t32([[5, 6], [7, 5]]), bias_values=f32([[30.0, 29.0], [28.0, 30.0]]))
    texts = []
    for k in (0, 3):
        pool, seq, ctx, prompt = start(tiny, fmt, B)
        counts = torch.empty((B, CFG.vocab), dtype=torch.int16, device=DEV)
        war.counts_begin(counts, seq, t32(prompt.ravel()), t32([0, 33, 66]))
        cons = war.Constraints(CFG.vocab, counts=counts, **kw())
        pend, acc, nxt = t32([9, 10]), t32([0] * B), t32([0] * B)
        text = [[], []]
        step = 0
        while min(map(len, text)) < n_out:
            drafts = None
            if k:
                d = [[(texts[0][b] + [0] * 30)[len(text[b]) + j] for j in range(k)] for b in range(B)]
                d[step % B][step % k] = 4001                         # a wrong draft each step
                drafts = t32(d)
            war.verify_step_constrained(tiny, pool, seq, ctx, pend, drafts, None, k, cons, acc, nxt)
            war.counts_add(counts, seq, pend, drafts, acc)
            war.kv_commit(pool, seq, ctx, acc)
            for b in range(B):
                text[b] += (d[b][: int(acc[b])] if k else []) + [int(nxt[b])]
            pend = nxt.clone()
            step += 1
        assert k == 0 or step < n_out                                # drafts were accepted
        texts.append([t[:n_out] for t in text])
        # the counts are the committed text
        for b in range(B):
            c = counts[b].cpu().numpy().view(np.uint16)
            assert int((c & 0x7FFF).sum()) == int(ctx[b]) - 33
        assert pool.state()["status"] == 0
    assert texts[0] == texts[1]
    # ids 5 and 6 are biased by 30 and 29, everything else by nothing: the text is these two, and
    # the penalty of an occurrence moves it from one to the other and back
    assert len(set(texts[0][0])) > 1


def test_constrained_greedy_and_tree_steps_follow_the_oracle(tiny):
    war, B, k = _war(), 3, 5
    rng = np.random.default_rng(4)
    for tree in (False, True):
        c = Case(CFG.vocab, B, k, 21 + tree, tree=tree, S=B, odd=False)
        c.seq = np.arange(B)
        c.index = np.arange(B * (k + 1)) % 4 - 1
        c.index[k + 1] = 1                                            # request 1: no token at its first row
        lens = t32(c.lens)
        pool, seq, ctx, _ = start(tiny, "bf16", B)
        raw = torch.empty((B * (k + 1), CFG.vocab), device=DEV)
        acc, nxt, path = t32([0] * B), t32([0] * B), t32(np.zeros((B, k)))
        # the raw logits of the same step, discarded
        if tree:
            war.verify_step_tree(tiny, pool, seq, ctx, t32(c.last), t32(c.drafts), t32(c.parents), lens, k, acc, nxt, path, raw)
        else:
            war.verify_step(tiny, pool, seq, ctx, t32(c.last), t32(c.drafts), lens, k, acc, nxt, raw)
        war.kv_commit(pool, seq, ctx, t32([-1] * B))
        c.z = raw.cpu().numpy()
        # drafts that the constrained target accepts, as far as they do not change the raw rows
        logits = torch.full_like(raw, 3.0)
        war.verify_step_constrained(tiny, pool, seq, ctx, t32(c.last), t32(c.drafts), lens, k, c.constraints(), acc, nxt, logits,
                                    draft_parents=t32(c.parents) if tree else None, accept_path=path if tree else None)
        war.kv_commit(pool, seq, ctx, t32([-1] * B))
        got = logits.cpu().numpy().astype(np.float64)
        for b in range(B):
            g = []
            for i in range(c.lens[b] + 1):
                r = b * (k + 1) + i
                want, ok = c.oracle_row(b, i, c.z[r]), c.allowed_row(r)
                fine = np.isfinite(want)
                assert (np.isfinite(got[r]) == fine).all()
                assert (np.abs(got[r] - want)[fine] <= c.bound_row(b, i)[fine]).all()
                g.append(oc.greedy(got[r], ok))
            ok_nodes, depth = [True], [0]
            for j in range(1, c.lens[b] + 1):
                p = c.parents[b][j - 1] if tree else j - 1
                ok_nodes.append(ok_nodes[p] and g[p] == c.drafts[b, j - 1])
                depth.append(depth[p] + 1)
            best = max((j for j in range(len(g)) if ok_nodes[j]), key=lambda j: (depth[j], -j))
            assert (int(acc[b]), int(nxt[b])) == (depth[best], g[best]), (tree, b)
        assert int(acc[1]) == 0 and int(nxt[1]) == -1
        assert pool.state()["status"] == 0


def test_accepted_drafts_are_the_constrained_greedy_tokens(tiny):
    """Draft what the constraints force: everything is accepted, a tree's branch too."""
    war, B, k = _war(), 1, 3
    only = [100, 200, 300, 400]
    allowed = np.zeros((4, CFG.vocab), bool)
    for i, t in enumerate(only):
        allowed[i, t] = True
    cons = war.Constraints(CFG.vocab, masks=bits_of(allowed), n_seqs=1)
    pool, seq, ctx, _ = start(tiny, "e4m3", B)
    acc, nxt, path = t32([0]), t32([0]), t32([[0] * 3])
    war.verify_step_constrained(tiny, pool, seq, ctx, t32([1]), t32([only[:3]]), None, k, cons, acc, nxt)
    war.kv_commit(pool, seq, ctx, t32([-1]))
    assert (int(acc[0]), int(nxt[0])) == (3, 400)
    idx = t32([0, 0, 1, 2])                                            # nodes 1 and 2 below the root, 3 below 2
    cons = war.Constraints(CFG.vocab, masks=bits_of(allowed), mask_index=idx, n_seqs=1)
    war.verify_step_constrained(tiny, pool, seq, ctx, t32([1]), t32([[7, 100, 200]]), None, k, cons, acc, nxt,
                                draft_parents=t32([[0, 0, 2]]), accept_path=path)
    war.kv_commit(pool, seq, ctx, acc)
    assert (int(acc[0]), int(nxt[0]), path[0].tolist()) == (2, 300, [2, 3, -1]) and int(ctx[0]) == 36


@pytest.mark.parametrize("share", [1.0, 0.33, 0.002, 0.0005])
def test_sampled_steps_under_constraints(tiny, share):
    """From most ids allowed to a few (fewer than top_k) and rows with none."""
    war, B, k, T, top_k = _war(), 4, 3, 0.8, 50
    rng = np.random.default_rng(int(share * 1e4))
    allowed = rng.random((B * (k + 1), CFG.vocab)) < share
    allowed[2 * (k + 1)] = False                                       # request 2's first row
    c = Case(CFG.vocab, B, k, 3, S=B, odd=False)
    c.seq = np.arange(B)
    drafts = rng.integers(0, CFG.vocab, (B, k))
    for b in range(B):
        for i in range(k):
            at = np.flatnonzero(allowed[b * (k + 1) + i])
            if at.size:
                drafts[b, i] = rng.choice(at)
    cons = war.Constraints(CFG.vocab, counts=table_of(c.table), repetition=f32(c.rep), masks=bits_of(allowed))
    pool, seq, ctx, _ = start(tiny, "bf16", B)
    u = rng.random((B * (k + 1), 2)).astype(np.float32)
    z, acc, nxt = torch.empty((B * (k + 1), CFG.vocab), device=DEV), t32([0] * B), t32([0] * B)
    war.verify_step_constrained(tiny, pool, seq, ctx, t32(c.last), t32(drafts), None, k, cons, acc, nxt, z, uniforms=f32(u),
                                temperature=T, top_k=top_k)
    war.kv_commit(pool, seq, ctx, acc)
    z = z.cpu().numpy().astype(np.float64)
    exact = 0
    for b in range(B):
        rows = z[b * (k + 1): (b + 1) * (k + 1)]
        live = 0
        while live < k + 1 and np.isfinite(rows[live]).any():
            live += 1
        uu = u[b * (k + 1): (b + 1) * (k + 1)].astype(np.float64)
        if live == 0:
            assert (int(acc[b]), int(nxt[b])) == (0, -1)
            exact += 1
            continue
        r = verify_sampled(rows[:live], drafts[b, : live - 1].tolist(), uu[:live, 0], uu[:live, 1], T, top_k)
        same = (int(acc[b]), int(nxt[b])) == (r["accept"], r["next"])
        assert same or min(r["margins"]) < 1e-5 or live < k + 1, (b, r)
        exact += same
        assert int(nxt[b]) == -1 or allowed[b * (k + 1) + int(acc[b]), int(nxt[b])]
    assert exact >= 3 and (int(acc[2]), int(nxt[2])) == (0, -1)


def test_refusals(tiny):
    war = _war()
    pool, seq, ctx, _ = start(tiny, "bf16", 2)
    V = CFG.vocab
    good = war.Constraints(V, repetition=torch.ones(2, device=DEV))
    acc, nxt = t32([0, 0]), t32([0, 0])
    z = torch.zeros((2, V), device=DEV)
    step = lambda cons, **kw: war.verify_step_constrained(tiny, pool, seq, ctx, t32([1, 2]), None, None, 0, cons, acc, nxt, **kw)
    with pytest.raises(war.WarError):
        step(war.Constraints(V, repetition=torch.ones(1, device=DEV)))          # fewer sequences than the pool
    with pytest.raises(ValueError):
        step(war.Constraints(V - 32, repetition=torch.ones(2, device=DEV)))     # another vocabulary
    with pytest.raises(ValueError):
        step(war.Constraints(V, masks=torch.zeros((1, V // 32), dtype=torch.int32, device=DEV), n_seqs=2))   # one mask, two rows
    for T, k in ((0.0, 5), (float("nan"), 5), (1.0, 0), (1.0, V + 1)):
        with pytest.raises(war.WarError):
            step(good, uniforms=torch.zeros((2, 2), device=DEV), temperature=T, top_k=k)
    with pytest.raises(ValueError):
        war.constrain_logits(z, good, seq, t32([1, 2]), None, None, 0, out=z.half())
    with pytest.raises(ValueError):
        war.constrain_logits(z, good, seq, t32([1]), None, None, 0, out=z)
    with pytest.raises(ValueError):
        war.constrain_logits(z, good, seq, t32([1, 2]), None, None, 0, greedy=acc, workspace=torch.empty(8, device=DEV))
    with pytest.raises(war.WarError):
        war.constrain_logits(z, good, seq, t32([1, 2]), None, None, 0)          # nothing wanted
    with pytest.raises(ValueError):
        war.counts_add(torch.zeros((2, V), device=DEV), seq, None, None, None)
    step(good)                                                                   # nothing above left a step behind
    war.kv_commit(pool, seq, ctx, acc)
    assert pool.state()["status"] == 0


def test_a_workspace_made_for_a_stream_is_that_streams_memory():
    """Memory that the current stream still reads, freed and free to be reused there, is
    not written by a call on another stream."""
    war = _war()
    c = Case(4096, 64, 3, 5, odd=False)
    cons, z = c.constraints(), f32(c.z)
    R = c.B * (c.k + 1)
    seq, last, drafts, lens = t32(c.seq), t32(c.last), t32(c.drafts[:, : c.k]), t32(c.lens)
    greedy, want = torch.empty(R, dtype=torch.int32, device=DEV), torch.empty(R, dtype=torch.int32, device=DEV)
    want.fill_(77), greedy.fill_(77)
    war.constrain_logits(z, cons, seq, last, drafts, lens, c.k, greedy=want)
    other = torch.cuda.Stream()
    n = war.lib().war_constrain_workspace(R, c.V)
    gc.collect()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    for _ in range(4):
        x = torch.full((n,), 9, dtype=torch.uint8, device=DEV)
        y = torch.empty_like(x)
        torch.cuda.synchronize()
        torch.cuda._sleep(20_000_000)
        y.copy_(x)                                     # waits behind the sleep
        del x
        war.constrain_logits(z, cons, seq, last, drafts, lens, c.k, greedy=greedy, stream=other)
        torch.cuda.synchronize()
        assert (y == 9).all()
        assert torch.equal(greedy, want)

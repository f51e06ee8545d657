"""Arguments that the host refuses before anything is enqueued: no GPU is needed, no
address is looked at."""
import ctypes as C

import pytest
import torch

from paper_2607_17299_amd import synth, war

INVALID = -1
A = 1 << 20   # an address that is never read


def constraints(**kw):
    c = war._Constraints()
    c.n_seqs = 2
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def test_constrain_logits_refuses():
    lib = war.lib()

    def call(c=constraints(), V=100, B=2, seq=A, last=A, drafts=A, parents=None, lens=None, k=1, z=A, zs=100, out=A, os=100,
             greedy=A, ws=A):
        return lib.war_constrain_logits(None if c is None else C.byref(c), V, B, seq, last, drafts, parents, lens, k, z, zs, out,
                                        os, greedy, ws, None)

    for bad in (dict(c=None), dict(c=constraints(n_seqs=0)), dict(c=constraints(n_bias=-1)), dict(c=constraints(n_bias=1025)),
                dict(c=constraints(n_bias=3)), dict(c=constraints(n_masks=1)), dict(c=constraints(mask_index=A)),
                dict(V=0), dict(V=(1 << 24) + 1, zs=1 << 25), dict(B=0), dict(B=1025), dict(k=-1), dict(k=64), dict(seq=None),
                dict(last=None), dict(drafts=None), dict(z=None), dict(zs=99), dict(os=99), dict(out=A, z=A, zs=100, os=101),
                dict(out=None, greedy=None), dict(ws=None), dict(ws=A + 8)):
        assert call(**bad) == INVALID, bad
        assert lib.war_last_error()


def test_counts_refuse():
    lib = war.lib()
    begin = lambda counts=A, V=10, S=2, B=1, seq=A, tok=A, m=5, off=A: lib.war_counts_begin(counts, V, S, B, seq, tok, m, off,
                                                                                             None)
    add = lambda counts=A, V=10, S=2, B=1, seq=A, first=A, tok=A, n=3: lib.war_counts_add(counts, V, S, B, seq, first, tok, n,
                                                                                      None, None, None)
    for bad in (dict(counts=None), dict(counts=A + 1), dict(V=0), dict(S=0), dict(B=0), dict(B=1025), dict(seq=None)):
        assert begin(**bad) == INVALID and add(**bad) == INVALID, bad
    for bad in (dict(tok=None), dict(off=None), dict(m=-1)):
        assert begin(**bad) == INVALID, bad
    for bad in (dict(tok=None), dict(n=-1), dict(n=4097)):
        assert add(**bad) == INVALID, bad


def test_pools_and_attention_refuse():
    lib = war.lib()
    cfg = war.config_struct(synth.TINY, 1)
    h = C.c_void_p()
    for fmt in (-1, 2):
        assert lib.war_kv_pool_create_format(C.byref(cfg), A, 4, fmt, A, 1, 4, None, C.byref(h)) == INVALID and not h.value
        assert lib.war_kv_pool_bytes(C.byref(cfg), 4, fmt) == -1
    assert lib.war_kv_pool_create_format(C.byref(cfg), A + 8, 4, 1, A, 1, 4, None, C.byref(h)) == INVALID
    assert lib.war_kv_pool_bytes(C.byref(cfg), 0, 1) == -1
    T = synth.TINY
    heads = T.n_layers * 4 * T.n_kv_heads
    assert lib.war_kv_pool_bytes(C.byref(cfg), 4, 0) == heads * 2 * 16 * T.head_dim * 2
    assert lib.war_kv_pool_bytes(C.byref(cfg), 4, 1) == heads * (2 * 16 * T.head_dim + 32)
    assert lib.war_attend_create(None, 1, 1, C.byref(h)) == INVALID
    assert lib.war_attend_update(None, 1, 1, A, A, None, None, None) == INVALID
    assert lib.war_attend_run(None, 0, A, 128, A, 128, None) == INVALID
    assert lib.war_kv_write(None, 0, 1, A, A, 1, None, A, 128, A, 128, None) == INVALID
    assert lib.war_kv_read(None, 0, 1, A, A, 1, None, A, 128, A, 128, None) == INVALID
    assert lib.war_constrain_workspace(3, 129) == 3 * 2 * 8 and lib.war_constrain_workspace(0, 5) == -1


def test_constraints_check_their_arrays():
    f, i = torch.zeros(2), torch.zeros((2, 4), dtype=torch.int32)
    counts = torch.zeros((2, 40), dtype=torch.int16)
    war.Constraints(40, counts=counts, repetition=f, bias_ids=i, bias_values=torch.zeros(2, 4), masks=torch.zeros((3, 2),
                    dtype=torch.int32), mask_index=torch.zeros(6, dtype=torch.int32))
    for bad in (dict(), dict(counts=counts.int()), dict(counts=counts[:, :39]), dict(repetition=torch.zeros(2, 1)),
                dict(repetition=f, frequency=torch.zeros(3)), dict(repetition=f.double()), dict(bias_ids=i),
                dict(bias_ids=i, bias_values=torch.zeros(2, 3)), dict(counts=counts.t().contiguous().t()),
                dict(masks=torch.zeros((3, 2), dtype=torch.int32)),
                dict(repetition=f, masks=torch.zeros((3, 3), dtype=torch.int32))):
        with pytest.raises(ValueError):
            war.Constraints(40, **bad)
    with pytest.raises(ValueError):
        war.Constraints(40, repetition=f, masks=torch.zeros((3, 2), dtype=torch.int32))._rows(4)

"""rope_write with five to eight query heads a kv-head, and what it refuses of a pool."""
import ctypes as C
import math

import pytest
import torch

import test_gpu_layer_ops as ops

pytestmark = pytest.mark.gpu
DEV = "cuda"
INVALID = -1


@pytest.mark.parametrize("rotary,adjacent,axes", [(1.0, False, "blocks"), (0.5, True, "turns"), (24, False, "one")])
@pytest.mark.parametrize("heads", [(10, 2, 128), (12, 2, 64), (14, 2, 64), (16, 2, 128), (8, 1, 64)])
def test_rope_write_of_wide_groups(heads, rotary, adjacent, axes):
    """Groups that fill the kernel's eight and that do not, in pages of both formats."""
    assert 5 <= heads[0] // heads[1] <= 8
    ops.test_rope_write(heads, rotary, adjacent, axes)


def test_wide_groups_in_place():
    war = ops._war()
    heads, B, n, ctx = (14, 2, 64), 3, 21, [3, 40, 16]
    g = torch.Generator(device=DEV).manual_seed(6)
    x = torch.randn((B, n, 18, 64), device=DEV, generator=g).bfloat16()
    ids, pos0, rope = ops.t32([0, 1, 2]), ops.t32(ctx), war.Rope(64)
    a, b = (ops.pool_of(heads, [p + n for p in ctx], "bf16") for _ in range(2))
    out = torch.empty((B, n, 14, 64), dtype=torch.bfloat16, device=DEV)
    war.rope_write(a, 0, rope, ids, pos0, x[:, :, :14], x[:, :, 14:16], x[:, :, 16:], out)
    y = x.clone()
    war.rope_write(b, 0, rope, ids, pos0, y[:, :, :14], y[:, :, 14:16], y[:, :, 16:], y[:, :, :14])
    assert torch.equal(y[:, :, :14], out) and torch.equal(y[:, :, 14:], x[:, :, 14:])
    assert torch.equal(a.kv.view(torch.uint8), b.kv.view(torch.uint8))          # (untouched numbers are NaN)


def test_rope_write_refuses_before_anything_is_written():
    """Every address is one of real memory, large enough for what each call names."""
    war = ops._war()
    lib, heads, n = war.lib(), (4, 2, 64), 5
    pool = ops.pool_of(heads, [16], "bf16", layers=2)
    before = pool.kv.clone()
    q, out = (torch.full((n + 1, 256 + 16), v, dtype=torch.bfloat16, device=DEV) for v in (1.0, 7.0))
    k, v = (torch.ones((n + 1, 128 + 16), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    ids, pos0 = ops.t32([0]), ops.t32([3])

    def rope_of(rotary=64, adjacent=0, n_axes=1, axes=None, freqs=[1.0] * 32):
        a = None if axes is None else (C.c_uint8 * 64)(*axes)
        f = None if freqs is None else (C.c_double * 64)(*freqs)
        r = war._Rope(rotary, adjacent, n_axes, None if a is None else C.addressof(a), None if f is None else C.addressof(f))
        r.keep = (a, f)
        return r

    def call(layer=0, rope=rope_of(), B=1, seq=ids.data_ptr(), p0=pos0.data_ptr(), n_max=n, q=q.data_ptr(), qs=272, out=out.data_ptr(),
             os=272, k=k.data_ptr(), ks=144, v=v.data_ptr(), vs=144):
        return lib.war_rope_write(pool.handle, layer, None if rope is None else C.byref(rope), B, seq, p0, n_max, None, None, q, qs, out,
                                  os, k, ks, v, vs, torch.cuda.current_stream().cuda_stream)

    bad = [dict(layer=-1), dict(layer=2), dict(rope=None), dict(B=0), dict(B=1025), dict(n_max=-1), dict(n_max=(1 << 26) + 1),
           dict(B=1024, n_max=(1 << 16) + 1), dict(seq=None), dict(p0=None), dict(q=q.data_ptr(), out=q.data_ptr(), os=256),
           dict(q=q.data_ptr(), qs=256, out=q.data_ptr())]
    bad += [dict(rope=rope_of(**r)) for r in (
        dict(rotary=0), dict(rotary=4), dict(rotary=12), dict(rotary=72), dict(rotary=128), dict(adjacent=2), dict(adjacent=-1),
        dict(n_axes=0), dict(n_axes=5), dict(axes=[0] * 31 + [1]), dict(n_axes=4, axes=[4] + [0] * 31), dict(freqs=None),
        dict(freqs=[1.0] * 31 + [math.nan]), dict(freqs=[math.inf] * 32), dict(freqs=[6.31] + [1.0] * 31), dict(freqs=[-6.31] + [1.0] * 31))]
    for name, row, t in (("q", 256, q), ("out", 256, out), ("k", 128, k), ("v", 128, v)):
        stride = {"out": "os"}.get(name, name + "s")
        bad += [{name: None}, {name: t.data_ptr() + 8}, {stride: row - 8}, {stride: row + 4}, {stride: -row}]
    for b in bad:
        assert call(**b) == INVALID, b
        assert lib.war_last_error()
    torch.cuda.synchronize()
    assert pool.state()["status"] == 0 and torch.equal(pool.kv.view(torch.uint8), before.view(torch.uint8)) and bool((out == 7).all())
    assert call(n_max=0, q=None, k=None, v=None, out=None) == 0
    assert call() == 0
    assert not bool((out[:n, :256] == 7).any()) and bool((out[n:] == 7).all()) and bool((out[:, 256:] == 7).all())
    assert call(rope=rope_of(rotary=32, n_axes=3, axes=[2] * 16, freqs=[-6.3] * 16), out=q.data_ptr(), os=272) == 0
    torch.cuda.synchronize()
    assert pool.state()["status"] == 0

"""What the operators of a decoder layer refuse before anything is enqueued: no GPU is
needed, no address is looked at."""
import ctypes as C

import pytest
import torch

from paper_2607_17299_amd import war

INVALID, UNSUPPORTED = -1, -4
A = 1 << 20   # an address that is never read


def mx(**kw):
    f = dict(format=2, rows=3, cols=64, codes=A, code_stride=64, scales=A, scale_stride=4)
    f.update(kw)
    return war._Mx(*[f[n] for n, _ in war._Mx._fields_])


BAD_MX = [dict(format=1), dict(format=4), dict(rows=-1), dict(rows=(1 << 20) + 1), dict(cols=0), dict(cols=48), dict(cols=65568),
          dict(codes=None), dict(scales=None), dict(code_stride=48), dict(code_stride=72), dict(codes=A + 8), dict(scale_stride=0),
          dict(scale_stride=6), dict(scales=A + 2), dict(rows=1 << 20, cols=65536, code_stride=65536, scale_stride=2048)]


def test_residual_norm_refuses():
    lib = war.lib()

    def call(rows=3, cols=64, x=A, xs=64, h=A, hs=64, ht=1, g=A, eps=1e-6, m=mx(), y=None, ys=0):
        return lib.war_residual_norm(rows, cols, x, xs, h, hs, ht, g, eps, None if m is None else C.byref(m), y, ys, None)

    for bad in [dict(m=mx(**b)) for b in BAD_MX] + [
            dict(rows=-1), dict(cols=40), dict(x=A + 2), dict(xs=56), dict(xs=68), dict(h=None), dict(h=A + 8), dict(hs=63),
            dict(ht=2), dict(g=None), dict(g=A + 8), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(m=None),
            dict(y=A, ys=64), dict(m=None, y=A, ys=60), dict(m=None, y=A + 8, ys=64), dict(rows=2), dict(cols=96)]:
        assert call(**bad) == INVALID, bad
        assert lib.war_last_error()
    assert call(rows=0, m=mx(rows=0)) == 0


def test_quantize_and_dequantize_refuse():
    lib = war.lib()
    q = lambda m=mx(), x=A, xs=64, g=None, gs=0, t=0: lib.war_quantize(None if m is None else C.byref(m), x, xs, g, gs, t, None)
    d = lambda m=mx(), x=A, xs=64, g=None, gs=0, t=0: lib.war_dequantize(None if m is None else C.byref(m), x, xs, t, None)
    for bad in [dict(m=None)] + [dict(m=mx(**b)) for b in BAD_MX] + [dict(x=None), dict(x=A + 8), dict(xs=56), dict(xs=65),
                                                                     dict(t=2), dict(t=-1)]:
        assert q(**bad) == INVALID and d(**bad) == INVALID, bad
    for bad in (dict(g=A, gs=63), dict(g=A + 4, gs=64)):
        assert q(**bad) == INVALID, bad
    assert q(m=mx(rows=0), x=None) == 0 and d(m=mx(rows=0), x=None) == 0


def test_linear_refuses():
    lib = war.lib()
    h = C.c_void_p()
    w = lambda **kw: mx(**{**dict(format=3, code_stride=32), **kw})
    for bad in (dict(format=1), dict(rows=0), dict(rows=-1), dict(cols=33), dict(codes=None), dict(code_stride=31),
                dict(scale_stride=1)):
        assert lib.war_linear_create(C.byref(w(**bad)), None, None, C.byref(h)) == INVALID and not h.value, bad
    assert lib.war_linear_create(None, None, None, C.byref(h)) == INVALID
    assert lib.war_linear_create(C.byref(w()), None, None, None) == INVALID
    assert lib.war_linear_create(C.byref(w()), A + 1, None, C.byref(h)) == INVALID
    assert lib.war_linear_create(C.byref(mx()), None, None, C.byref(h)) == UNSUPPORTED and not h.value
    assert lib.war_linear_run(None, C.byref(mx()), A, 64, 0, None) == INVALID
    lib.war_linear_destroy(None)


def test_shapes_are_chosen_for_every_size():
    lib = war.lib()
    for fmt in (2, 3):
        for yt in (0, 1):
            for M in (1, 16, 17, 64, 65, 100, 1000, 65536, 1 << 20):
                for N in (1, 100, 5003, 151936, 1 << 20):
                    for K in (32, 544, 4096, 65536):
                        s = lib.war_debug_linear_shape(M, N, K, fmt, yt)
                        assert 0 <= s < 10 and (s >= 3 or M <= 64)
    assert lib.war_debug_linear(None, C.byref(mx()), A, 64, 0, 10, None) == INVALID
    assert lib.war_debug_linear(None, C.byref(mx()), A, 64, 0, -1, None) == INVALID


def test_rope_write_refuses():
    lib = war.lib()
    r = war.Rope(64)
    assert lib.war_rope_write(None, 0, r._ref, 1, A, A, 1, None, None, A, 256, A, 256, A, 128, A, 128, None) == INVALID
    for bad in (dict(head_dim=96), dict(rotary_dim=4), dict(rotary_dim=12), dict(rotary_dim=72), dict(axes=[0] * 31),
                dict(axes=[4] * 32), dict(axes=[-1] * 32), dict(freqs=[1.0])):
        with pytest.raises(ValueError):
            war.Rope(**{**dict(head_dim=64), **bad})


def test_matrices_are_checked():
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)
    m = war.Mx(u8(3, 64), u8(3, 4)[:, :2], "e4m3")
    assert m.shape == (3, 64) and war.Mx(u8(3, 32), u8(3, 4)[:, :2], "e2m1").shape == (3, 64) and m[1:].shape == (2, 64)
    e = war.Mx.empty(5, 160, "e2m1", "cpu")
    assert e.codes.shape == (5, 80) and e.scales.shape == (5, 5) and e.scales.stride(0) == 8
    for codes, scales, fmt in ((u8(3, 64), u8(3, 3), "e4m3"), (u8(3, 48), u8(3, 2), "e4m3"), (u8(3, 64), u8(2, 2), "e4m3"),
                               (u8(3, 64).int(), u8(3, 2), "e4m3"), (u8(3, 128)[:, ::2], u8(3, 2), "e4m3"),
                               (u8(3, 64), u8(3, 2), "e5m2"), (u8(64), u8(2), "e4m3"), (u8(3, 0), u8(3, 0), "e4m3")):
        with pytest.raises(ValueError):
            war.Mx(codes, scales, fmt)
    h, g = torch.zeros(3, 64), torch.zeros(64).bfloat16()
    x = torch.zeros(3, 64).bfloat16()
    for args in ((x[:2], h, g, 1e-6, m), (x.float(), h, g, 1e-6, m), (x, h.double(), g, 1e-6, m), (x, h, g.float(), 1e-6, m),
                 (x, h, g[:32], 1e-6, m), (x, h, g, 1e-6, e), (x, h, g, 1e-6, h)):
        with pytest.raises(ValueError):
            war.residual_norm(*args)
    with pytest.raises(ValueError, match="GPU"):
        war.residual_norm(x, h, g, 1e-6, m)
    with pytest.raises(ValueError, match="GPU"):
        war.dequantize(m, x)
    with pytest.raises(ValueError):
        war.quantize(x, m, gate=h)
    with pytest.raises(ValueError):
        war.quantize(x.t(), m)
    with pytest.raises(ValueError):
        war.dequantize(m, x[:2])


def test_residual_norm_in_place_wants_one_stride():
    """A row of y at another stride than x's would land on rows of x that other workgroups
    have yet to read."""
    lib = war.lib()
    for xs, ys in ((72, 64), (64, 72)):
        assert lib.war_residual_norm(3, 64, A, xs, 2 * A, 64, 1, A, 1e-6, None, A, ys, None) == INVALID
        assert b"in place" in lib.war_last_error()


def test_residual_norm_of_no_rows():
    """An empty tensor has no address: no rows are no work, whichever output they go to."""
    lib = war.lib()
    norm = lambda m, y, rows=0: lib.war_residual_norm(rows, 64, None, 64, None, 64, 1, A, 1e-6, m, y, 64, None)
    assert norm(None, None) == 0 and norm(None, A) == 0 and norm(C.byref(mx(rows=0)), None) == 0
    assert norm(C.byref(mx(rows=0)), A) == INVALID and norm(None, None, 1) == INVALID


def test_rows_of_a_matrix_share_its_memory():
    m = war.Mx.empty(6, 64, "e2m1", "cpu")
    for rows in (slice(1, 4), slice(None, None, 2), slice(6, 6)):
        part = m[rows]
        assert part.codes.untyped_storage().data_ptr() == m.codes.untyped_storage().data_ptr()
        assert part.shape == (len(range(6)[rows]), 64)
    for rows in (torch.tensor([0, 2]), [0, 2], torch.ones(6, dtype=torch.bool), 3, (slice(0, 2), slice(0, 16))):
        with pytest.raises(ValueError):                          # (copies, which a call would write to in vain)
            m[rows]

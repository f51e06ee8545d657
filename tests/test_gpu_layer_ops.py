"""The operators of a decoder layer over microscaled numbers against the float64 oracle:
residual_norm, quantize, dequantize, linear and rope_write."""
import numpy as np
import pytest
import torch

from oracle import mx as omx
from paper_2607_17299_amd import synth

pytestmark = pytest.mark.gpu
DEV = "cuda"
FMTS = ["e4m3", "e2m1"]


def _war():
    from paper_2607_17299_amd import war
    return war


def t32(a):
    return torch.tensor(np.asarray(a), dtype=torch.int32, device=DEV)


def as64(x):
    return x.double().cpu().numpy()


def padded(rows, cols, pad, dtype, fill):
    """A [rows, cols] view whose rows are `pad` elements apart, in memory of `fill`."""
    return torch.full((rows, cols + pad), fill, dtype=dtype, device=DEV)[:, :cols]


def mx_of(rows, cols, fmt, pad=0):
    """An Mx whose memory starts as 0xaa; pad: bytes between its rows of codes."""
    war = _war()
    w = cols if fmt == "e4m3" else cols // 2
    codes = torch.full((rows + 1, w + pad), 0xaa, dtype=torch.uint8, device=DEV)
    scales = torch.full((rows + 1, -(-cols // 128) * 4 + pad), 0xaa, dtype=torch.uint8, device=DEV)
    m = war.Mx(codes[:rows, :w], scales[:rows, : cols // 32], fmt)
    m.whole = (codes, scales)
    return m


def untouched(m):
    """Whether the bytes beside the matrix are as they were."""
    for whole, part in zip(m.whole, (m.codes, m.scales)):
        keep = whole.clone()
        keep[: part.shape[0], : part.shape[1]] = 0xaa
        if not bool((keep == 0xaa).all()):
            return False
    return True


def codes_of(m):
    c = m.codes.cpu().numpy()
    return (c.astype(np.int64) if m.format == "e4m3" else omx.unpack_e2m1(c)), m.scales.cpu().numpy().astype(np.int64)


def check_codes(m, y, rel=0.0, floor=0.0):
    """The matrix holds float64 y, where y is known to a relative `rel` (and absolute
    `floor`): exactly what the oracle stores, or what it stores of a number that near."""
    codes, scales = codes_of(m)
    if rel == 0.0 and np.ndim(floor) == 0 and floor == 0.0:
        wc, ws = omx.quantise(y, m.format)
        np.testing.assert_array_equal(scales, ws)
        live = np.repeat(ws != 255, 32, axis=1)
        np.testing.assert_array_equal(codes[live], wc[live])
        return
    R, C = y.shape
    ok = np.isfinite(y.reshape(R, -1, 32)).all(-1)
    np.testing.assert_array_equal(scales == 255, ~ok)
    z = np.where(np.repeat(ok, 32, axis=1), y, 0.0)
    lo, hi = z - np.abs(z) * rel - floor, z + np.abs(z) * rel + floor
    size = lambda v: np.abs(v).reshape(R, -1, 32).max(-1)
    e = scales - 127
    near = np.maximum(np.abs(lo), np.abs(hi))
    assert (omx.exponent(size(near), m.format)[ok] >= e[ok]).all()
    far = np.where(np.sign(lo) != np.sign(hi), 0.0, np.minimum(np.abs(lo), np.abs(hi)))
    assert (omx.exponent(size(far), m.format)[ok] <= e[ok]).all()
    f = np.exp2(np.repeat(np.where(ok, e, 0), 32, axis=1).astype(np.float64))
    top = omx.NUMBERS[m.format][-1]
    got = omx.numbers(codes, np.where(ok, scales, 127), m.format) / f
    val = lambda v: omx.numbers(omx.nearest_code(np.clip(v / f, -top, top), m.format), np.full_like(scales, 127), m.format)
    live = np.repeat(ok, 32, axis=1)
    assert (got >= val(lo))[live].all() and (got <= val(hi))[live].all()


def spread(rng, rows, cols):
    """Blocks of every size, subnormal ones, zeros and numbers that are not finite."""
    x = rng.standard_normal((rows, cols // 32, 32)) * 2.0 ** rng.integers(-140, 120, (rows, cols // 32, 1))
    x[rng.random((rows, cols // 32)) < 0.1] = 0.0
    x = x.reshape(rows, cols)
    if rows > 2:
        x[1, 5], x[2, cols - 1], x[0, cols // 2] = np.inf, np.nan, -np.inf
    return x


# ------------------------------------------------------------ codes and numbers
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("rows,cols", [(1, 32), (5, 96), (33, 4096), (3, 65536)])
def test_quantize_is_the_oracles_bit_for_bit(rows, cols, fmt, dtype):
    war = _war()
    x = torch.tensor(spread(np.random.default_rng(rows + cols), rows, cols)).to(dtype).to(DEV)
    held = padded(rows, cols, 24, dtype, 7.0)
    held.copy_(x)
    m = mx_of(rows, cols, fmt, pad=32)
    war.quantize(held, m)
    check_codes(m, as64(x))
    assert untouched(m)


@pytest.mark.parametrize("fmt", FMTS)
def test_quantize_rounds_every_bf16_number(fmt):
    """All finite bf16 numbers beside a block's largest of each size."""
    war = _war()
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    x = bits[torch.isfinite(bits)]
    x = torch.cat([x, x[: -len(x) % 32]]).view(-1, 32)          # neighbours by bit pattern share a block
    x = torch.cat([x, x.flatten()[torch.randperm(x.numel(), generator=torch.Generator().manual_seed(0))].view(-1, 32)]).to(DEV)
    m = mx_of(*x.shape, fmt)
    war.quantize(x, m)
    check_codes(m, as64(x))


def test_midpoints_go_to_the_even_code():
    war = _war()
    for fmt in FMTS:
        n = omx.NUMBERS[fmt]
        mid = np.concatenate([(n[1:] + n[:-1]) / 2, np.nextafter(((n[1:] + n[:-1]) / 2).astype(np.float32), np.float32(1e9)),
                              np.nextafter(((n[1:] + n[:-1]) / 2).astype(np.float32), np.float32(-1e9))])
        mid = np.concatenate([mid, -mid])
        x = np.zeros((len(mid), 32))
        x[:, 3], x[:, 17] = mid, n[-1]
        x = torch.tensor(x).float().to(DEV)
        m = mx_of(*x.shape, fmt)
        war.quantize(x, m)
        check_codes(m, as64(x))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("fmt", FMTS)
def test_gate(fmt, dtype):
    """A lane's exp, division and products are off by under 2^-20 together; where exp
    overflows (gates below -88.7) the result is 0 for less than 3e-37 |x|."""
    war = _war()
    rng = np.random.default_rng(5)
    rows, cols = 37, 352
    xg = torch.tensor(rng.standard_normal((rows, 2 * cols)) * 8).to(dtype).to(DEV)
    xg[3, :64] = torch.linspace(-120, 120, 64).to(dtype)
    xg[4, 7], xg[5, cols + 40], xg[6, 33] = float("inf"), float("nan"), float("-inf")
    g, x = xg[:, :cols], xg[:, cols:]
    m = mx_of(rows, cols, fmt, pad=16)
    war.quantize(x, m, gate=g)
    check_codes(m, omx.gated(as64(x), as64(g)), 2.0 ** -20, 3e-37 * np.nan_to_num(np.abs(as64(x)), posinf=0))
    assert untouched(m)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("fmt", FMTS)
def test_dequantize_every_code_and_scale(fmt, dtype):
    war = _war()
    half = 256 if fmt == "e4m3" else 16
    codes = np.tile(np.arange(half), (256, 1)) if fmt == "e4m3" else np.tile(np.arange(16), (256, 2))
    scales = np.tile(np.arange(256)[:, None], (1, codes.shape[1] // 32))
    m = mx_of(256, codes.shape[1], fmt, pad=16)
    m.codes.copy_(torch.tensor(codes if fmt == "e4m3" else omx.pack_e2m1(codes), dtype=torch.uint8))
    m.scales.copy_(torch.tensor(scales, dtype=torch.uint8))
    out = padded(256, codes.shape[1], 8, dtype, 7.0)
    war.dequantize(m, out)
    with np.errstate(over="ignore"):
        want = torch.tensor(omx.numbers(codes, scales, fmt)).to(torch.float32).to(dtype)
    torch.testing.assert_close(out.cpu(), want, rtol=0, atol=0, equal_nan=True)
    assert bool((out._base[:, codes.shape[1]:] == 7).all())


# ------------------------------------------------------------------------- norm
NORM_REL = 2.0 ** -19  # a sum of squares of n <= 2^16 fp32 numbers in lanes of at most 64, waves and 16 partial
                       # sums: under 90 roundings of 2^-24, halved by the root; its division and products: 5 more


@pytest.mark.parametrize("h_type", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("out", ["bf16"] + FMTS)
@pytest.mark.parametrize("rows,cols", [(1, 32), (7, 96), (4, 256), (3, 544), (5, 2048), (3, 4096), (2, 4128), (2, 12288), (1, 20000),
                                       (1, 65536)])
def test_residual_norm(rows, cols, out, h_type):
    war = _war()
    rng = np.random.default_rng(cols)
    x, h = padded(rows, cols, 8, torch.bfloat16, 3.0), padded(rows, cols, 16, h_type, 5.0)
    x.copy_(torch.tensor(rng.standard_normal((rows, cols))))
    h.copy_(torch.tensor(rng.standard_normal((rows, cols)) * 4))
    gain = torch.tensor(1 + 0.3 * rng.standard_normal(cols)).bfloat16().to(DEV)
    if rows > 2:
        x[0], h[0] = 0.0, 0.0                       # a row of zeros
        x[1], h[1] = 0.0, h[1] * 2.0 ** -70         # squares below fp32's range: eps alone
        x[2, 5] = float("nan")
    total = (h.float() + x.float())
    want = omx.norm(as64(total), as64(gain), 1e-6)
    y = padded(rows, cols, 8, torch.bfloat16, 9.0) if out == "bf16" else mx_of(rows, cols, out, pad=16)
    war.residual_norm(x, h, gain, 1e-6, y)
    torch.testing.assert_close(h, total.to(h_type), rtol=0, atol=0, equal_nan=True)
    assert bool((h._base[:, cols:] == 5).all())
    if out == "bf16":
        np.testing.assert_allclose(as64(y), want, rtol=2.0 ** -8 + NORM_REL, atol=1e-38)
        assert bool((y._base[:, cols:] == 9).all())
    else:
        check_codes(y, want, NORM_REL, 1e-38)
        assert untouched(y)


def test_norm_alone_leaves_h_and_may_overwrite_x():
    war = _war()
    g = torch.Generator(device=DEV).manual_seed(1)
    h = torch.randn((6, 512), device=DEV, generator=g)
    x = torch.randn((6, 512), device=DEV, generator=g).bfloat16()
    gain = torch.ones(512, device=DEV).bfloat16()
    keep, y = h.clone(), torch.empty_like(x)
    war.residual_norm(None, h, gain, 0.0, y)
    assert torch.equal(h, keep)
    np.testing.assert_allclose(as64(y), omx.norm(as64(keep), np.ones(512), 0.0), rtol=2.0 ** -8 + NORM_REL)
    want = torch.empty_like(x)
    war.residual_norm(x, h, gain, 0.0, want)
    war.residual_norm(x, keep, gain, 0.0, x)
    assert torch.equal(x, want) and torch.equal(h, keep)


# --------------------------------------------------------------------- products
def coded(rng, rows, cols, fmt, exact, pad=0):
    """A matrix of codes with its numbers.  exact: products of two such are multiples of 2^-9
    below 2^10 that span at most 13 places in every group of eight, sums below 2^15 in
    magnitude: fp32 holds all of them."""
    m = mx_of(rows, cols, fmt, pad)
    if exact:
        codes = rng.integers(0, 16, (rows, cols)) if fmt == "e2m1" else rng.integers(0x30, 0x50, (rows, cols)) + 128 * rng.integers(0, 2, (rows, cols))
        scales = rng.integers(125, 129, (rows, cols // 32))
    else:
        x = rng.standard_normal((rows, cols)) * 2.0 ** rng.integers(-3, 4, (rows, 1))
        x[:, :: max(1, cols // 7)] *= 16
        codes, scales = omx.quantise(x, fmt)
    m.codes.copy_(torch.tensor(codes if fmt == "e4m3" else omx.pack_e2m1(codes), dtype=torch.uint8))
    m.scales.copy_(torch.tensor(scales, dtype=torch.uint8))
    return m, omx.numbers(codes, scales, fmt)


def product_tolerance(x, w, fmt, y_type=torch.bfloat16):
    """What fp32 sums may be off by: K / 8 + 64 additions, each 2^-23 (half a step and a cut
    end) of the magnitudes; e4m3 on the way to bf16: eight numbers of a group lose less than
    2^-13 of its largest each."""
    mag = np.abs(x) @ np.abs(w).T
    tol = (x.shape[1] / 8 + 64) * 2.0 ** -23 * mag
    if fmt == "e4m3" and y_type == torch.bfloat16:
        for k in range(0, x.shape[1], 8):
            tol += 8 * 2.0 ** -13 * np.max(np.abs(x[:, None, k:k + 8] * w[None, :, k:k + 8]), axis=-1)
    return tol


SHAPES = [(1, 1, 32), (4, 512, 256), (1, 24, 4096), (15, 17, 544), (16, 48, 512), (17, 300, 1120), (33, 130, 96), (72, 257, 2080), (64, 64, 12288),
          (130, 515, 1024), (257, 300, 640), (300, 1000, 416), (1001, 272, 160)]


@pytest.mark.parametrize("y_type", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_products_that_fp32_holds_are_exact(M, N, K, fmt, y_type):
    war = _war()
    rng = np.random.default_rng(M + N + K)
    (x, xn), (w, wn) = coded(rng, M, K, fmt, True, pad=16), coded(rng, N, K, "e2m1", True)
    bias = torch.tensor(rng.integers(-64, 65, N) / 4).bfloat16().to(DEV)
    for b in (None, bias):
        lin = war.Linear(w, b)
        y = padded(M, N, 3, y_type, 9.0)
        war.linear(lin, x, y)
        want = torch.tensor(xn @ wn.T + (0.0 if b is None else as64(b))).float()
        assert float(want.abs().max()) < 2.0 ** 14
        torch.testing.assert_close(y.cpu(), want.to(y_type), rtol=0, atol=0)
        assert bool((y._base[:, N:] == 9).all())
    even = torch.full((M, -(-N // 8) * 8), 9.0, dtype=y_type, device=DEV)     # rows that may be written in wide pieces
    war.linear(lin, x, even[:, :N])
    assert torch.equal(even[:, :N], y) and bool((even[:, N:] == 9).all())


@pytest.mark.parametrize("y_type", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("shape", range(10))
def test_every_shape_of_workgroups(shape, fmt, y_type):
    """Each shape on rows, columns and blocks that fill no tile, one step and many, scales
    that are read one at a time and four, whatever shape such a product would get."""
    war = _war()
    rng = np.random.default_rng(shape)
    for M, N, K, pad in ((1, 1, 32, 16), (33, 129, 64, 16), (97, 260, 160, 0), (130, 65, 512, 48), (17, 300, 544, 16), (258, 513, 1024, 16),
                         (100, 40, 2080, 16), (40, 257, 3584, 0)):
        (x, xn), (w, wn) = coded(rng, M, K, fmt, True, pad=pad), coded(rng, N, K, "e2m1", True)
        x.whole[1][M:] = 255
        bias = torch.tensor(rng.integers(-64, 65, N) / 4).bfloat16().to(DEV)
        lin = war.Linear(w, bias)
        want = torch.tensor(xn @ wn.T + as64(bias)).float().to(y_type)
        for gap in (3, -N % 8):
            y = padded(M + 1, N, gap, y_type, 9.0)
            war.debug_linear(lin, x, y[:M], shape)
            torch.testing.assert_close(y[:M].cpu(), want, rtol=0, atol=0)
            assert bool((y._base[:, N:] == 9).all()) and bool((y._base[M] == 9).all())


@pytest.mark.parametrize("y_type", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("bm,bn,shape", [(128, 128, 5), (96, 256, 6), (128, 256, 7), (192, 256, 8), (256, 256, 9)])
def test_more_tiles_than_compute_units(bm, bn, shape, fmt, y_type):
    """Several bands of tiles on every XCD, the last ones not whole, of one step of the
    columns and of several."""
    war = _war()
    rng = np.random.default_rng(shape)
    M, N = 24 * bm + 17, 22 * bn + 9
    for K, gap in ((96, 7), (672, 1)):
        (x, xn), (w, wn) = coded(rng, M, K, fmt, True), coded(rng, N, K, "e2m1", True)
        bias = torch.tensor(rng.integers(-64, 65, N) / 4).bfloat16().to(DEV)
        lin = war.Linear(w, bias)
        y = padded(M + 1, N, gap, y_type, 9.0)
        war.debug_linear(lin, x, y[:M], shape)
        want = torch.tensor(xn @ wn.T + as64(bias)).float().to(y_type)
        assert torch.equal(y[:M].cpu(), want)
        assert bool((y._base[:, N:] == 9).all()) and bool((y._base[M] == 9).all())


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("M,N,K", [(3, 40, 4096), (65, 96, 2080), (200, 384, 1536), (520, 140, 768)])
def test_products_of_activations(M, N, K, fmt):
    war = _war()
    rng = np.random.default_rng(M)
    (x, xn), (w, wn) = coded(rng, M, K, fmt, False), coded(rng, N, K, "e2m1", False)
    lin = war.Linear(w)
    y = war.linear(lin, x, torch.empty((M, N), device=DEV))
    want = xn @ wn.T
    assert (np.abs(as64(y) - want) <= product_tolerance(xn, wn, fmt, torch.float32)).all()
    z, tol = war.linear(lin, x, torch.empty((M, N), dtype=torch.bfloat16, device=DEV)), product_tolerance(xn, wn, fmt)
    assert (np.abs(as64(z) - want) <= (1 + 2.0 ** -8) * tol + 2.0 ** -8 * np.abs(want)).all()
    if fmt == "e2m1":
        assert torch.equal(z, y.bfloat16())
    again = war.linear(lin, x, torch.empty((M, N), device=DEV))
    assert torch.equal(y, again)


@pytest.mark.parametrize("fmt", FMTS)
@pytest.mark.parametrize("M", [3, 40, 300])
def test_scales_of_every_size_and_rows_that_are_not_finite(M, fmt):
    war = _war()
    rng = np.random.default_rng(M)
    N, K = 50, 672
    (x, xn), (w, wn) = coded(rng, M, K, fmt, True), coded(rng, N, K, "e2m1", True)
    # a row by 2^100, a column by 2^-100, a row by 2^-120; a column that reads as NaN, a row too
    sx, sw = x.scales.cpu().numpy().astype(np.int64), w.scales.cpu().numpy().astype(np.int64)
    sx[0] += 100
    sx[2] -= 120
    sw[7] -= 100
    sx[1, 20], sw[9, 0] = 255, 255
    x.scales.copy_(torch.tensor(sx, dtype=torch.uint8))
    w.scales.copy_(torch.tensor(sw, dtype=torch.uint8))
    xn, wn = omx.numbers(codes_of(x)[0], sx, fmt), omx.numbers(codes_of(w)[0], sw, "e2m1")
    y = war.linear(war.Linear(w), x, torch.empty((M, N), device=DEV)).cpu()
    want = torch.tensor(np.where(np.isnan(xn).any(1)[:, None] | np.isnan(wn).any(1)[None], np.nan,
                                 np.nan_to_num(xn) @ np.nan_to_num(wn).T)).float()
    keep = want.abs() >= 2.0 ** -120   # (2^-120 * 2^-100 leaves the range of fp32)
    keep |= torch.isnan(want)
    torch.testing.assert_close(y[keep], want[keep], rtol=0, atol=0, equal_nan=True)
    assert float(y[~keep].abs().max()) < 2.0 ** -119 if bool((~keep).any()) else True


def test_a_row_does_not_depend_on_the_rows_beside_it():
    """Zero, one and all rows; rows past the last of a view are not read as numbers."""
    war = _war()
    rng = np.random.default_rng(2)
    (x, _), (w, _) = coded(rng, 90, 1056, "e4m3", False), coded(rng, 200, 1056, "e2m1", False)
    lin = war.Linear(w)
    for n in (1, 16, 17, 64, 90):
        y = war.linear(lin, x[:n], torch.empty((n, 200), device=DEV))
        bad = mx_of(90, 1056, "e4m3")
        bad.codes.copy_(x.codes)
        bad.scales.copy_(x.scales)
        bad.codes[n:], bad.scales[n:] = 0x7f, 255
        assert torch.equal(war.linear(lin, bad[:n], torch.empty((n, 200), device=DEV)), y)
        if n > 1:
            bad.codes[1:n], bad.scales[1:n] = 0x7f, 255
            z = war.linear(lin, bad[:n], torch.empty((n, 200), device=DEV))
            assert torch.equal(z[0], y[0]) and bool(z[1:].isnan().all())
    out = torch.full((1, 200), 5.0, device=DEV)
    war.linear(lin, x[:0], out[:0])
    war.quantize(torch.empty((0, 1056), device=DEV), x[:0])
    assert bool((out == 5).all())


def test_scale_bytes_behind_the_last_block_do_not_count():
    war = _war()
    rng = np.random.default_rng(3)
    for K in (32, 96, 544, 1120):
        for M in (5, 200):
            (x, xn), (w, wn) = coded(rng, M, K, "e4m3", True), coded(rng, 40, K, "e2m1", True)
            lin = war.Linear(w)
            want = war.linear(lin, x, torch.empty((M, 40), device=DEV))
            x.whole[1][:, K // 32:] = 255
            assert torch.equal(war.linear(lin, x, torch.empty((M, 40), device=DEV)), want)


def test_weights_from_a_matrix_and_any_place_of_their_codes():
    war = _war()
    g = torch.Generator(device=DEV).manual_seed(4)
    wf = torch.randn((70, 320), device=DEV, generator=g).bfloat16()
    x = war.quantize(torch.randn((9, 320), device=DEV, generator=g), war.Mx.empty(9, 320, "e4m3", DEV))
    a = war.Linear(wf)
    m = war.quantize(wf, war.Mx.empty(70, 320, "e2m1", DEV))
    raw = torch.zeros(70 * 163 + 5, dtype=torch.uint8, device=DEV)
    odd = raw[5:].view(70, 163)[:, :160]
    odd.copy_(m.codes)
    b = war.Linear(war.Mx(odd, m.scales.contiguous(), "e2m1"))
    ya, yb = (war.linear(l, x, torch.empty((9, 70), device=DEV)) for l in (a, b))
    assert torch.equal(ya, yb)
    a.close()
    with pytest.raises(ValueError):
        war.linear(a, x, ya)


# ------------------------------------------------------------------------- rope
def pool_of(heads, tokens, fmt, layers=1):
    war = _war()
    cfg = synth.ModelConfig(n_layers=layers, d_model=128, n_q_heads=heads[0], n_kv_heads=heads[1], head_dim=heads[2], ffn_dim=128, vocab=128)
    pages = [-(-t // 16) for t in tokens]
    pool = war.Pool(cfg, sum(pages) + 2, len(tokens), max(max(pages), 1), device=DEV, kv_format=fmt)
    pool.kv.view(torch.uint8).fill_(255)
    for part in range(1, 5):
        pool.alloc(list(range(len(tokens))), [t * part // 4 for t in tokens])
    return pool


AXES = {"one": lambda n: [0] * n, "blocks": lambda n: [0 if j < n // 4 else 1 + (j % 2) for j in range(n)], "turns": lambda n: [j % 4 for j in range(n)]}


@pytest.mark.parametrize("adjacent", [False, True])
def test_rope_of_numbers_that_are_not_finite(adjacent):
    """Infinities, NaN and turns past bf16's range are what the formula makes of them, and no
    other number's business."""
    war = _war()
    rng = np.random.default_rng(3)
    D, R, top = 64, 64, 3.3895313892515355e38
    x = rng.standard_normal((1, 4, 4, D))
    a, b = ([0, 2, 4, 6], [1, 3, 5, 7]) if adjacent else ([0, 1, 2, 3], [32, 33, 34, 35])
    for h in (0, 2):                                    # a query's head and a key's
        x[0, 0, h, a[0]], x[0, 1, h, b[1]], x[0, 2, h, a[2]] = np.inf, -np.inf, np.nan
        x[0, 3, h, a[3]] = x[0, 3, h, b[3]] = top
    x = torch.tensor(x).bfloat16().to(DEV)
    pool = pool_of((2, 1, D), [9], "bf16")
    out = torch.empty((1, 4, 2, D), dtype=torch.bfloat16, device=DEV)
    war.rope_write(pool, 0, war.Rope(D, R, adjacent=adjacent), t32([0]), t32([5]), x[:, :, :2], x[:, :, 2:3], x[:, :, 3:4], out)
    k, v = (torch.empty((1, 4, 1, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    war.kv_read(pool, 0, t32([0]), t32([5]), k, v)
    j = np.arange(R // 2)
    angle = np.arange(5, 9)[:, None, None] * 10000.0 ** (-2 * j / R)
    pairs = (slice(0, R, 2), slice(1, R, 2)) if adjacent else (slice(0, R // 2), slice(R // 2, R))
    z = as64(x[0])
    with np.errstate(invalid="ignore", over="ignore"):
        want = z.copy()
        want[..., pairs[0]] = z[..., pairs[0]] * np.cos(angle) - z[..., pairs[1]] * np.sin(angle)
        want[..., pairs[1]] = z[..., pairs[1]] * np.cos(angle) + z[..., pairs[0]] * np.sin(angle)
    want[np.abs(want) >= 3.4e38] *= np.inf              # (bf16's largest and half a step: 3.396e38)
    size = np.zeros_like(z)
    size[..., pairs[0]] = size[..., pairs[1]] = np.abs(z[..., pairs[0]]) + np.abs(z[..., pairs[1]])
    for got, lo in ((as64(out[0]), 0), (as64(k[0]), 2)):
        ref = want[:, lo:lo + got.shape[1]]
        assert (np.isnan(got) == np.isnan(ref)).all() and (np.isinf(got) == np.isinf(ref)).all()
        assert (np.sign(got) == np.sign(ref))[np.isinf(ref)].all()
        f = np.isfinite(ref)
        assert (np.abs(got[f] - ref[f]) <= 2.0 ** -8 * np.abs(ref[f]) + 2.0 ** -20 * size[:, lo:lo + got.shape[1]][f]).all()
    torch.testing.assert_close(v, x[:, :, 3:4], rtol=0, atol=0)


@pytest.mark.parametrize("axes", list(AXES))
@pytest.mark.parametrize("rotary,adjacent", [(1.0, False), (0.5, True), (0.5, False), (1.0, True), (24, False)])
@pytest.mark.parametrize("heads", [(4, 2, 64), (32, 8, 128), (9, 3, 128)])
def test_rope_write(heads, rotary, adjacent, axes):
    """Angles are off by under 2^-21 and by 2^-51 of themselves; then one rounding."""
    war = _war()
    rng = np.random.default_rng(7)
    nq, nkv, D = heads
    R = int(D * rotary) if isinstance(rotary, float) else rotary
    pos, n, n_max = [0, 5, 16, 31, 47, 0, 300], [1, 0, 16, 40, 2, 37, 40], 40
    B = len(pos)
    ax, freqs = AXES[axes](R // 2), [1e6 ** (-2 * j / R) for j in range(R // 2)]
    rope = war.Rope(D, R, base=1e6, axes=ax, adjacent=adjacent)
    x = torch.tensor(rng.standard_normal((B, n_max, nq + 2 * nkv + 1, D))).bfloat16().to(DEV)      # rows with a gap behind them
    q, k, v = x[:, :, :nq], x[:, :, nq:nq + nkv], x[:, :, nq + nkv:nq + 2 * nkv]
    positions = rng.integers(-1000, 100000, (rope.n_axes, B, n_max))
    positions[:, 3, 7] = [2 ** 31 - 1, -2 ** 31, 2 ** 30 + 1, 0][: rope.n_axes]
    ids = t32(np.arange(B)[::-1].copy())
    pools = {f: pool_of(heads, [p + n_max for p in pos][::-1], f, layers=2) for f in ("bf16", "e4m3")}
    outs = {}
    for f, pool in pools.items():
        before = pool.kv.clone().view(torch.uint8)
        out = torch.full((B, n_max, nq, D), 7.0, dtype=torch.bfloat16, device=DEV)
        war.rope_write(pool, 1, rope, ids, t32(pos), q, k, v, out, t32(n), positions=t32(positions))
        got = [torch.full((B, n_max, nkv, D), 7.0, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        war.kv_read(pool, 1, ids, t32(pos), *got, t32(n))
        assert pool.state()["status"] == 0
        outs[f] = [out, *got]
        # kv_write of the same bf16 numbers stores the same bytes, and touches no others
        again = pool_of(heads, [p + n_max for p in pos][::-1], f, layers=2)
        war.kv_write(again, 1, ids, t32(pos), outs["bf16"][1], v, t32(n))
        assert torch.equal(again.kv.view(torch.uint8), pool.kv.view(torch.uint8))
        assert not torch.equal(before, pool.kv.view(torch.uint8))
    assert torch.equal(outs["bf16"][0], outs["e4m3"][0])
    for b in range(B):
        p = positions[:, b, : n[b]]
        t = np.abs(p.max(0, initial=0)).astype(float)
        ang = 2.0 ** -21 + np.abs(p).max(0, initial=0)[:, None, None] * 2.0 ** -51
        for src, got in ((q, outs["bf16"][0]), (k, outs["bf16"][1])):
            xb = as64(src[b, : n[b]])
            want = omx.turned(xb, p, ax, freqs, adjacent)
            other = omx.turned(np.abs(xb), np.zeros_like(p), ax, freqs, adjacent)
            size = np.abs(xb).max(-1, keepdims=True)
            assert (np.abs(as64(got[b, : n[b]]) - want) <= 2.0 ** -8 * np.abs(want) + ang * 2 * size).all()
            np.testing.assert_array_equal(as64(got[b, : n[b]])[..., R:], xb[..., R:])
            assert bool((got[b, n[b]:] == 7).all())
        assert torch.equal(outs["bf16"][2][b, : n[b]], v[b, : n[b]])


def test_rope_in_place_by_default_positions_and_one_row_at_a_time():
    war = _war()
    heads, B, n = (8, 2, 128), 3, 21
    g = torch.Generator(device=DEV).manual_seed(5)
    x = torch.randn((B, n, 12, 128), device=DEV, generator=g).bfloat16()
    ctx = [3, 40, 16]
    rope = war.Rope(128, base=500000.0)
    a, b, c = (pool_of(heads, [p + n for p in ctx], "e4m3") for _ in range(3))
    out = torch.empty((B, n, 8, 128), dtype=torch.bfloat16, device=DEV)
    war.rope_write(a, 0, rope, t32([0, 1, 2]), t32(ctx), x[:, :, :8], x[:, :, 8:10], x[:, :, 10:], out)
    pos = t32([[[p + i for i in range(n)] for p in ctx]] + [[[-1] * n] * B])      # an axis that no pair follows
    y = x.clone()
    war.rope_write(b, 0, rope, t32([0, 1, 2]), t32(ctx), y[:, :, :8], y[:, :, 8:10], y[:, :, 10:], y[:, :, :8], positions=pos)
    assert torch.equal(y[:, :, :8], out) and torch.equal(y[:, :, 8:], x[:, :, 8:])
    assert torch.equal(a.kv, b.kv)
    one = torch.empty((B, 1, 8, 128), dtype=torch.bfloat16, device=DEV)
    for i in range(n):
        war.rope_write(c, 0, rope, t32([0, 1, 2]), t32([p + i for p in ctx]), x[:, i:i + 1, :8], x[:, i:i + 1, 8:10], x[:, i:i + 1, 10:], one)
        assert torch.equal(one[:, 0], out[:, i])
    assert torch.equal(a.kv, c.kv)


def test_rope_flags_what_kv_write_flags():
    war = _war()
    heads = (4, 2, 64)
    x = torch.ones((4, 5, 8, 64), dtype=torch.bfloat16, device=DEV)
    x[3, 2, 5, 9] = float("nan")                       # a key of request 3: its token reads as NaN, others do not
    pool = pool_of(heads, [16, 16, 16, 16], "e4m3")
    out = torch.full((4, 5, 4, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    rope = war.Rope(64)
    war.rope_write(pool, 0, rope, t32([0, 9, 2, 3]), t32([0, 0, 12, 11]), x[:, :, :4], x[:, :, 4:6], x[:, :, 6:], out)
    assert pool.state()["status"] == -5 and pool.state()["status"] == 0
    assert bool((out[1:3] == 7).all()) and not bool((out[0] == 7).any())
    k, v = (torch.zeros((4, 5, 2, 64), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    war.kv_read(pool, 0, t32([3]), t32([11]), k[3:], v[3:])
    bad = torch.zeros((5, 2), dtype=torch.bool)
    bad[2, 1] = True
    assert torch.equal(k[3].isnan().all(-1).cpu(), bad) and torch.equal(v[3].isnan().all(-1).cpu(), bad)
    for wrong in (dict(rope=war.Rope(128)), dict(positions=t32(np.zeros((1, 3, 5)))), dict(out=out[:3])):
        with pytest.raises(ValueError):
            war.rope_write(pool, 0, wrong.get("rope", rope), t32([0, 1, 2, 3]), t32([0] * 4), x[:, :, :4], x[:, :, 4:6], x[:, :, 6:],
                           wrong.get("out", out), positions=wrong.get("positions"))
    with pytest.raises(war.WarError):
        war.rope_write(pool, 1, rope, t32([0, 1, 2, 3]), t32([0] * 4), x[:, :, :4], x[:, :, 4:6], x[:, :, 6:], out)


# -------------------------------------------------------------- a layer of them
class Layer:
    """A decoder layer of the operators, as a program whose weights are in 4 bits runs it."""

    def __init__(self, war, cfg, fmt, seed=0):
        rng = np.random.default_rng(seed)
        D, H = cfg.head_dim, cfg.n_q_heads + 2 * cfg.n_kv_heads
        mat = lambda n, k: torch.tensor(rng.standard_normal((n, k)) * k ** -0.5).bfloat16().to(DEV)
        self.war, self.cfg, self.fmt = war, cfg, fmt
        self.norms = [torch.tensor(1 + 0.1 * rng.standard_normal(cfg.d_model)).bfloat16().to(DEV) for _ in range(2)]
        self.ws = dict(qkv=mat(H * D, cfg.d_model), o=mat(cfg.d_model, cfg.n_q_heads * D), up=mat(2 * cfg.ffn_dim, cfg.d_model),
                       down=mat(cfg.d_model, cfg.ffn_dim))
        self.bias = torch.tensor(rng.standard_normal(H * D) * 0.1).bfloat16().to(DEV)
        self.lin = {n: war.Linear(w, self.bias if n == "qkv" else None) for n, w in self.ws.items()}
        self.rope = war.Rope(D, base=1e6, axes=[j % 3 for j in range(D // 2)])

    def buffers(self, B, n):
        c, war, R = self.cfg, self.war, B * n
        H = c.n_q_heads + 2 * c.n_kv_heads
        bf = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device=DEV)
        return dict(u=war.Mx.empty(R, c.d_model, self.fmt, DEV), qkv=bf(R, H * c.head_dim), q=bf(B, n, c.n_q_heads, c.head_dim),
                    o=bf(B, n, c.n_q_heads, c.head_dim), om=war.Mx.empty(R, c.n_q_heads * c.head_dim, self.fmt, DEV), a=bf(R, c.d_model),
                    f=war.Mx.empty(R, c.d_model, self.fmt, DEV), gu=bf(R, 2 * c.ffn_dim), g=war.Mx.empty(R, c.ffn_dim, self.fmt, DEV),
                    y=bf(R, c.d_model))

    def run(self, h, x, pool, plan, ids, ctx, lens, positions, w, stream=None):
        war, c = self.war, self.cfg
        with torch.cuda.stream(stream or torch.cuda.current_stream()):
            w["o"].zero_()                      # rows beyond a request's live ones stay as they are
        B, n = w["q"].shape[:2]
        s = dict(stream=stream)
        war.residual_norm(x, h, self.norms[0], 1e-6, w["u"], **s)
        war.linear(self.lin["qkv"], w["u"], w["qkv"], **s)
        qkv = w["qkv"].view(B, n, -1, c.head_dim)
        war.rope_write(pool, 0, self.rope, ids, ctx, qkv[:, :, :c.n_q_heads], qkv[:, :, c.n_q_heads:c.n_q_heads + c.n_kv_heads],
                       qkv[:, :, c.n_q_heads + c.n_kv_heads:], w["q"], lens, positions, **s)
        plan.update(ids, ctx, lens, **s)
        war.attend(plan, 0, w["q"], w["o"], **s)
        war.quantize(w["o"].view(B * n, -1), w["om"], **s)
        war.linear(self.lin["o"], w["om"], w["a"], **s)
        war.residual_norm(w["a"], h, self.norms[1], 1e-6, w["f"], **s)
        war.linear(self.lin["up"], w["f"], w["gu"], **s)
        war.quantize(w["gu"][:, c.ffn_dim:], w["g"], gate=w["gu"][:, :c.ffn_dim], **s)
        return war.linear(self.lin["down"], w["g"], w["y"], **s)


def numbers_of(m):
    return omx.numbers(*codes_of(m), m.format)


@pytest.mark.parametrize("fmt", FMTS)
def test_a_layer_each_operator_against_the_oracle_on_what_the_one_before_left(fmt):
    war = _war()
    cfg = synth.TINY
    layer = Layer(war, cfg, fmt)
    B, n, lens, ctx = 3, 5, [5, 3, 1], [20, 0, 33]
    g = torch.Generator(device=DEV).manual_seed(9)
    R, nq, nkv, D, F = B * n, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim, cfg.ffn_dim
    pool = pool_of((nq, nkv, D), [c + n for c in ctx], "e4m3")
    ids = t32([2, 0, 1])
    pool = pool_of((nq, nkv, D), [ctx[i] + n for i in (1, 2, 0)], "e4m3")
    past = [torch.randn((B, max(ctx), nkv, D), device=DEV, generator=g).bfloat16() for _ in range(2)]
    war.kv_write(pool, 0, ids, t32([0] * B), *past, t32(ctx))
    h = torch.randn((R, cfg.d_model), device=DEV, generator=g)
    x = torch.randn((R, cfg.d_model), device=DEV, generator=g).bfloat16()
    positions = torch.randint(0, 500, (3, B, n), device=DEV, generator=g, dtype=torch.int32)
    w = layer.buffers(B, n)
    plan = war.AttendPlan(pool, B, n)
    h1 = as64(h + x.float())
    y = layer.run(h, x, pool, plan, ids, t32(ctx), t32(lens), positions, w)
    ws = {k: omx.numbers(*omx.quantise(as64(v), "e2m1"), "e2m1") for k, v in layer.ws.items()}

    def product(name, m, got, bias=0.0):
        x64 = numbers_of(m)
        tol = product_tolerance(x64, ws[name], fmt)
        want = x64 @ ws[name].T + bias
        assert (np.abs(as64(got) - want) <= 2.0 ** -8 * np.abs(want) + 1.01 * tol + 2.0 ** -22 * np.abs(want)).all(), name

    check_codes(w["u"], omx.norm(h1, as64(layer.norms[0]), 1e-6), NORM_REL, 1e-38)
    product("qkv", w["u"], w["qkv"], as64(layer.bias))
    qkv = as64(w["qkv"]).reshape(R, -1, D)
    turned = omx.turned(qkv[:, : nq + nkv], positions.reshape(3, R).cpu().numpy(), [j % 3 for j in range(D // 2)],
                        [1e6 ** (-2 * j / D) for j in range(D // 2)], False)
    live = np.concatenate([np.arange(n) < m for m in lens])
    size = np.abs(qkv[:, : nq + nkv]).max(-1, keepdims=True)
    got_q = as64(w["q"]).reshape(R, nq, D)
    assert (np.abs(got_q - turned[:, :nq]) <= 2.0 ** -8 * np.abs(turned[:, :nq]) + 2.0 ** -20 * size[:, :nq])[live].all()
    assert (got_q[~live] == 0).all()
    ks, vs = (torch.zeros((B, max(ctx) + n, nkv, D), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    war.kv_read(pool, 0, ids, t32([0] * B), ks, vs, t32([c + m for c, m in zip(ctx, lens)]))
    kv = [as64(t) for t in (ks, vs)]
    for b in range(B):
        for i in range(lens[b]):
            r, s = b * n + i, ctx[b] + i
            # a key is off by half a step of e4m3 in its block (2^-4 of the number, 2^-10 of the scale) behind bf16's
            assert (np.abs(kv[0][b, s] - turned[r, nq:]) <= 0.07 * np.abs(turned[r, nq:]) + 2.0 ** -9 * size[r, nq:]).all()
            for hq in range(nq):
                k, v = kv[0][b, : s + 1, hq // (nq // nkv)], kv[1][b, : s + 1, hq // (nq // nkv)]
                z = got_q[r, hq] @ k.T / np.sqrt(D)
                p = np.exp(z - z.max())
                p /= p.sum()
                # weights and output in bf16 or better, scores to 2^-20 of their magnitudes
                tol = 2.0 ** -8 * np.abs(p @ v) + (2.0 ** -8 + 2.0 ** -18 * np.abs(got_q[r, hq]) @ np.abs(k).max(0)) * (p @ np.abs(v))
                assert (np.abs(as64(w["o"])[b, i, hq] - p @ v) <= tol).all()
    check_codes(w["om"], as64(w["o"]).reshape(R, -1))
    product("o", w["om"], w["a"])
    h2 = as64(torch.tensor(h1).float() + w["a"].float().cpu())
    np.testing.assert_array_equal(as64(h), h2)
    check_codes(w["f"], omx.norm(h2, as64(layer.norms[1]), 1e-6), NORM_REL, 1e-38)
    product("up", w["f"], w["gu"])
    gu = as64(w["gu"])
    check_codes(w["g"], omx.gated(gu[:, F:], gu[:, :F]), 2.0 ** -20, 3e-37 * np.abs(gu[:, F:]))
    product("down", w["g"], y)


def test_a_layer_on_another_stream_and_captured():
    """The same layer eagerly, on a stream of its own, and replayed from a graph between
    eager work, over inputs that change: the same bits each time."""
    war = _war()
    cfg = synth.TINY
    layer = Layer(war, cfg, "e4m3", seed=3)
    B, n, ctx = 4, 3, [7, 31, 0, 64]
    g = torch.Generator(device=DEV).manual_seed(2)
    heads = (cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim)
    past = [torch.randn((B, max(ctx), heads[1], heads[2]), device=DEV, generator=g).bfloat16() for _ in range(2)]
    inputs = [(torch.randn((B * n, cfg.d_model), device=DEV, generator=g), torch.randn((B * n, cfg.d_model), device=DEV, generator=g).bfloat16(),
               torch.randint(0, 99, (3, B, n), device=DEV, generator=g, dtype=torch.int32), t32(rng)) for rng in ([3, 1, 2, 3], [1, 3, 3, 0], [3, 3, 3, 3])]
    ids, d_ctx = t32(range(B)), t32(ctx)

    def setup():
        pool = pool_of(heads, [c + n for c in ctx], "e4m3")
        war.kv_write(pool, 0, ids, t32([0] * B), *past, t32(ctx))
        return pool, war.AttendPlan(pool, B, n), layer.buffers(B, n)

    pool, plan, w = setup()
    want = []
    for h, x, pos, lens in inputs:
        hh = h.clone()
        y = layer.run(hh, x, pool, plan, ids, d_ctx, lens, pos, w).clone()
        want.append((hh, y))
    stream = torch.cuda.Stream()
    pool2, plan2, w2 = setup()
    bufs = [t.clone() for t in inputs[0]]
    stream.wait_stream(torch.cuda.current_stream())
    for (h, x, pos, lens), (hh, y) in zip(inputs, want):
        with torch.cuda.stream(stream):
            h2 = h.clone()
        y2 = layer.run(h2, x, pool2, plan2, ids, d_ctx, lens, pos, w2, stream=stream)
        stream.synchronize()
        assert torch.equal(h2, hh) and torch.equal(y2, y)
    graph = torch.cuda.CUDAGraph()
    pool3, plan3, w3 = setup()
    with torch.cuda.graph(graph):
        y3 = layer.run(bufs[0], bufs[1], pool3, plan3, ids, d_ctx, bufs[3], bufs[2], w3)
    for turn in range(3):
        for given, (hh, y) in zip(inputs, want):
            for dst, src in zip(bufs, given):
                dst.copy_(src)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(bufs[0], hh) and torch.equal(y3, y)
            again = given[0].clone()
            assert torch.equal(layer.run(again, given[1], pool, plan, ids, d_ctx, given[3], given[2], w), y)


def test_two_products_at_once_on_two_streams():
    war = _war()
    rng = np.random.default_rng(8)
    (x, _), (w, _) = coded(rng, 200, 2048, "e4m3", False), coded(rng, 1024, 2048, "e2m1", False)
    lin = war.Linear(w)
    want = war.linear(lin, x, torch.empty((200, 1024), device=DEV))
    streams = [torch.cuda.Stream() for _ in range(2)]
    ys = [torch.zeros((200, 1024), device=DEV) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, y in zip(streams, ys):
            war.linear(lin, x, y, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(y, want) for y in ys)


# ----------------------------------------------------------------- large offsets
def test_matrices_past_4_gb():
    """Codes, numbers and products at offsets that 32 bits do not hold."""
    war = _war()
    rows, cols = 70000, 65536
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device=DEV)
    pattern = torch.linspace(-3, 3, cols, device=DEV).bfloat16()
    x[-3:] = pattern
    m = war.Mx.empty(rows, cols, "e4m3", DEV)
    war.quantize(x, m)
    want = war.quantize(x[-3:].clone(), war.Mx.empty(3, cols, "e4m3", DEV))
    assert torch.equal(m.codes[-3:], want.codes) and torch.equal(m.scales[-3:], want.scales)
    x.fill_(5)
    war.dequantize(m, x)
    assert torch.equal(x[-3:], war.dequantize(want, torch.empty((3, cols), dtype=torch.bfloat16, device=DEV)))
    assert not bool(x[0].any()) and not bool(x[rows // 2].any())
    lin = war.Linear(torch.ones((24, cols), device=DEV))
    y = war.linear(lin, m, torch.empty((rows, 24), device=DEV))
    assert torch.equal(y[-3:], war.linear(lin, m[rows - 3:], torch.empty((3, 24), device=DEV))) or rows > 16
    ref = war.linear(lin, want, torch.empty((3, 24), device=DEV))
    np.testing.assert_allclose(as64(y[-3:]), as64(ref), atol=2.0 ** -10 * float(pattern.float().abs().sum()) / 100)
    assert not bool(y[: rows - 3].any())
    del x, m, y
    h = torch.zeros((70000, 32768), device=DEV)          # 9 GB
    h[-1] = 1.0
    out = war.residual_norm(None, h, torch.ones(32768, device=DEV).bfloat16(), 0.5, war.Mx.empty(70000, 32768, "e2m1", DEV))
    back = war.dequantize(out[69999:], torch.empty((1, 32768), device=DEV))
    assert float(back.min()) == float(back.max()) > 0.7 and not bool(out.codes[69998].any())
    del h, out
    # outputs
    big = torch.empty((9000, 131072 + 8), device=DEV)    # 4.7 GB
    wide = war.Linear(torch.ones((131072, 32), device=DEV))
    a = war.quantize(torch.arange(9000, device=DEV).view(-1, 1).expand(9000, 32).contiguous().float(), war.Mx.empty(9000, 32, "e4m3", DEV))
    war.linear(wide, a, big[:, :131072])
    num = war.dequantize(a, torch.empty((9000, 32), device=DEV))
    assert torch.equal(big[:, 0], num.sum(1)) and torch.equal(big[:, 131071], num.sum(1)) and torch.equal(big[8999, :131072].min(), big[8999, 0])


def test_no_rows():
    """Empty batches are no work for any of the operators."""
    war = _war()
    bf = lambda *shape: torch.empty(shape, dtype=torch.bfloat16, device=DEV)
    gain, m = torch.ones(64, device=DEV).bfloat16(), war.Mx.empty(0, 64, "e4m3", DEV)
    for h in (bf(0, 64), torch.empty((0, 64), device=DEV)):
        for x in (None, bf(0, 64)):
            for out in (bf(0, 64), m, war.Mx.empty(0, 64, "e2m1", DEV)):
                war.residual_norm(x, h, gain, 1e-6, out)
    war.quantize(bf(0, 64), m, gate=bf(0, 64))
    war.dequantize(m, bf(0, 64))
    war.linear(war.Linear(torch.ones((24, 64), device=DEV)), m, bf(0, 24))
    pool = pool_of((4, 2, 64), [16], "bf16")
    war.rope_write(pool, 0, war.Rope(64), t32([0]), t32([3]), bf(1, 0, 4, 64), bf(1, 0, 2, 64), bf(1, 0, 2, 64), bf(1, 0, 4, 64))
    torch.cuda.synchronize()
    assert pool.state()["status"] == 0


@pytest.mark.parametrize("fmt", FMTS)
def test_gates_whose_exp_is_close_to_the_largest_number(fmt):
    """Down to a gate of -88.7, where exp(-g) is 2^127.97, the result is not zero: its
    reciprocal is below the smallest normal number, its product with x need not be."""
    war = _war()
    near = torch.cat([torch.linspace(-88.7, -86.0, 32 * 20), torch.linspace(-87.4, -87.3, 32 * 4)]).view(-1, 32)
    for g in (near, (torch.arange(32 * 6) // 32 * 0.5 - 88.5).view(-1, 32).bfloat16()):
        for x in (1.0, -1e30, 3e38, 2.0 ** 40):
            x = torch.full_like(g, x).to(DEV)
            m = mx_of(len(g), 32, fmt)
            war.quantize(x, m, gate=g.to(DEV))
            check_codes(m, omx.gated(as64(x), as64(g)), 2.0 ** -20)

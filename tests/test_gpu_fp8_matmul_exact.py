"""zc_fp8_matmul on operands whose sums are whole numbers of quarters, exact in FP32 in any order: every element has to be right to the
bit, so a product too many or too few, a wrong scale byte or a sum that starts from a stale accumulator shows.  The sizes take the kernel
of block pairs through several scale words a tile and several tiles a pair, as a training step's do."""
import pytest
import torch

from paper_2508_19263_b200 import binding as zc

pytestmark = pytest.mark.gpu
DEV = "cuda"
REAL = [torch.float32, torch.bfloat16, torch.float16]
FP8 = {zc.FMT_FP8_E4M3: torch.float8_e4m3fn, zc.FMT_FP8_E5M2: torch.float8_e5m2}


def matrix(rows, cols, fmt, block, seed):
    """Elements -3 .. 3, scales 1/2, 1 and 2; what lies behind the columns and rows of scale bytes is NaN.  (matrix, its values in 64 bits)"""
    g = torch.Generator(device=DEV).manual_seed(seed)
    pitch = -(-cols // 16) * 16 + 16
    buf = torch.full((rows, pitch), 0x7F, dtype=torch.uint8, device=DEV)
    elems = buf[:, :cols]
    elems.copy_(torch.randint(-3, 4, (rows, cols), generator=g, device=DEV).float().to(FP8[fmt]).view(torch.uint8))
    shape = (-(-rows // block), -(-cols // 128))
    scales = torch.full((shape[0], shape[1] + 3), 255, dtype=torch.uint8, device=DEV)[:, : shape[1]]
    scales.copy_(torch.randint(126, 129, shape, generator=g, device=DEV, dtype=torch.uint8))
    s = torch.exp2(scales.double() - 127).repeat_interleave(block, 0)[:rows].repeat_interleave(128, 1)[:, :cols]
    return zc.Fp8Matrix(elems, scales, fmt, block), elems.view(FP8[fmt]).double() * s


def result(m, n, pitch, dtype, seed=None):
    """A result inside a larger buffer, of whole numbers where it is added to; (result, buffer)."""
    buf = torch.full((m + 1, pitch), 7.0, dtype=dtype, device=DEV)
    d = buf[:m, :n]
    if seed is not None:
        d.copy_(torch.randint(-50, 51, (m, n), generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV))
    return d, buf


def check(m, n, k, fmt_a, fmt_b, block_a, block_b, dtypes=REAL, accumulates=(False, True), pitches=None):
    # a sum is at most 9 * 4 * k, in quarters below 2^24 for k up to 116508; what the result held adds 200 quarters
    a, va = matrix(m, k, fmt_a, block_a, m + k)
    b, vb = matrix(n, k, fmt_b, block_b, n + k + 1)
    exact = va @ vb.t()
    del va, vb
    for dtype in dtypes:
        for pitch in pitches or (n, n + 1, -(-n // 16) * 16):
            for accumulate in accumulates:
                d, buf = result(m, n, pitch, dtype, 5 if accumulate else None)
                want = (exact + d.double() if accumulate else exact).float().to(dtype)
                zc.fp8_matmul(a, b, d, accumulate=accumulate)
                assert torch.equal(d, want), (dtype, pitch, accumulate)
                assert bool((buf[m:] == 7).all()) and bool((buf[:, n:] == 7).all())      # nothing outside
    assert zc.fp8_status() == zc.OK


# 37 and more tiles of 256 x 256: the kernel of block pairs.  49, 56, 110 and 289 tiles on 74 pairs: one, two and four a pair, whole and
# ragged, one to 32 steps of 128 columns
PAIRS = [(1600, 1792, 1100), (1601, 1795, 2050), (2600, 2400, 4096), (4200, 4100, 1153), (1600, 1792, 100)]


@pytest.mark.parametrize("m,n,k", PAIRS)
@pytest.mark.parametrize("block_a", [1, 128])
@pytest.mark.parametrize("block_b", [1, 128])
def test_pairs(m, n, k, block_a, block_b):
    check(m, n, k, zc.FMT_FP8_E4M3, zc.FMT_FP8_E4M3, block_a, block_b)


@pytest.mark.parametrize("fmt_a,fmt_b", [(5, 2), (2, 5), (5, 5)])
@pytest.mark.parametrize("m,n,k", [(1601, 1800, 2050), (2600, 2400, 1024)])
def test_pairs_of_other_formats(m, n, k, fmt_a, fmt_b):
    check(m, n, k, fmt_a, fmt_b, 1, 128)


def test_pairs_over_many_columns():
    check(1600, 1792, 14336, zc.FMT_FP8_E4M3, zc.FMT_FP8_E4M3, 1, 128, accumulates=(False,))


SMALL = [(1, 4096, 4096), (1, 640, 14336), (64, 1000, 4096), (77, 1001, 2050), (300, 520, 1153), (128, 128, 8192), (513, 129, 31), (1024, 300, 2100)]


@pytest.mark.parametrize("m,n,k", SMALL)
@pytest.mark.parametrize("block_b", [1, 128])
def test_small_tiles(m, n, k, block_b):
    check(m, n, k, zc.FMT_FP8_E4M3, zc.FMT_FP8_E4M3, 1, block_b)


@pytest.mark.parametrize("tokens,n,k", [(2100, 1800, 2500)])
def test_linear_layer_of_a_training_step(tokens, n, k):
    """The three products of a linear layer on matrices as the quantiser makes them (whole numbers are quantised without a loss), each
    of a size for the kernel of block pairs; the weights' gradient is added to one that is there."""
    g = torch.Generator(device=DEV).manual_seed(61)
    x, w, dy = (torch.randint(-3, 4, s, generator=g, device=DEV).float() for s in ((tokens, k), (n, k), (tokens, n)))
    qx, qxt = zc.fp8_empty(tokens, k), zc.fp8_empty(k, tokens)
    qw, qwt = zc.fp8_empty(n, k, block_rows=128), zc.fp8_empty(k, n, block_rows=128)
    qd, qdt = zc.fp8_empty(tokens, n, zc.FMT_FP8_E5M2), zc.fp8_empty(n, tokens, zc.FMT_FP8_E5M2)
    zc.fp8_quantize(x, qx, qxt)
    zc.fp8_quantize(w, qw, qwt)
    zc.fp8_quantize(dy, qd, qdt)
    y, dx = torch.empty((tokens, n), dtype=torch.bfloat16, device=DEV), torch.empty((tokens, k), dtype=torch.bfloat16, device=DEV)
    dw = torch.randint(-50, 51, (n, k), generator=g, device=DEV).float()
    want = dw.double() + dy.double().t() @ x.double()
    zc.fp8_matmul(qx, qw, y)
    zc.fp8_matmul(qd, qwt, dx)
    zc.fp8_matmul(qdt, qxt, dw, accumulate=True)
    assert torch.equal(y, (x.double() @ w.double().t()).float().bfloat16())
    assert torch.equal(dx, (dy.double() @ w.double()).float().bfloat16())
    assert torch.equal(dw, want.float())


@pytest.mark.parametrize("n", [40, 300])
def test_more_rows_than_a_grid_has_blocks_along_its_second_axis(n):
    # 65536 tiles of 128 rows and a piece of one; 40 columns take the kernel of small tiles, 300 that of pairs
    m, k = 65536 * 128 + 77, 32
    a, va = matrix(m, k, zc.FMT_FP8_E4M3, 128, 81)
    b, vb = matrix(n, k, zc.FMT_FP8_E4M3, 1, 82)
    d = torch.full((m, n), 7.0, dtype=torch.float16, device=DEV)
    zc.fp8_matmul(a, b, d)
    for part in range(0, m, 1 << 20):
        assert torch.equal(d[part: part + (1 << 20)], (va[part: part + (1 << 20)] @ vb.t()).half())
    assert zc.fp8_status() == zc.OK


def positive(r, k, g):
    return zc.Fp8Matrix(torch.randint(0, 0x40, (r, k), generator=g, device=DEV, dtype=torch.uint8),
                        torch.full((r, -(-k // 128)), 127, dtype=torch.uint8, device=DEV), zc.FMT_FP8_E4M3, 1)


def short(k):
    """What a sum of k positive products may be short by: less than a unit, 2^-23, of the sum as it is after every 32 columns.  The sum grows
    evenly, so that is (k / 32 + 1) / 2 units of the whole; a product's deviation is 2.62 times its mean (that of the values of the 64 bytes
    0 .. 0x3F 1.34 times), so the average of the sums on the way is off by 2.62 / sqrt(12 k) of the whole, against its half, six standard
    deviations of which are 9.1 / sqrt(k)."""
    return (k / 32 + 1) * 2.0 ** -24 * (1 + 9.1 / k ** 0.5)


@pytest.mark.parametrize("k", [1024, 4096, 14336, 65536])
@pytest.mark.parametrize("m,n", [(1600, 1792), (128, 128)])
def test_sums_of_one_sign(m, n, k):
    g = torch.Generator(device=DEV).manual_seed(71)
    a, b = positive(m, k, g), positive(n, k, g)
    want = a.elems.view(torch.float8_e4m3fn).double() @ b.elems.view(torch.float8_e4m3fn).double().t()
    d = zc.fp8_matmul(a, b, torch.empty((m, n), device=DEV))
    assert ((d.double() - want) / want).abs().max().item() <= short(k)


def test_sums_of_one_sign_in_parts():
    # fourteen parts of 1024 columns, added to nearest: half a unit, 2^-24, of the sum each
    m, n, k, parts = 1600, 1792, 14336, 14
    g = torch.Generator(device=DEV).manual_seed(72)
    a, b = positive(m, k, g), positive(n, k, g)
    want = a.elems.view(torch.float8_e4m3fn).double() @ b.elems.view(torch.float8_e4m3fn).double().t()
    d = torch.zeros((m, n), device=DEV)
    for i in range(parts):
        x, y = (zc.Fp8Matrix(v.elems[:, i * 1024: (i + 1) * 1024], v.scales[:, i * 8: (i + 1) * 8], v.format, 1) for v in (a, b))
        zc.fp8_matmul(x, y, d, accumulate=True)
    assert ((d.double() - want) / want).abs().max().item() <= short(1024) + parts * 2.0 ** -24

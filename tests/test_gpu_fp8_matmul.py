"""zc_fp8_quantize and zc_fp8_matmul against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

import fp8_reference as ref
from paper_2508_19263_b200 import binding as zc

pytestmark = pytest.mark.gpu
DEV = "cuda"
REAL = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
FORMATS = [zc.FMT_FP8_E4M3, zc.FMT_FP8_E5M2]


def strided(rows, cols, pitch, dtype, fill=0, offset=0):
    """A matrix of the given row pitch inside a larger buffer that is filled with `fill`; (matrix, buffer)."""
    buf = torch.full((offset + rows * pitch,), fill, dtype=dtype, device=DEV)
    return buf[offset:].as_strided((rows, cols), (pitch, 1), offset), buf


def empty_matrix(rows, cols, fmt, block, fill=0xAB):
    pitch = -(-cols // 16) * 16 + 16
    elems, ebuf = strided(rows, cols, pitch, torch.uint8, fill)
    scales, sbuf = strided(-(-rows // block), -(-cols // 128), -(-cols // 128) + 3, torch.uint8, fill)
    return zc.Fp8Matrix(elems, scales, fmt, block), ebuf, sbuf


def untouched(buf, view, fill=0xAB):
    """Whether the bytes of `buf` that `view` does not cover still hold the fill."""
    mask = torch.ones_like(buf, dtype=torch.bool)
    mask.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(False)
    return bool((buf[mask] == fill).all())


def hostile(rows, cols, seed, dtype):
    """Values of very different sizes, zero blocks, ties, subnormals, infinities and NaN."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, cols), generator=g, dtype=torch.float64)
    x *= torch.exp2(torch.randint(-20, 12, (rows, 1), generator=g).double())
    flat = x.reshape(-1)
    n = flat.numel()
    at = torch.randperm(n, generator=g)
    flat[at[: n // 16]] = 0.0
    flat[at[n // 16: n // 16 + 8]] = torch.tensor([448.0, 464.0, 480.0, 57344.0, 61440.0, 1.0625, 17.0, 2.0 ** -9], dtype=torch.float64)[: max(0, min(8, n - n // 16))]
    if n > 300:
        flat[at[-1]], flat[at[-2]], flat[at[-3]] = float("nan"), float("inf"), -float("inf")
    if rows > 2:
        x[1] = 0.0
        x[2] = x[2].nan_to_num(0, 0, 0) * 1e-39 if dtype == torch.float32 else 0.0
    return x.to(dtype).to(DEV)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("src", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,cols,extra,offset", [(1, 1, 0, 0), (1, 128, 0, 0), (3, 129, 3, 1), (127, 250, 6, 0), (130, 384, 0, 0), (257, 1000, 24, 8), (128, 4096, 0, 0)])
def test_quantize_is_exact(fmt, block, src, rows, cols, extra, offset):
    x0 = hostile(rows, cols, rows + cols + fmt, REAL[src])
    x, _ = strided(rows, cols, cols + extra, REAL[src], 0, offset)
    x.copy_(x0)
    q, qe, qs = empty_matrix(rows, cols, fmt, block)
    t, te, ts = empty_matrix(cols, rows, fmt, block)
    only, _, _ = empty_matrix(rows, cols, fmt, block)
    only_t, _, _ = empty_matrix(cols, rows, fmt, block)
    zc.fp8_quantize(x, q, t)
    zc.fp8_quantize(x, only)
    zc.fp8_quantize(x, None, only_t)
    x64 = x0.double().cpu().numpy()
    for m, want in ((q, x64), (only, x64), (t, x64.T), (only_t, x64.T)):
        elems, scales, nan = ref.quantize(np.ascontiguousarray(want), fmt, block)
        got = m.elems.cpu().numpy()
        assert np.array_equal(m.scales.cpu().numpy(), scales)
        assert np.array_equal(np.isnan(ref.table(fmt)[got]), nan)
        assert np.array_equal(got[~nan], elems[~nan])            # rounding to FP8 is exact arithmetic: no tolerance
    for buf, view in ((qe, q.elems), (qs, q.scales), (te, t.elems), (ts, t.scales)):
        assert untouched(buf, view)


def operand(rows, cols, fmt, block, seed, spread=6):
    """An FP8 matrix of random bytes (no NaN, no infinity) and scales around 1, between bytes that must not be used."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    m, ebuf, sbuf = empty_matrix(rows, cols, fmt, block, fill=0x7F)         # 0x7F: NaN in both formats
    b = torch.randint(0, 256, (rows, cols), generator=g, device=DEV, dtype=torch.uint8)
    bad = (b & 127 == 127) if fmt == zc.FMT_FP8_E4M3 else (b & 127 >= 0x7C)
    m.elems.copy_(torch.where(bad, b & 0x8F, b))
    sbuf.fill_(255)                                                          # NaN where no scale byte belongs
    m.scales.copy_(torch.randint(127 - spread, 128 + spread, m.scales.shape, generator=g, device=DEV, dtype=torch.uint8))
    return m


def exact(a, b):
    x = ref.values(a.elems.cpu().numpy(), a.scales.cpu().numpy(), a.format, a.block_rows)
    y = ref.values(b.elems.cpu().numpy(), b.scales.cpu().numpy(), b.format, b.block_rows)
    return x @ y.T, np.abs(x) @ np.abs(y).T


def allowed(d, magnitude, k, dtype):
    """Products of two FP8 values are exact in FP32; each of at most k additions loses at most a unit in the last place
    (2^-23, were it cut off) of a partial sum, which is at most `magnitude`; then one rounding to the output's type, half a
    step of it, or half of its smallest step."""
    return k * 2.0 ** -23 * magnitude + torch.finfo(dtype).eps / 2 * (np.abs(d) + k * 2.0 ** -23 * magnitude) + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2


def near(d, want, magnitude, k):
    """Whether d is the rounding of `want` within `allowed`.  FP16 ends at 65504 with a step of 32: from 65520 on, half a step
    above it, to nearest is infinity."""
    got = d.double().cpu().numpy()
    bound = allowed(want, magnitude, k, d.dtype)
    ok = np.abs(got - want) <= bound
    if d.dtype == torch.float16:
        ok |= np.isinf(got) & (np.sign(got) == np.sign(want)) & (np.abs(want) + k * 2.0 ** -23 * magnitude >= 65520)
    return bool(ok.all())


SIZES = [(1, 1, 1), (1, 128, 128), (2, 129, 130), (128, 128, 512), (129, 255, 640), (77, 1001, 2050), (256, 256, 4096), (300, 520, 1153), (1, 4096, 4096), (64, 640, 2048), (513, 129, 31),
         (1024, 1300, 700), (2100, 2500, 390)]


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("fmt_a,fmt_b", [(2, 2), (5, 2), (2, 5), (5, 5)])
def test_matmul(m, n, k, fmt_a, fmt_b):
    block_a, block_b = ((1, 128), (1, 1), (128, 1), (128, 128))[(m + fmt_a) % 4]
    a, b = operand(m, k, fmt_a, block_a, 1), operand(n, k, fmt_b, block_b, 2)
    for x in (a, b):                                                         # smaller values, so that FP16 holds most results
        x.elems &= 0xBF if x.format == 2 else 0xBB
    want, magnitude = exact(a, b)
    for name, dtype in REAL.items():
        for pitch in (n, n + 1, -(-n // 16) * 16):
            d, buf = strided(m, n, pitch, dtype, 7)
            zc.fp8_matmul(a, b, d)
            assert near(d, want, magnitude, k), (name, pitch)
            assert untouched(buf, d, 7)
            first = d.clone()
            zc.fp8_matmul(a, b, d)
            assert torch.equal(first.view(torch.uint8), d.view(torch.uint8))     # the same every time
    assert zc.fp8_status() == zc.OK


@pytest.mark.parametrize("dtype", list(REAL.values()))
@pytest.mark.parametrize("m,n,k", [(5, 300, 260), (200, 131, 128), (700, 900, 384)])
def test_matmul_accumulates(m, n, k, dtype):
    a, b = operand(m, k, 2, 1, 3), operand(n, k, 2, 128, 4)
    a.elems &= 0xBF
    b.elems &= 0xBF
    want, magnitude = exact(a, b)
    d = torch.randn((m, n), device=DEV).to(dtype)
    before = d.double().cpu().numpy()
    zc.fp8_matmul(a, b, d, accumulate=True)
    # one more addition than the product alone
    assert near(d, want + before, magnitude + np.abs(before), k + 1)


def test_matmul_extreme_scales_and_special_values():
    # scales at both ends of their range cancel; a NaN scale, a NaN element and infinities spread to their rows alone
    a, b = operand(130, 256, 5, 1, 5), operand(140, 256, 5, 1, 6)
    for x in (a, b):
        x.elems &= 0xBB
    a.scales.fill_(0)
    b.scales.fill_(254)
    want, magnitude = exact(a, b)
    d = torch.empty((130, 140), device=DEV)
    zc.fp8_matmul(a, b, d)
    assert near(d, want, magnitude, 256)
    a.scales[3, 1] = 255
    a.elems[7, 200] = 0x7C
    b.elems[9, 200] = 0x7F
    zc.fp8_matmul(a, b, d)
    got = d.cpu()
    assert torch.isnan(got[3]).all() and torch.isnan(got[:, 9]).all()
    assert not torch.isfinite(got[7]).any()                                 # infinity, or NaN where it met a zero
    keep = [i for i in range(130) if i not in (3, 7)], [j for j in range(140) if j != 9]
    sub = got[keep[0]][:, keep[1]].double().numpy()
    assert (np.abs(sub - want[np.ix_(*keep)]) <= allowed(want, magnitude, 256, torch.float32)[np.ix_(*keep)]).all()


def test_matmul_of_positive_values_does_not_drift():
    # all products of one sign: a sum that cuts off instead of rounding would fall short by k / 32 units
    m, n, k = 128, 128, 14336
    a, b = operand(m, k, 2, 1, 8, spread=0), operand(n, k, 2, 1, 9, spread=0)
    for x in (a, b):
        x.elems &= 0x3F
    want, magnitude = exact(a, b)
    d = torch.empty((m, n), device=DEV)
    zc.fp8_matmul(a, b, d)
    assert near(d, want, magnitude, k)


def test_matmul_without_columns_and_rows():
    a = zc.Fp8Matrix(torch.empty((3, 0), dtype=torch.uint8, device=DEV), torch.empty((3, 0), dtype=torch.uint8, device=DEV), 2, 1)
    b = zc.Fp8Matrix(torch.empty((5, 0), dtype=torch.uint8, device=DEV), torch.empty((5, 0), dtype=torch.uint8, device=DEV), 2, 1)
    d = torch.ones((3, 5), device=DEV)
    zc.fp8_matmul(a, b, d, accumulate=True)
    assert bool((d == 1).all())
    zc.fp8_matmul(a, b, d)
    assert bool((d == 0).all())
    empty = zc.fp8_empty(0, 128)
    zc.fp8_matmul(empty, operand(5, 128, 2, 1, 1), torch.empty((0, 5), device=DEV))
    zc.fp8_quantize(torch.empty((0, 128), device=DEV), empty)
    assert zc.fp8_status() == zc.OK


def test_streams_and_graphs():
    # two products on two streams at once, and a captured quantise + product replayed on new inputs
    a, b = operand(200, 1024, 2, 1, 11), operand(384, 1024, 2, 128, 12)
    want = torch.empty((200, 384), device=DEV)
    zc.fp8_matmul(a, b, want)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.empty_like(want) for _ in streams]
    for _ in range(8):
        for s, d in zip(streams, outs):
            zc.fp8_matmul(a, b, d, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(d, want) for d in outs)

    x = torch.randn((200, 1024), device=DEV, dtype=torch.bfloat16)
    q = zc.fp8_empty(200, 1024)
    out = torch.empty((200, 384), device=DEV, dtype=torch.bfloat16)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        zc.fp8_quantize(x, q)
        zc.fp8_matmul(q, b, out)
    for seed in (1, 2):
        x.copy_(torch.randn((200, 1024), generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(torch.bfloat16))
        g.replay()
        torch.cuda.synchronize()
        q2 = zc.fp8_empty(200, 1024)
        eager = torch.empty_like(out)
        zc.fp8_matmul(zc.fp8_quantize(x, q2), b, eager)
        assert torch.equal(out.view(torch.uint8), eager.view(torch.uint8))


def test_kernels_that_start_early_wait_for_those_before():
    # every kernel here may be on the GPU before the one in front of it is done: inputs that change from pass to pass, without a wait
    b = operand(384, 512, 2, 128, 22)
    xs = [torch.randn((129, 512), generator=torch.Generator(device=DEV).manual_seed(i), device=DEV).bfloat16() for i in range(40)]
    wants = []
    for x in xs:
        q, d = zc.fp8_empty(129, 512), torch.empty((129, 384), device=DEV)
        zc.fp8_matmul(zc.fp8_quantize(x, q), b, d)
        torch.cuda.synchronize()
        wants.append(d)
    x, q, d = torch.empty_like(xs[0]), zc.fp8_empty(129, 512), torch.empty((129, 384), device=DEV)
    outs = [torch.empty_like(d) for _ in xs]
    for src, out in zip(xs, outs):
        x.copy_(src)
        zc.fp8_quantize(x, q)
        zc.fp8_matmul(q, b, d)
        out.copy_(d)
    assert all(torch.equal(a, w) for a, w in zip(outs, wants))


def test_offsets_beyond_32_bits():
    rows, cols = 66000, 33000                                                # 2.2e9 elements: FP8 offsets pass 2^31, BF16 ones 2^32
    x = torch.zeros((rows, cols), dtype=torch.bfloat16, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(31)
    tail = torch.randn((300, cols), generator=g, device=DEV).bfloat16()
    x[-300:] = tail
    q = zc.fp8_quantize(x, zc.fp8_empty(rows, cols))
    del x
    elems, scales, _ = ref.quantize(tail.double().cpu().numpy(), zc.FMT_FP8_E4M3, 1)
    assert np.array_equal(q.elems[-300:].cpu().numpy(), elems) and np.array_equal(q.scales[-300:].cpu().numpy(), scales)
    assert not bool(q.elems[:1000].any())
    b = operand(40, cols, 2, 1, 32)
    b.elems &= 0xBF
    d = torch.empty((rows, 40), device=DEV)
    zc.fp8_matmul(q, b, d)
    last = zc.Fp8Matrix(q.elems[-300:], q.scales[-300:], zc.FMT_FP8_E4M3, 1)
    want, magnitude = exact(last, b)
    assert near(d[-300:], want, magnitude, cols) and not bool(d[:-300].any())
    del q, last, d
    # a result of 4.5 GB: the last rows and the first
    a, b = operand(70000, 128, 2, 1, 33), operand(16000, 128, 2, 1, 34)
    for m in (a, b):
        m.elems &= 0xBF
    d = torch.empty((70000, 16000), device=DEV)
    zc.fp8_matmul(a, b, d)
    for part in (slice(0, 50), slice(69950, 70000)):
        want, magnitude = exact(zc.Fp8Matrix(a.elems[part], a.scales[part], a.format, 1), b)
        assert near(d[part], want, magnitude, 128)


def test_a_wait_that_runs_out_is_reported_and_later_calls_work():
    a, b = operand(256, 2048, 2, 1, 13), operand(512, 2048, 2, 128, 14)
    d = torch.empty((256, 512), device=DEV)
    big = operand(4096, 512, 2, 1, 15), operand(4096, 512, 2, 1, 16)
    d_big = torch.empty((4096, 4096), device=DEV)
    try:
        zc.test_set_wait_limit(1000)
        zc.test_stall_decoder(True)                                          # no copies are started
        zc.fp8_matmul(a, b, d)
        zc.fp8_matmul(*big, d_big)
        assert zc.fp8_status() == zc.E_DEVICE_TIMEOUT
    finally:
        zc.test_set_wait_limit(0)
        zc.test_stall_decoder(False)
    assert zc.fp8_status() == zc.OK                                          # read once
    want, magnitude = exact(a, b)
    zc.fp8_matmul(a, b, d)
    assert near(d, want, magnitude, 2048)
    assert zc.fp8_status() == zc.OK


def test_linear_layer_and_its_gradients():
    """Forward product, gradient of the input and of the weights as a training step makes them, against the formulas on the
    quantised operands, and the gradients against differences of the (linear) layer itself."""
    tokens, n, k = 300, 260, 390
    g = torch.Generator(device=DEV).manual_seed(21)
    x, w = (torch.randn(s, generator=g, device=DEV) for s in ((tokens, k), (n, k)))
    dy = torch.randn((tokens, n), generator=g, device=DEV) * 1e-3
    make = lambda r, c, f, b: zc.fp8_empty(r, c, f, b)  # noqa: E731
    qx, qxt = make(tokens, k, 2, 1), make(k, tokens, 2, 1)
    qw, qwt = make(n, k, 2, 128), make(k, n, 2, 128)
    qd, qdt = make(tokens, n, 5, 1), make(n, tokens, 5, 1)
    zc.fp8_quantize(x, qx, qxt)
    zc.fp8_quantize(w, qw, qwt)
    zc.fp8_quantize(dy, qd, qdt)
    y, dx, dw = (torch.empty(s, device=DEV) for s in ((tokens, n), (tokens, k), (n, k)))
    zc.fp8_matmul(qx, qw, y)
    zc.fp8_matmul(qd, qwt, dx)
    zc.fp8_matmul(qdt, qxt, dw)
    for got, a, b, inner in ((y, qx, qw, k), (dx, qd, qwt, n), (dw, qdt, qxt, tokens)):
        want, magnitude = exact(a, b)
        assert near(got, want, magnitude, inner)
    # the transposed weights are the same values: 128 x 128 blocks transpose onto themselves
    vw = ref.values(qw.elems.cpu().numpy(), qw.scales.cpu().numpy(), 2, 128)
    assert np.array_equal(vw.T, ref.values(qwt.elems.cpu().numpy(), qwt.scales.cpu().numpy(), 2, 128))
    # differences: loss = sum(dy * (x w^T)) is linear in x and in w; what separates them from the gradients is the rounding
    # of the two operands to FP8, at most half a step of the value or of the format's smallest value, and the sums' in FP32
    def off(v, m):
        half, least = (2.0 ** -4, 2.0 ** -10) if m.format == 2 else (2.0 ** -3, 2.0 ** -17)
        s = torch.exp2(m.scales.double() - 127).repeat_interleave(m.block_rows, 0)[: v.shape[0]].repeat_interleave(128, 1)[:, : v.shape[1]]
        return half * v.abs() + least * s

    x64, w64, dy64 = (v.double() for v in (x, w, dy))
    v = torch.randn((tokens, k), generator=g, device=DEV, dtype=torch.float64)
    u = torch.randn((n, k), generator=g, device=DEV, dtype=torch.float64)
    loss = lambda p, q: (dy64 * (p @ q.t())).sum()  # noqa: E731
    for grad, step, diff, (l, ml), (r, mr) in ((dx, v, loss(x64 + v, w64) - loss(x64 - v, w64), (dy64, qd), (w64.t().contiguous(), qwt)),
                                               (dw, u, loss(x64, w64 + u) - loss(x64, w64 - u), (dy64.t().contiguous(), qdt), (x64.t().contiguous(), qxt))):
        wide = (l.abs() + off(l, ml)) @ (r.abs() + off(r, mr)).t()
        bound = ((wide - l.abs() @ r.abs().t() + l.shape[1] * 2.0 ** -23 * wide) * step.abs()).sum()
        assert abs((grad.double() * step).sum() - diff / 2) <= bound

"""What the operators on FP8 matrices refuse, before anything reaches a GPU."""
import ctypes as C

import pytest
import torch

from paper_2508_19263_b200 import binding as zc

L = zc._lib


def matrix(rows=256, cols=256, **change):
    d = dict(d_elems=1 << 20, d_scales=1 << 21, rows=rows, cols=cols, ld_elems=-(-cols // 16) * 16, ld_scales=-(-cols // 128), format=2, block_rows=1)
    d.update(change)
    return zc.Fp8MatrixDesc(**d)


def quantize(q, qt=None, real=zc.REAL_F32, d_in=1 << 22, ld=256):
    return L.zc_fp8_quantize(real, d_in, ld, C.addressof(q) if q else None, C.addressof(qt) if qt else None, None)


def matmul(a, b, real=zc.REAL_F32, d_out=1 << 22, ld=256):
    return L.zc_fp8_matmul(C.addressof(a) if a else None, C.addressof(b) if b else None, real, d_out, ld, 0, None)


BAD_MATRIX = [(dict(d_elems=None), zc.E_INVALID_ARG), (dict(d_scales=None), zc.E_INVALID_ARG), (dict(d_elems=(1 << 20) + 8), zc.E_INVALID_ARG),
              (dict(ld_elems=250), zc.E_INVALID_ARG), (dict(ld_elems=240), zc.E_INVALID_ARG), (dict(ld_elems=264), zc.E_INVALID_ARG),
              (dict(ld_scales=1), zc.E_INVALID_ARG), (dict(ld_elems=1 << 40), zc.E_INVALID_ARG), (dict(ld_scales=1 << 40), zc.E_INVALID_ARG),
              (dict(format=1), zc.E_UNSUPPORTED), (dict(format=3), zc.E_UNSUPPORTED), (dict(format=4), zc.E_UNSUPPORTED), (dict(block_rows=0), zc.E_UNSUPPORTED),
              (dict(block_rows=32), zc.E_UNSUPPORTED), (dict(rows=1 << 31), zc.E_TOO_LARGE), (dict(cols=1 << 31, ld_elems=1 << 31, ld_scales=1 << 24), zc.E_TOO_LARGE)]


@pytest.mark.parametrize("change,status", BAD_MATRIX)
def test_matrices(change, status):
    bad, good = matrix(**change), matrix()
    assert quantize(bad) == status and quantize(None, bad) == status and quantize(good, bad) == status
    assert matmul(bad, good) == status and matmul(good, bad) == status


def test_quantize():
    q = matrix(100, 256)
    assert quantize(None) == zc.E_INVALID_ARG
    assert quantize(q, real=3) == zc.E_UNSUPPORTED
    assert quantize(q, d_in=None) == zc.E_INVALID_ARG
    assert quantize(q, d_in=(1 << 22) + 2) == zc.E_INVALID_ARG
    assert quantize(q, real=zc.REAL_BF16, d_in=(1 << 22) + 1) == zc.E_INVALID_ARG
    assert quantize(q, ld=255) == zc.E_INVALID_ARG
    assert quantize(q, ld=1 << 40) == zc.E_INVALID_ARG
    for change in (dict(rows=255), dict(cols=99), dict(format=5), dict(block_rows=128)):
        assert quantize(q, matrix(**{**dict(rows=256, cols=100), **change})) == zc.E_INVALID_ARG
    assert quantize(matrix((1 << 31) - 1, (1 << 31) - 1, ld_elems=1 << 31, ld_scales=1 << 24), ld=1 << 31) == zc.E_TOO_LARGE
    assert quantize(matrix(0, 256)) == zc.OK and quantize(matrix(256, 0)) == zc.OK      # nothing to do


def test_matmul():
    a, b = matrix(64), matrix(256)
    assert matmul(None, b) == zc.E_INVALID_ARG and matmul(a, None) == zc.E_INVALID_ARG
    assert matmul(a, b, real=3) == zc.E_UNSUPPORTED
    assert matmul(a, matrix(256, 255)) == zc.E_INVALID_ARG
    assert matmul(a, b, d_out=None) == zc.E_INVALID_ARG
    assert matmul(a, b, d_out=(1 << 22) + 2) == zc.E_INVALID_ARG
    assert matmul(a, b, real=zc.REAL_F16, d_out=(1 << 22) + 1) == zc.E_INVALID_ARG
    assert matmul(a, b, ld=255) == zc.E_INVALID_ARG
    assert matmul(a, b, ld=1 << 40) == zc.E_INVALID_ARG
    assert matmul(matrix(0), b) == zc.OK and matmul(a, matrix(0)) == zc.OK


def test_binding():
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)  # noqa: E731
    with pytest.raises(ValueError):
        zc.Fp8Matrix(u8(4, 256), u8(4, 1))                           # too few scale bytes
    with pytest.raises(ValueError):
        zc.Fp8Matrix(u8(4, 256), u8(4, 2), block_rows=128)
    with pytest.raises(ValueError):
        zc.Fp8Matrix(u8(4, 256).to(torch.int8), u8(4, 2))
    with pytest.raises(ValueError):
        zc.Fp8Matrix(u8(256, 4).t(), u8(4, 2))                       # rows not contiguous
    m = zc.Fp8Matrix(u8(4, 256), u8(4, 2))
    assert m.shape == (4, 256) and m.desc.ld_elems == 256 and m.desc.ld_scales == 2
    one = zc.Fp8Matrix(u8(1, 250), u8(1, 2))
    assert one.desc.ld_elems == 256                                  # a single row has no pitch of its own
    with pytest.raises(ValueError):
        zc.fp8_quantize(torch.zeros((4, 255)), m)                    # shapes
    with pytest.raises(TypeError):
        zc.fp8_quantize(torch.zeros((4, 256), dtype=torch.float64), m)
    with pytest.raises(ValueError):
        zc.fp8_quantize(torch.zeros((256, 4)).t(), m)                # columns contiguous
    with pytest.raises(ValueError):
        zc.fp8_matmul(m, m, torch.zeros((4, 5)))


def layer(**change):
    d = dict(d_router=1 << 20, d_gate_up=1 << 21, d_gate_up_scales=1 << 22, d_down=1 << 23, d_down_scales=1 << 24, ld_router=256, ld_gate_up=256, ld_down=128, n_experts=8, top_k=2,
             hidden=256, inter=128, format=2, real_type=zc.REAL_BF16)
    d.update(change)
    return zc.Fp8MoeLayerDesc(**d)


def moe(desc, tokens=4, x=1 << 25, ld_x=256, y=1 << 26, ld_y=256, ids=None, weights=None, ws=1 << 27, ws_bytes=1 << 30):
    return L.zc_fp8_moe(C.addressof(desc) if desc else None, tokens, x, ld_x, y, ld_y, ids, weights, ws, ws_bytes, None)


@pytest.mark.parametrize("change,status", [
    (dict(d_router=None), zc.E_INVALID_ARG), (dict(d_gate_up=None), zc.E_INVALID_ARG), (dict(d_gate_up_scales=None), zc.E_INVALID_ARG), (dict(d_down=None), zc.E_INVALID_ARG),
    (dict(d_down_scales=None), zc.E_INVALID_ARG), (dict(d_router=(1 << 20) + 8), zc.E_INVALID_ARG), (dict(d_gate_up=(1 << 21) + 8), zc.E_INVALID_ARG), (dict(d_down=(1 << 23) + 1), zc.E_INVALID_ARG),
    (dict(ld_router=248), zc.E_INVALID_ARG), (dict(ld_router=260), zc.E_INVALID_ARG), (dict(ld_gate_up=240), zc.E_INVALID_ARG), (dict(ld_gate_up=264), zc.E_INVALID_ARG),
    (dict(ld_down=112), zc.E_INVALID_ARG), (dict(ld_down=136), zc.E_INVALID_ARG), (dict(ld_down=1 << 33), zc.E_INVALID_ARG),
    (dict(n_experts=0), zc.E_INVALID_ARG), (dict(top_k=0), zc.E_INVALID_ARG), (dict(top_k=9), zc.E_INVALID_ARG), (dict(hidden=0), zc.E_INVALID_ARG), (dict(inter=0), zc.E_INVALID_ARG),
    (dict(n_experts=257), zc.E_TOO_LARGE), (dict(n_experts=64, top_k=17), zc.E_TOO_LARGE), (dict(hidden=65537, ld_router=65544, ld_gate_up=65552), zc.E_TOO_LARGE), (dict(inter=65537, ld_down=65552), zc.E_TOO_LARGE),
    (dict(format=3), zc.E_UNSUPPORTED), (dict(real_type=zc.REAL_F32), zc.E_UNSUPPORTED)])
def test_moe_layers(change, status):
    bad = layer(**change)
    assert moe(bad) == status
    assert L.zc_fp8_moe_workspace_bytes(C.addressof(bad), 4) == 0


def test_moe_arguments():
    good = layer()
    need = L.zc_fp8_moe_workspace_bytes(C.addressof(good), 4)
    assert need > 0 and L.zc_fp8_moe_workspace_bytes(None, 4) == 0 and L.zc_fp8_moe_workspace_bytes(C.addressof(good), 65) == 0
    assert moe(None) == zc.E_INVALID_ARG
    assert moe(good, tokens=65) == zc.E_TOO_LARGE
    assert moe(good, tokens=0) == zc.OK
    assert moe(good, ws_bytes=need - 1) == zc.E_BUFFER_TOO_SMALL
    for change in (dict(x=None), dict(x=(1 << 25) + 8), dict(ld_x=248), dict(ld_x=260), dict(ld_x=1 << 33), dict(y=None), dict(y=(1 << 26) + 1), dict(ld_y=255), dict(ld_y=1 << 33),
                   dict(ids=2), dict(weights=2), dict(ws=None), dict(ws=(1 << 27) + 128)):
        assert moe(good, **change) == zc.E_INVALID_ARG, change


def test_moe_binding():
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)  # noqa: E731
    make = lambda router=torch.zeros((4, 64), dtype=torch.bfloat16), gu=u8(4, 2, 32, 64), gs=u8(4, 2, 1, 1), d=u8(4, 64, 32), ds=u8(4, 1, 1): zc.Fp8MoeLayer(router, gu, gs, d, ds, 2)  # noqa: E731
    m = make()
    assert (m.experts, m.hidden, m.inter) == (4, 64, 32) and m.workspace_bytes(3) > 0
    for bad in (dict(router=torch.zeros((5, 64), dtype=torch.bfloat16)), dict(gu=u8(4, 1, 32, 64)), dict(gs=u8(4, 2, 1, 2)), dict(d=u8(4, 32, 64)), dict(ds=u8(4, 2, 1)),
                dict(gu=u8(4, 2, 32, 64).to(torch.int8)), dict(d=u8(4, 128, 32)[:, ::2]), dict(d=u8(4, 80, 32)[:, :64])):
        if "d" in bad and bad["d"].shape == (4, 64, 32) and bad["d"].stride(1) == 64:
            assert make(**bad).desc.ld_down == 64                    # every other row: one pitch, no gaps
            continue
        with pytest.raises(ValueError):
            make(**bad)
    x = torch.zeros((3, 64), dtype=torch.bfloat16)
    with pytest.raises(TypeError):
        zc.fp8_moe(m, x.half(), x.half(), u8(1))
    with pytest.raises(ValueError):
        zc.fp8_moe(m, x[:, :32], x[:, :32], u8(1))
    with pytest.raises(ValueError):
        zc.fp8_moe(m, x, x.clone(), u8(1), d_ids=torch.zeros((3, 3), dtype=torch.int32))

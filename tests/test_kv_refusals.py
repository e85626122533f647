"""What the operators on a quantised key/value cache refuse, before anything reaches a GPU."""
import ctypes as C

import pytest
import torch

from paper_2508_19263_b200 import binding as zc

L = zc._lib
K = 1 << 20


def cache(**change):
    d = dict(d_k_elems=K, d_k_scales=2 * K, d_v_elems=3 * K, d_v_scales=4 * K, n_pages=10, page_tokens=16, kv_heads=4, head_dim=128, format=3)
    return zc.KvCacheDesc(**{**d, **change})


def batch(**change):
    d = dict(d_page_table=5 * K, d_lens=6 * K, d_first=7 * K, ld_page_table=8, n_rows=5, max_pages=8, n_seqs=3, max_new=1)
    return zc.KvBatchDesc(**{**d, **change})


def tensor(**change):
    return zc.KvTensorDesc(**{**dict(d=8 * K, ld_row=2048, ld_head=128), **change})


def args(**change):
    d = dict(q=tensor(), out=tensor(d=16 * K), d_lse=None, type=zc.REAL_BF16, q_heads=8, scale=0.1, causal=1, window=0)
    return zc.KvAttentionArgs(**{**d, **change})


def ref(d):
    return C.addressof(d) if d is not None else None


def append(c=cache(), b=batch(), real=zc.REAL_BF16, k=tensor(), v=tensor(d=9 * K)):
    return L.zc_kv_append(ref(c), ref(b), real, ref(k), ref(v), None)


def read(c=cache(), b=batch(), real=zc.REAL_BF16, k=tensor(), v=tensor(d=9 * K)):
    return L.zc_kv_read(ref(c), ref(b), real, ref(k), ref(v), None)


def need(c=cache(), b=batch(), q_heads=8):
    return L.zc_kv_attention_workspace_bytes(ref(c), ref(b), q_heads)


def attention(c=cache(), b=batch(), a=args(), ws=1 << 28, size=1 << 30):
    return L.zc_kv_attention(ref(c), ref(b), ref(a), ws, size, None)


BAD_CACHE = [(dict(format=1), zc.E_UNSUPPORTED), (dict(format=4), zc.E_UNSUPPORTED), (dict(format=5), zc.E_UNSUPPORTED), (dict(head_dim=32), zc.E_UNSUPPORTED),
             (dict(head_dim=96), zc.E_UNSUPPORTED), (dict(head_dim=256), zc.E_UNSUPPORTED), (dict(page_tokens=8), zc.E_UNSUPPORTED), (dict(page_tokens=48), zc.E_UNSUPPORTED),
             (dict(page_tokens=512), zc.E_UNSUPPORTED), (dict(kv_heads=0), zc.E_INVALID_ARG), (dict(kv_heads=1025), zc.E_TOO_LARGE),
             (dict(n_pages=1 << 25), zc.E_TOO_LARGE), (dict(n_pages=1 << 62), zc.E_TOO_LARGE), (dict(d_k_elems=None), zc.E_INVALID_ARG), (dict(d_v_scales=None), zc.E_INVALID_ARG),
             (dict(d_k_scales=2 * K + 8), zc.E_INVALID_ARG), (dict(d_v_elems=3 * K + 4), zc.E_INVALID_ARG)]
BAD_BATCH = [(dict(n_seqs=4097), zc.E_TOO_LARGE), (dict(n_rows=1 << 31), zc.E_TOO_LARGE), (dict(max_pages=1 << 27), zc.E_TOO_LARGE), (dict(d_lens=None), zc.E_INVALID_ARG),
             (dict(d_first=None), zc.E_INVALID_ARG), (dict(d_page_table=None), zc.E_INVALID_ARG), (dict(ld_page_table=7), zc.E_INVALID_ARG),
             (dict(ld_page_table=1 << 40), zc.E_INVALID_ARG), (dict(d_lens=6 * K + 2), zc.E_INVALID_ARG), (dict(d_page_table=5 * K + 1), zc.E_INVALID_ARG)]
BAD_TENSOR = [(dict(d=None), zc.E_INVALID_ARG), (dict(d=8 * K + 1), zc.E_INVALID_ARG), (dict(ld_row=100), zc.E_INVALID_ARG), (dict(ld_head=64), zc.E_INVALID_ARG),
              (dict(ld_row=1 << 39), zc.E_INVALID_ARG), (dict(ld_head=1 << 39), zc.E_INVALID_ARG)]
BAD_ARGS = [(dict(type=zc.REAL_F32), zc.E_UNSUPPORTED), (dict(type=9), zc.E_UNSUPPORTED), (dict(q_heads=0), zc.E_INVALID_ARG), (dict(q_heads=6), zc.E_INVALID_ARG),
            (dict(q_heads=4 * 257), zc.E_TOO_LARGE), (dict(scale=float("nan")), zc.E_INVALID_ARG), (dict(scale=float("inf")), zc.E_INVALID_ARG),
            (dict(causal=2), zc.E_INVALID_ARG), (dict(causal=0, window=5), zc.E_INVALID_ARG), (dict(d_lse=2), zc.E_INVALID_ARG)]


@pytest.mark.parametrize("change,status", BAD_CACHE)
def test_caches(change, status):
    assert append(cache(**change)) == status and read(cache(**change)) == status and attention(cache(**change)) == status
    assert need(cache(**change)) == 0


@pytest.mark.parametrize("change,status", BAD_BATCH)
def test_batches(change, status):
    assert append(b=batch(**change)) == status and read(b=batch(**change)) == status and attention(b=batch(**change)) == status
    assert need(b=batch(**change)) == 0


@pytest.mark.parametrize("change,status", BAD_TENSOR)
def test_tensors(change, status):
    bad = tensor(**change)
    assert append(k=bad) == status and append(v=bad) == status and read(k=bad) == status and read(v=bad) == status
    assert attention(a=args(q=bad)) == status and attention(a=args(out=bad)) == status


@pytest.mark.parametrize("change,status", BAD_ARGS)
def test_arguments(change, status):
    assert attention(a=args(**change)) == status


def test_missing():
    assert append(None) == read(None) == attention(None) == zc.E_INVALID_ARG
    assert append(b=None) == read(b=None) == attention(b=None) == zc.E_INVALID_ARG
    assert append(k=None) == append(v=None) == read(k=None, v=None) == attention(a=None) == zc.E_INVALID_ARG
    assert append(real=7) == read(real=-1) == zc.E_UNSUPPORTED
    assert attention(ws=None) == attention(ws=(1 << 28) + 16) == zc.E_INVALID_ARG
    assert need() > 0 and attention(size=need() - 1) == zc.E_BUFFER_TOO_SMALL
    for q_heads in (0, 6, 4 * 257):
        assert need(q_heads=q_heads) == 0


def test_nothing_to_do():
    for b in (batch(n_seqs=0), batch(n_rows=0), batch(n_seqs=0, d_lens=None, d_first=None, d_page_table=None)):
        assert append(b=b) == read(b=b) == attention(b=b) == zc.OK


def host(fmt=zc.FMT_FP4_E2M1):
    return zc.kv_empty(4, 2, 16, 64, fmt, device="cpu")


def small_batch(max_new=1):
    i = lambda *v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    return zc.KvBatch(i(0, 1).reshape(1, 2), i(20), i(0, 1), max_new)


def test_binding():
    c, b = host(), small_batch()
    x = torch.zeros((1, 2, 64), dtype=torch.bfloat16)
    ws = torch.zeros(1 << 10, dtype=torch.uint8)
    with pytest.raises(ValueError, match="host memory"):
        zc.kv_append(c, b, x, x)
    with pytest.raises(ValueError, match="host memory"):
        zc.kv_attention(c, b, x, torch.empty_like(x), ws)
    with pytest.raises(TypeError):
        zc.kv_append(c, b, x.double(), x.double())
    with pytest.raises(ValueError):
        zc.kv_append(c, b, x, x.float())
    with pytest.raises(ValueError):
        zc.kv_append(c, b, x, None)
    with pytest.raises(ValueError):
        zc.kv_read(c, b, None, None)
    with pytest.raises(ValueError):
        zc.kv_read(c, b, x[:, :1], None)
    with pytest.raises(ValueError):
        zc.kv_read(c, b, torch.zeros((1, 2, 128), dtype=torch.bfloat16)[..., ::2], None)
    with pytest.raises(TypeError):
        zc.kv_attention(c, b, x, x.half(), ws)
    with pytest.raises(ValueError):
        zc.kv_attention(c, b, x, x[:, :1], ws)
    with pytest.raises(ValueError):
        zc.kv_attention(c, b, x, torch.empty_like(x), ws, d_lse=torch.empty((1, 3)))
    with pytest.raises(ValueError):
        zc.KvCache(c.k_elems, c.k_scales, c.v_elems, c.v_scales, zc.FMT_BF16)
    with pytest.raises(ValueError):
        zc.KvCache(c.k_elems, c.k_scales, c.v_elems[:2], c.v_scales)
    with pytest.raises(ValueError):
        zc.KvCache(c.k_elems, c.k_scales[..., :1], c.v_elems, c.v_scales)
    with pytest.raises(ValueError):
        zc.KvCache(c.k_elems.transpose(1, 2), c.k_scales, c.v_elems, c.v_scales)
    with pytest.raises(ValueError):
        zc.KvBatch(b.page_table, b.lens.long(), b.first)
    with pytest.raises(ValueError):
        zc.KvBatch(b.page_table, b.lens, b.lens)
    with pytest.raises(ValueError):
        zc.KvBatch(b.page_table, b.lens, b.first, -1)

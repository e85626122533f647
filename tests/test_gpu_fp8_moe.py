"""zc_fp8_moe against its definition in 64 bits, and the FP8 operators together with the codec."""
import numpy as np
import pytest
import torch

import fp8_reference as ref
from paper_2508_19263_b200 import binding as zc
from paper_2508_19263_b200 import workloads as wl

pytestmark = pytest.mark.gpu
DEV = "cuda"
REAL = {"bf16": torch.bfloat16, "f16": torch.float16}


def blocks(n):
    return -(-n // 128)


def largest_of_128(v):
    """The largest magnitude of every 128 columns, at each of them."""
    wide = np.zeros((v.shape[0], blocks(v.shape[1]) * 128))
    wide[:, : v.shape[1]] = np.abs(v)
    return np.repeat(wide.reshape(v.shape[0], -1, 128).max(axis=2), 128, 1)[:, : v.shape[1]]


class Layer:
    """A layer of random weights; bytes behind the rows' ends are NaN, so that a use of them shows."""

    def __init__(self, experts, top_k, hidden, inter, fmt, dtype, seed, router=None):
        g = torch.Generator(device=DEV).manual_seed(seed)
        pad = lambda n, m: -(-n // m) * m  # noqa: E731
        rand = lambda *s: torch.randint(0, 256, s, generator=g, device=DEV, dtype=torch.uint8)  # noqa: E731

        def weights(*shape):
            buf = torch.full((*shape[:-1], pad(shape[-1], 16)), 0x7F, dtype=torch.uint8, device=DEV)
            view = buf[..., : shape[-1]]
            view.copy_(rand(*shape) & (0xBF if fmt == zc.FMT_FP8_E4M3 else 0xBB))          # up to 1.875 (1.75)
            return view

        self.fmt, self.top_k = fmt, top_k
        self.gate_up, self.down = weights(experts, 2, inter, hidden), weights(experts, hidden, inter)
        self.gate_up_scales = torch.randint(118, 126, (experts, 2, blocks(inter), blocks(hidden)), generator=g, device=DEV, dtype=torch.uint8)
        self.down_scales = torch.randint(118, 126, (experts, blocks(hidden), blocks(inter)), generator=g, device=DEV, dtype=torch.uint8)
        wide = torch.full((experts, pad(hidden, 8)), float("nan"), dtype=dtype, device=DEV)
        self.router = wide[:, :hidden]
        self.router.copy_(torch.randn((experts, hidden), generator=g, device=DEV) / hidden ** 0.5 if router is None else router)
        self.layer = zc.Fp8MoeLayer(self.router, self.gate_up, self.gate_up_scales, self.down, self.down_scales, top_k, fmt)

    def tokens(self, n, seed):
        g = torch.Generator(device=DEV).manual_seed(seed)
        hidden = self.layer.hidden
        wide = torch.full((n, -(-hidden // 8) * 8 + 8), float("nan"), dtype=self.layer.dtype, device=DEV)
        x = wide[:, :hidden]
        x.copy_(torch.randn((n, hidden), generator=g, device=DEV))
        return x

    def run(self, x, **more):
        n = x.shape[0]
        wide = torch.full((n + 2, self.layer.hidden + 3), 7.0, dtype=x.dtype, device=DEV)
        y = wide[:n, : self.layer.hidden]
        ids = torch.full((n, self.top_k), -1, dtype=torch.int32, device=DEV)
        weights = torch.full((n, self.top_k), -1.0, device=DEV)
        ws = torch.full((self.layer.workspace_bytes(n),), 0xCD, dtype=torch.uint8, device=DEV)
        zc.fp8_moe(self.layer, x, y, ws, d_ids=ids, d_weights=weights, **more)
        assert bool((wide[n:] == 7).all()) and bool((wide[:, self.layer.hidden:] == 7).all())      # nothing outside
        return y, ids, weights

    def exact(self, x):
        """(y, ids, weights, bound on y's error before its rounding)."""
        x = x.double().cpu().numpy()
        logits = x @ self.router.double().cpu().numpy().T
        ids = np.argsort(-logits, axis=1, kind="stable")[:, : self.top_k]
        top = np.take_along_axis(logits, ids, 1)
        p = np.exp(top - top[:, :1])
        p /= p.sum(axis=1, keepdims=True)
        y, bound = np.zeros(x.shape), np.zeros(x.shape)
        hidden, inter = self.layer.hidden, self.layer.inter
        for e in np.unique(ids):
            tok, slot = np.nonzero(ids == e)
            m = [ref.values(t.cpu().numpy(), s.cpu().numpy(), self.fmt, 128) for t, s in
                 ((self.gate_up[e, 0], self.gate_up_scales[e, 0]), (self.gate_up[e, 1], self.gate_up_scales[e, 1]), (self.down[e], self.down_scales[e]))]
            gate, up = x[tok] @ m[0].T, x[tok] @ m[1].T
            # FP32 sums of exact products: at most a unit in the last place of a partial sum for each of the additions
            unit = 2.0 ** -23
            # x in three pieces of E4M3, each rounding what the ones before leave: exact for 8 and 11 bits but where a piece is
            # below the smallest normal value; its step there is 2^-9 2^-8 2^s, and the largest of 128 columns is above 224 2^s
            d_x = 2.0 ** -25 * largest_of_128(x[tok])
            d_gate, d_up = ((hidden + 8) * unit * (np.abs(x[tok]) @ np.abs(w).T) + d_x @ np.abs(w).T for w in m[:2])
            silu = gate / (1 + np.exp(-gate))
            w = p[tok, slot][:, None]
            h = w * silu * up
            # |silu'| <= 1.1; a few roundings in FP32; three (FP16: four) pieces of E4M3 leave 2^-4 of the value each, or half of
            # the last one's smallest step, and what the first leaves is held in FP16, 2^-12 of 2^-4; the router's parts of 128 columns are FP32 sums, so a logit is off by 128 units of
            # its part and p by twice that relative
            pieces = 4 if self.layer.dtype == torch.float16 else 3
            d_logit = 128 * unit * (np.abs(x[tok]) @ np.abs(self.router[e].double().cpu().numpy())).max()
            d_h = w * (1.1 * d_gate * np.abs(up) + np.abs(silu) * d_up + 1.1 * d_gate * d_up) + np.abs(h) * (16 * unit + 2 * d_logit)
            d_h = d_h + (2.0 ** (-4 * pieces) + 2.0 ** -16) * (np.abs(h) + d_h) + 2.0 ** (-13 - 4 * pieces) * largest_of_128(np.abs(h) + d_h)
            y[tok] += h @ m[2].T
            bound[tok] += d_h @ np.abs(m[2]).T + (inter + 16 + self.top_k) * unit * ((np.abs(h) + d_h) @ np.abs(m[2]).T)
        return y, ids, p, bound


def check(L, x, got):
    y, ids, weights = got
    want, want_ids, p, bound = L.exact(x)
    assert np.array_equal(ids.cpu().numpy(), want_ids)
    # a logit is off by at most 128 units of its largest part's magnitude, p by twice that and the roundings of exp and the division
    d_logit = 128 * 2.0 ** -23 * (np.abs(x.double().cpu().numpy()) @ np.abs(L.router.double().cpu().numpy()).T).max()
    assert (np.abs(weights.double().cpu().numpy() - p) <= p * (2 * d_logit + 32 * 2.0 ** -24)).all()
    t = torch.finfo(y.dtype)
    # one rounding of y: half a step of the value, or of the smallest value
    assert (np.abs(y.double().cpu().numpy() - want) <= bound + t.eps / 2 * (np.abs(want) + bound) + t.smallest_normal * t.eps / 2).all()


SHAPES = [(1, 1, 1, 1, 1), (1, 4, 2, 64, 8), (3, 8, 3, 130, 72), (8, 16, 4, 256, 128), (9, 5, 5, 513, 257), (17, 40, 8, 384, 130), (33, 4, 2, 512, 200), (64, 3, 3, 200, 520), (64, 130, 6, 264, 136),
          (64, 256, 16, 128, 64), (2, 256, 16, 1100, 40), (5, 2, 1, 2048, 1024)]


@pytest.mark.parametrize("tokens,experts,top_k,hidden,inter", SHAPES)
@pytest.mark.parametrize("fmt", [zc.FMT_FP8_E4M3, zc.FMT_FP8_E5M2])
@pytest.mark.parametrize("real", list(REAL))
def test_moe(tokens, experts, top_k, hidden, inter, fmt, real):
    L = Layer(experts, top_k, hidden, inter, fmt, REAL[real], tokens + hidden)
    x = L.tokens(tokens, 3)
    got = L.run(x)
    check(L, x, got)
    again = L.run(x)
    assert all(torch.equal(a, b) for a, b in zip(got, again))                # the same every time


@pytest.mark.parametrize("real", list(REAL))
@pytest.mark.parametrize("experts", [70, 8])
def test_ties_go_to_the_lowest_index_and_all_tokens_may_choose_one_expert(real, experts):
    # all logits equal: experts 0 .. top_k - 1 for every token; the lists are as long as they get, in passes of 16 and of 32 tokens
    L = Layer(experts, 4, 256, 128, zc.FMT_FP8_E4M3, REAL[real], 5, router=torch.zeros((experts, 256), device=DEV))
    x = L.tokens(64, 1)
    y, ids, weights = L.run(x)
    assert ids.cpu().tolist() == [[0, 1, 2, 3]] * 64 and bool((weights == 0.25).all())
    check(L, x, (y, ids, weights))


def test_a_token_of_nan_and_infinities_stays_by_itself():
    L = Layer(16, 2, 300, 200, zc.FMT_FP8_E4M3, torch.bfloat16, 6)
    x = L.tokens(12, 2)
    clean = L.run(x)
    bad = L.tokens(12, 2)
    bad[3, 17] = float("nan")
    bad[7] = float("inf")
    y, ids, weights = L.run(bad)
    keep = [i for i in range(12) if i not in (3, 7)]
    assert ids[3].cpu().tolist() == [0, 1]                                   # NaN logits: the lowest value, ties to the lowest index
    assert bool(torch.isnan(y[3]).all()) and not bool(torch.isfinite(y[7]).any())
    assert bool(((ids >= 0) & (ids < 16)).all())
    want, want_ids, p, bound = L.exact(bad[keep])
    assert np.array_equal(ids[keep].cpu().numpy(), want_ids)
    assert torch.equal(ids[keep], clean[1][keep])
    assert (np.abs(y[keep].double().cpu().numpy() - want) <= bound + 2.0 ** -8 * (np.abs(want) + bound) + 2.0 ** -134).all()


def test_a_token_whose_buffer_ends_with_it():
    # one token of an odd width, no pitch behind it; what follows in the allocation is NaN
    L = Layer(4, 2, 513, 64, zc.FMT_FP8_E4M3, torch.bfloat16, 10)
    buf = torch.full((1024,), float("nan"), dtype=torch.bfloat16, device=DEV)
    x = buf[:513].view(1, 513)
    x.copy_(L.tokens(1, 6))
    check(L, x, L.run(x))


def test_graph_streams_and_shared_weights():
    L = Layer(32, 4, 512, 256, zc.FMT_FP8_E4M3, torch.bfloat16, 7)
    xs = [L.tokens(n, n) for n in (1, 64)]
    wants = [L.run(x)[0] for x in xs]
    # two streams at once, workspaces of their own
    streams = [torch.cuda.Stream() for _ in xs]
    outs = [torch.empty_like(w) for w in wants]
    ws = [torch.empty(L.layer.workspace_bytes(x.shape[0]), dtype=torch.uint8, device=DEV) for x in xs]
    torch.cuda.synchronize()
    for _ in range(10):
        for x, y, w, s in zip(xs, outs, ws, streams):
            zc.fp8_moe(L.layer, x, y, w, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, wants))
    # two captured graphs that share a workspace, replayed one after the other, on new tokens
    shared = torch.empty(L.layer.workspace_bytes(64), dtype=torch.uint8, device=DEV)
    graphs = []
    for x, y in zip(xs, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            for _ in range(2):
                zc.fp8_moe(L.layer, x, y, shared)
        graphs.append(g)
    for seed in (11, 12):
        for x in xs:
            x.copy_(L.tokens(x.shape[0], seed))
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(y, L.run(x)[0]) for x, y in zip(xs, outs))


def test_a_wait_that_runs_out_is_reported_and_later_calls_work():
    L = Layer(8, 2, 512, 256, zc.FMT_FP8_E4M3, torch.bfloat16, 8)
    x = L.tokens(20, 5)
    want = L.run(x)
    try:
        zc.test_set_wait_limit(1000)
        zc.test_stall_decoder(True)                                          # no copies are started
        L.run(x)
        assert zc.fp8_status() == zc.E_DEVICE_TIMEOUT
    finally:
        zc.test_set_wait_limit(0)
        zc.test_stall_decoder(False)
    assert zc.fp8_status() == zc.OK                                          # read once
    assert all(torch.equal(a, b) for a, b in zip(L.run(x), want))
    assert zc.fp8_status() == zc.OK


def _through_the_codec(fmt, t):
    """A byte tensor compressed and decompressed; a new tensor."""
    flat = t.contiguous().reshape(-1)
    p = zc.plan(fmt, flat.numel(), 4096)
    # element bytes start on a 16-byte boundary as everything the allocator returns
    cb = zc.build_codebook(p, zc.histogram(p, flat).cpu().numpy(), zc.POLICY_AUTO)
    comp = torch.empty(p.max_compressed_bytes, dtype=torch.uint8, device=DEV)
    ws = torch.empty(p.workspace_bytes, dtype=torch.uint8, device=DEV)
    n = zc.compress(p, cb, flat, comp, ws)
    back = torch.empty_like(flat)
    zc.decompress(p, comp, n, back, ws)
    assert zc.device_status(p, ws) == zc.OK
    assert torch.equal(back, flat)
    return back.reshape(t.shape), n


def test_quantise_store_load_multiply():
    """What a user does: a BF16 checkpoint tensor is quantised, stored as an FP8 container and a container of scale bytes,
    loaded again and multiplied by; the products of what was stored and of what was loaded are the same."""
    spec = wl.TensorSpec("w", (640, 1024), 0.02, 3)
    raw, _, _ = wl.make_weight(spec, zc.FMT_BF16, DEV)
    w = raw.view(torch.bfloat16).reshape(spec.shape)
    q = zc.fp8_quantize(w, zc.fp8_empty(*spec.shape, block_rows=128))
    elems, n_elems = _through_the_codec(zc.FMT_FP8_E4M3, q.elems)
    scales, _ = _through_the_codec(zc.FMT_SCALE_U8, q.scales)
    assert n_elems < elems.numel()                                           # Gaussian weights in FP8 compress
    loaded = zc.Fp8Matrix(elems, scales, zc.FMT_FP8_E4M3, 128)
    x = torch.randn((33, 1024), device=DEV, dtype=torch.bfloat16)
    qx = zc.fp8_quantize(x, zc.fp8_empty(33, 1024))
    y, want = (torch.empty((33, 640), device=DEV, dtype=torch.bfloat16) for _ in range(2))
    zc.fp8_matmul(qx, q, want)
    zc.fp8_matmul(qx, loaded, y)
    assert torch.equal(y, want) and bool(torch.isfinite(y).all())


def test_experts_from_containers():
    """Experts that are kept compressed, decoded and used: what comes out is what the uncompressed layer gives."""
    L = Layer(8, 2, 512, 256, zc.FMT_FP8_E4M3, torch.bfloat16, 9)
    x = L.tokens(7, 4)
    want = L.run(x)
    for name, fmt in (("gate_up", zc.FMT_FP8_E4M3), ("down", zc.FMT_FP8_E4M3), ("gate_up_scales", zc.FMT_SCALE_U8), ("down_scales", zc.FMT_SCALE_U8)):
        setattr(L, name, _through_the_codec(fmt, getattr(L, name))[0])
    L.layer = zc.Fp8MoeLayer(L.router, L.gate_up, L.gate_up_scales, L.down, L.down_scales, 2)
    assert all(torch.equal(a, b) for a, b in zip(L.run(x), want))

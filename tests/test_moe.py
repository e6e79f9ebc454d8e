"""Mixture-of-experts layers of a few tokens: the router and the experts against plain 64-bit forms."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2604_21026_amd import nvq
from tests import np_mx

DEV = "cuda:0"
gpu = pytest.mark.gpu


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def f64(t):
    return t.double().cpu().numpy()


# ---- refusals (no device is touched) ----
def test_route_refusals_before_any_launch():
    L, a = nvq.lib(), 0x1000
    big = 1 << 20

    def call(x=a, r=a, M=4, E=64, K=128, k=4, renorm=1, ids=a, w=a, ws=a, bytes_=big):
        return L.nvq_moe_route(x, r, M, E, K, k, renorm, ids, w, ws, bytes_, None)

    assert call(x=None) == 1 and call(r=None) == 1 and call(ids=None) == 1 and call(w=None) == 1 and call(renorm=2) == 1
    assert call(M=0) == 2 and call(M=33) == 2 and call(E=0) == 2 and call(E=513) == 2 and call(K=100) == 2
    assert call(K=0) == 2 and call(K=65568) == 2 and call(k=0) == 2 and call(k=17) == 2 and call(E=3, k=4) == 2
    assert call(x=a + 8) == 3 and call(r=a + 2) == 3 and call(ids=a + 2) == 3 and call(w=a + 1) == 3
    need = L.nvq_moe_route_workspace_bytes(4, 64)
    assert need > 256 and call(ws=None) == 6 and call(ws=a + 16) == 6 and call(bytes_=need - 1) == 6
    assert L.nvq_moe_route_workspace_bytes(33, 64) == 0 and L.nvq_moe_route_workspace_bytes(4, 0) == 0
    assert L.nvq_moe_route_workspace_bytes(4, 513) == 0


def test_experts_refusals_before_any_launch():
    L, a = nvq.lib(), 0x1000
    big = 1 << 24

    def call(e=None, x=a, ids=a, w=a, M=4, k=2, y=a, dt=1, ws=a, bytes_=big, **kw):
        v = dict(gate_up=a, gate_up_scales=a, down=a, down_scales=a, format=1, E=8, K=64, F=96)
        v.update(kw)
        s = nvq.ExpertsStruct(*v.values())
        return L.nvq_moe_experts(C.addressof(s), x, ids, w, M, k, y, dt, ws, bytes_, None)

    s = nvq.ExpertsStruct(a, a, a, a, 1, 8, 64, 96)
    need = L.nvq_moe_workspace_bytes(C.addressof(s), 4, 2)
    assert need >= 4 * 2 * 96 * 2 and call(bytes_=need - 1) == 6 and call(ws=None) == 6 and call(ws=a + 16) == 6
    assert L.nvq_moe_experts(None, a, a, a, 4, 2, a, 1, a, big, None) == 1
    for f in ("gate_up", "gate_up_scales", "down", "down_scales"):
        assert call(**{f: None}) == 1
    assert call(x=None) == 1 and call(ids=None) == 1 and call(w=None) == 1 and call(y=None) == 1 and call(dt=2) == 1
    assert call(format=2) == 1
    assert call(E=0) == 2 and call(E=513) == 2 and call(K=80) == 2 and call(K=0) == 2 and call(F=48) == 2 and call(F=0) == 2
    assert call(K=65568) == 2 and call(F=65568) == 2 and call(M=0) == 2 and call(M=33) == 2 and call(k=0) == 2 and call(k=17) == 2
    assert call(gate_up=a + 8) == 3 and call(down=a + 4) == 3 and call(x=a + 2) == 3 and call(ids=a + 1) == 3
    assert call(w=a + 2) == 3 and call(y=a + 1) == 3 and call(y=a + 2, dt=0) == 3
    assert call(format=0, gate_up_scales=a + 1) == 3 and call(format=0, down_scales=a + 1) == 3
    s.F = 95
    assert L.nvq_moe_workspace_bytes(C.addressof(s), 4, 2) == 0 and L.nvq_moe_workspace_bytes(None, 4, 2) == 0


def test_the_binding_refuses_experts_that_do_not_fit():
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)
    with pytest.raises(ValueError):
        nvq.Experts(u8(2, 128, 32), u8(2, 128, 2), u8(2, 64, 32), u8(2, 64, 2))  # host tensors
    with pytest.raises(ValueError):
        nvq.Experts(u8(2, 128, 32), torch.zeros((2, 128, 2)), u8(2, 64, 32), u8(2, 64, 2))
    with pytest.raises(ValueError):
        nvq.Experts(u8(2, 128, 32), u8(2, 128, 2), u8(2, 64, 16), u8(2, 64, 2))
    with pytest.raises(ValueError):
        nvq.Experts(u8(2, 96, 32), u8(2, 96, 2), u8(2, 64, 24), u8(2, 64, 1))  # F = 48


# ---- the router ----
ROUTE = [(1, 1, 32, 1), (1, 8, 64, 8), (3, 5, 96, 2), (1, 64, 2048, 8), (16, 17, 160, 16), (17, 64, 512, 1),
         (32, 128, 4096, 4), (8, 64, 320, 8), (9, 65, 320, 9), (13, 300, 256, 16), (31, 511, 64, 7), (6, 129, 4128, 5), (5, 200, 1440, 6), (32, 256, 288, 8), (9, 512, 2048, 16), (2, 300, 65536, 3)]


@gpu
@pytest.mark.parametrize("M,E,K,k", ROUTE)
@pytest.mark.parametrize("renorm", [True, False])
def test_route_of_exact_logits_with_ties(M, E, K, k, renorm):
    """Small whole numbers: every sum exact, many logits equal."""
    rng = np.random.default_rng(M + E + K)
    x = rng.integers(-1, 2, (M, K)) * (rng.random((M, K)) < 24 / K)
    r = rng.integers(-1, 2, (E, K)).astype(np.float64)
    logits = (x @ r.T).astype(np.float64)
    ids, w = nvq.moe_route(dev(x).bfloat16(), dev(r).bfloat16(), k, renorm)
    want = np_mx.best(logits, k)
    assert np.array_equal(ids.cpu().numpy(), want)
    p = np.exp(logits - logits.max(1, keepdims=True))
    chosen = np.take_along_axis(p, want, 1)
    p = chosen / (chosen if renorm else p).sum(1, keepdims=True)
    # exp to two units (of 2^-24) beside its rounded argument (|difference| < 64 units), sums of up to E / 64 + 22 terms
    assert (np.abs(f64(w) - p) <= p * (2 * (4 + 64 + E / 64 + 22) * np_mx.EPS32)).all()


@gpu
@pytest.mark.parametrize("M,E,K,k", [(1, 64, 2048, 8), (32, 128, 4096, 4), (7, 40, 1440, 3), (20, 256, 8192, 8)])
def test_route_of_ordinary_logits(M, E, K, k):
    g = torch.Generator().manual_seed(K + E)
    x, r = torch.randn((M, K), generator=g).bfloat16(), (torch.randn((E, K), generator=g) * 0.02).bfloat16()
    logits = f64(x) @ f64(r).T
    d = 2 * (K + 40) * np_mx.EPS32 * (np.abs(f64(x)) @ np.abs(f64(r)).T).max(1)  # two logits' error
    ws = nvq.moe_route_workspace(32, 256, DEV)
    for _ in range(3):  # the workspace is as it was after each call
        ids, w = nvq.moe_route(x.to(DEV), r.to(DEV), k, workspace=ws)
        got = ids.cpu().numpy()
        assert int(ws[:256].sum()) == 0
        l = np.take_along_axis(logits, got, 1)
        assert (l[:, :-1] >= l[:, 1:] - d[:, None]).all()  # in order
        rest = logits.copy()
        np.put_along_axis(rest, got, -np.inf, 1)
        assert (l[:, -1] >= rest.max(1) - d).all()  # and the best
        assert all(len(set(row)) == k for row in got.tolist())
        p = np.exp(l - l.max(1, keepdims=True))
        p /= p.sum(1, keepdims=True)
        assert (np.abs(f64(w) - p) <= p * (2 * d[:, None] + 200 * np_mx.EPS32)).all()


@gpu
def test_route_gives_distinct_ids_in_range_whatever_the_inputs():
    g = torch.Generator().manual_seed(4)
    x, r = torch.randn((5, 64), generator=g).bfloat16(), torch.randn((20, 64), generator=g).bfloat16()
    x[0], x[1, 3], x[2, 0] = 0.0, float("nan"), float("inf")
    r[7, 5] = float("nan")
    ids, w = nvq.moe_route(x.to(DEV), r.to(DEV), 6)
    got = ids.cpu().numpy()
    assert (got >= 0).all() and (got < 20).all() and all(len(set(row)) == 6 for row in got.tolist())
    assert got[0].tolist() == [0, 1, 2, 3, 4, 5] and got[1].tolist() == [0, 1, 2, 3, 4, 5]
    assert not (got[3:] == 7).any() and bool(torch.isfinite(w[3:]).all())


# ---- the experts ----
def make(fmt, E, K, F, seed):
    """Experts of N(0, 0.02) weights in their format: the handle, and what they stand for in 64 bits."""
    g = torch.Generator().manual_seed(seed)
    parts, values = [], []
    for rows, cols in ((2 * F, K), (K, F)):
        w = (torch.randn((E * rows, cols), generator=g) * 0.02).to(DEV)
        q, s = nvq.pack_int4(w) if fmt == "int4" else nvq.quant_mxfp4(w)
        parts += [q.view(E, rows, cols // 2), s.view(E, rows, cols // 32)]
        f = np_mx.dequant_int4 if fmt == "int4" else np_mx.dequant
        sc = s.cpu().numpy().view(np.uint16) if fmt == "int4" else s.cpu().numpy()
        values.append(f(q.cpu().numpy(), sc).reshape(E, rows, cols))
    return nvq.Experts(*parts), values


def choose(rng, M, E, k):
    ids = np.stack([rng.permutation(E)[:k] if k <= E else rng.integers(0, E, k) for _ in range(M)]).astype(np.int32)
    w = rng.random((M, k)).astype(np.float32) + 0.05
    return ids, w / w.sum(1, keepdims=True)


def check(y, x, values, ids, w):
    want, tol = np_mx.experts(f64(x), *values, ids, w.astype(np.float64))
    if y.dtype == torch.bfloat16:
        tol = tol + np_mx.EPS16 * (np.abs(want) + tol)
    err = np.abs(f64(y) - want)
    assert (err <= tol).all(), (err.max(), (err / np.maximum(tol, 1e-300)).max())


EXPERTS = [(1, 1, 1, 32, 32), (1, 2, 2, 64, 96), (1, 64, 8, 512, 256), (2, 4, 3, 160, 64), (5, 40, 3, 1440, 224),
           (16, 8, 2, 256, 128), (17, 3, 2, 128, 416), (32, 2, 1, 96, 32), (32, 16, 4, 512, 512), (32, 1, 1, 288, 64),
           (7, 300, 4, 64, 32), (32, 20, 16, 128, 160), (3, 2, 5, 64, 64),
           # the second launch: tiles of 64 outputs, several workgroups to a tile, experts in slices
           (16, 64, 4, 4096, 32), (32, 16, 8, 4096, 288), (32, 8, 5, 4128, 288), (29, 2, 2, 160, 800), (32, 64, 2, 4096, 96), (9, 6, 6, 4160, 1056), (4, 70, 16, 2048, 160),
           # a few tokens by dot products: one block to a lane and two, in both launches, lanes without
           (1, 8, 2, 4096, 1792), (7, 40, 3, 1440, 992), (4, 8, 2, 2080, 1056), (2, 64, 8, 1056, 2048), (3, 16, 2, 768, 2048), (1, 1, 1, 96, 2048),
           (8, 64, 5, 160, 448), (8, 64, 8, 160, 416), (4, 16, 4, 96, 512), (3, 8, 2, 4096, 1056), (1, 20, 16, 32, 1024), (4, 4, 1, 64, 16384), (1, 8, 2, 4128, 1792),
           # the first one with the activations in registers: a short last wave, 128 inputs to a lane-row in all
           (7, 8, 4, 2080, 4096), (3, 3, 3, 4096, 11008)]


@gpu
@pytest.mark.parametrize("M,E,k,K,F", EXPERTS)
@pytest.mark.parametrize("fmt", ["int4", "mxfp4"])
def test_experts_match_the_plain_form(M, E, k, K, F, fmt):
    rng = np.random.default_rng(M * E + K)
    ex, values = make(fmt, E, K, F, K + F)
    ids, w = choose(rng, M, E, k)
    x = torch.randn((M, K), generator=torch.Generator().manual_seed(M)).bfloat16().to(DEV)
    first = None
    for dtype in (torch.float32, torch.bfloat16):
        y = nvq.moe_experts(ex, x, dev(ids), dev(w), out_dtype=dtype)
        check(y, x, values, ids, w)
        first = y if first is None else first
    assert torch.equal(first.bfloat16(), y)
    assert torch.equal(first, nvq.moe_experts(ex, x, dev(ids), dev(w), out_dtype=torch.float32))


@gpu
@pytest.mark.parametrize("fmt", ["int4", "mxfp4"])
def test_many_tokens_of_one_expert_of_many_rows(fmt):
    """Two tiles of tokens past the same weights, the second one of two tokens; an expert without any."""
    rng = np.random.default_rng(2)
    ex, values = make(fmt, 4, 2144, 8192, 5)
    ids = np.array([[0]] * 18 + [[3], [2], [-1], [3]], np.int32)[rng.permutation(22)]
    w = rng.random(ids.shape).astype(np.float32)
    x = torch.randn((22, 2144), generator=torch.Generator().manual_seed(2)).bfloat16().to(DEV)
    y = nvq.moe_experts(ex, x, dev(ids), dev(w), out_dtype=torch.float32)
    check(y, x, values, ids, w)
    for _ in range(3):
        assert torch.equal(y, nvq.moe_experts(ex, x, dev(ids), dev(w), out_dtype=torch.float32))


@gpu
@pytest.mark.parametrize("fmt", ["int4", "mxfp4"])
@pytest.mark.parametrize("M,E,k", [(6, 10, 3), (20, 4, 4), (1, 30, 4)])
def test_unused_slots_padding_and_an_expert_twice(fmt, M, E, k):
    rng = np.random.default_rng(M)
    ex, values = make(fmt, E, 96, 64, 7)
    ids, w = choose(rng, M, E, k)
    x = torch.randn((M, 96), generator=torch.Generator().manual_seed(M)).bfloat16().to(DEV)
    ids[0, 1] = ids[0, 0]                     # twice
    ids[M // 2, 0], ids[M - 1, 2] = -1, E     # unused slots
    if M > 2:
        ids[2], ids[M - 2] = -5, 2 ** 30      # padding
    y = nvq.moe_experts(ex, x, dev(ids), dev(w), out_dtype=torch.float32)
    check(y, x, values, ids, w)
    if M > 2:
        assert not y[2].any() and not y[M - 2].any()
    none = nvq.moe_experts(ex, x, dev(np.full_like(ids, -1)), dev(w))
    assert not none.any()


@gpu
@pytest.mark.parametrize("fmt", ["int4", "mxfp4"])
@pytest.mark.parametrize("M,E,k,K,F", [(1, 20, 6, 96, 352), (3, 20, 6, 96, 352), (2, 24, 8, 2144, 1056), (7, 70, 6, 160, 384)])
def test_few_tokens_with_unused_slots_and_whatever_the_workspace_holds(fmt, M, E, k, K, F):
    """Slots out of range, an expert twice, a token without any; a workspace of NaN, and no number in an expert that is not chosen."""
    rng = np.random.default_rng(M + k)
    ex, values = make(fmt, E, K, F, 11)
    ids = np.stack([1 + rng.permutation(E - 1)[:k] for _ in range(M)]).astype(np.int32)
    w = rng.random((M, k)).astype(np.float32)
    ids[0, 1], ids[0, 3], ids[0, 4], ids[M - 1, k - 1] = -1, ids[0, 0], E, 2 ** 31 - 1
    w[0, 1], w[0, 4] = np.nan, np.inf
    if M > 2:
        ids[1] = -7
    for s in (ex.keep[1], ex.keep[3]):
        s[0] = 0x7e00 if fmt == "int4" else 255
    x = torch.randn((M, K), generator=torch.Generator().manual_seed(M)).bfloat16().to(DEV)
    ws = ex.workspace(M, k)
    ws.fill_(255)
    y = nvq.moe_experts(ex, x, dev(ids), dev(w), out_dtype=torch.float32, workspace=ws)
    check(y, x, values, ids, np.nan_to_num(w, posinf=0.0))
    if M > 2:
        assert not y[1].any()
    assert torch.equal(y, nvq.moe_experts(ex, x, dev(ids), dev(w), out_dtype=torch.float32, workspace=ws))
    one = nvq.moe_experts(ex, x[:1].contiguous(), dev(ids[:1]), dev(w[:1]), out_dtype=torch.float32)
    check(one, x[:1], values, ids[:1], np.nan_to_num(w[:1], posinf=0.0))


@gpu
@pytest.mark.parametrize("fmt", ["int4", "mxfp4"])
@pytest.mark.parametrize("M,E,k", [(30, 9, 3), (32, 4, 11), (32, 7, 16)])
def test_an_expert_in_several_slots_of_tokens_anywhere_in_the_list(fmt, M, E, k):
    """Slots next to each other and apart, tokens whose slots lie on both sides of a multiple of 64 pairs, all of them equal."""
    rng = np.random.default_rng(k)
    ex, values = make(fmt, E, 96, 64, 9)
    ids = rng.integers(-1, E, (M, k)).astype(np.int32)
    ids[64 // k] = ids[128 // k if 128 // k < M else 0] = [E - 1] * k
    ids[64 // k - 1] = [(i % 2) for i in range(k)]
    w = rng.random((M, k)).astype(np.float32)
    x = torch.randn((M, 96), generator=torch.Generator().manual_seed(M)).bfloat16().to(DEV)
    y = nvq.moe_experts(ex, x, dev(ids), dev(w), out_dtype=torch.float32)
    check(y, x, values, ids, w)


@gpu
@pytest.mark.parametrize("fmt", ["int4", "mxfp4"])
@pytest.mark.parametrize("M", [5, 21])
def test_other_tokens_and_other_experts_do_not_reach_a_token(fmt, M):
    """NaN and infinite inputs of other tokens, weights without a number in experts that a token did not choose."""
    rng = np.random.default_rng(M)
    E, K, F = 6, 160, 96
    ex, _ = make(fmt, E, K, F, 3)
    ids, w = choose(rng, M, E, 2)
    ids[1:][ids[1:] == 4] = 5
    ids[0] = [4, 2]
    x = torch.randn((M, K), generator=torch.Generator().manual_seed(M)).bfloat16().to(DEV)
    clean = nvq.moe_experts(ex, x, dev(ids), dev(w))
    bad = x.clone()
    bad[0], bad[3, 7] = float("nan"), float("inf")
    up, down = ex.keep[1], ex.keep[3]
    up[4, 3], down[4, 5] = (0x7e00, 0x7c00) if fmt == "int4" else (255, 255)
    y = nvq.moe_experts(ex, bad, dev(ids), dev(w))
    others = [m for m in range(M) if m not in (0, 3)]
    assert torch.equal(y[others], clean[others])
    assert bool(torch.isnan(y[0]).any())


@gpu
def test_many_experts_beyond_the_32_bit_offsets():
    """Codes of more than 4 GiB: the last experts are read where they are."""
    E, K, F = 512, 4096, 2080
    rng = np.random.default_rng(1)
    gu = torch.zeros((E, 2 * F, K // 2), dtype=torch.uint8, device=DEV)
    gs = torch.full((E, 2 * F, K // 32), 110, dtype=torch.uint8, device=DEV)
    dn = torch.zeros((E, K, F // 2), dtype=torch.uint8, device=DEV)
    ds = torch.full((E, K, F // 32), 122, dtype=torch.uint8, device=DEV)
    assert gu.numel() > 2 ** 32
    values = [np.zeros((2, 2 * F, K)), np.zeros((2, K, F))]
    for i, e in enumerate((3, E - 1)):
        for j, (q, s) in enumerate(((gu, gs), (dn, ds))):
            c = rng.integers(0, 256, tuple(q.shape[1:]), dtype=np.uint8)
            q[e] = dev(c)
            values[j][i] = np_mx.dequant(c, s[e].cpu().numpy())
    ex = nvq.Experts(gu, gs, dn, ds)
    x = torch.randn((2, K), generator=torch.Generator().manual_seed(1)).bfloat16().to(DEV)
    ids, w = np.array([[E - 1, 3], [3, E - 1]], np.int32), np.array([[0.75, 0.25], [0.5, 0.5]], np.float32)
    y = nvq.moe_experts(ex, x, dev(ids), dev(w), out_dtype=torch.float32)
    check(y, x, values, np.where(ids == 3, 0, 1), w)


@gpu
def test_the_layer_as_a_program_runs_it():
    """Weights quantised, tokens routed, experts, residual sum and norm, and the next layer's microscaled product: eager,
    on a side stream, and captured and replayed with other inputs, every replay against the eager result."""
    E, K, F, k, M = 12, 256, 128, 3, 20
    g = torch.Generator().manual_seed(8)
    ex, values = make("mxfp4", E, K, F, 8)
    router = (torch.randn((E, K), generator=g) * 0.05).bfloat16().to(DEV)
    gamma = torch.ones(K, dtype=torch.bfloat16, device=DEV)
    q, s = nvq.quant_mxfp4((torch.randn((300, K), generator=g) * 0.02).to(DEV))
    x = torch.randn((M, K), generator=g).bfloat16().to(DEV)
    ids, w = torch.empty((M, k), dtype=torch.int32, device=DEV), torch.empty((M, k), device=DEV)
    rws, ews = nvq.moe_route_workspace(M, E, DEV), ex.workspace(M, k)
    y = torch.empty((M, K), dtype=torch.bfloat16, device=DEV)
    c = (torch.empty((M, K // 2), dtype=torch.uint8, device=DEV), torch.empty((M, K // 32), dtype=torch.uint8, device=DEV))
    z = torch.empty((M, 300), device=DEV)

    def layer():
        nvq.moe_route(x, router, k, out=(ids, w), workspace=rws)
        nvq.moe_experts(ex, x, ids, w, out=y, workspace=ews)
        n, _ = nvq.rms_norm(y, gamma, 1e-5, res=x)
        nvq.quant_mxfp4(n, out=c)
        nvq.gemm_mxfp4(q, s, *c, out=z)

    layer()
    check(y, x, values, ids.cpu().numpy(), w.cpu().numpy())
    eager = z.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        z.zero_()
        layer()
    side.synchronize()
    assert torch.equal(z, eager)
    graphs = []
    for _ in range(2):  # two graphs that share workspaces, replayed in turn
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            layer()
        graphs.append(graph)
    for i in range(4):
        x.copy_(torch.randn((M, K), generator=g).bfloat16())
        z.zero_()
        graphs[i % 2].replay()
        torch.cuda.synchronize()
        got = (ids.clone(), w.clone(), y.clone(), z.clone())
        layer()
        for a, b in zip(got, (ids, w, y, z)):
            assert torch.equal(a, b)


@gpu
def test_the_binding_refuses_what_does_not_fit(monkeypatch):
    ex, _ = make("mxfp4", 4, 64, 32, 1)
    x, router = torch.zeros((3, 64), dtype=torch.bfloat16, device=DEV), torch.zeros((4, 64), dtype=torch.bfloat16, device=DEV)
    ids, w = torch.zeros((3, 2), dtype=torch.int32, device=DEV), torch.zeros((3, 2), device=DEV)
    y, ws, rws = torch.empty_like(x), ex.workspace(3, 2), nvq.moe_route_workspace(3, 4, DEV)
    good = nvq.moe_experts(ex, x, ids, w, out=y, workspace=ws)
    for _ in range(2):
        for call in (lambda: nvq.moe_experts(ex, x[:2], ids, w, out=y, workspace=ws),
                     lambda: nvq.moe_experts(ex, x, ids.long(), w, out=y, workspace=ws),
                     lambda: nvq.moe_experts(ex, x, ids, w[:, :1], out=y, workspace=ws),
                     lambda: nvq.moe_experts(ex, x, ids, w, out=y[:2], workspace=ws),
                     lambda: nvq.moe_experts(ex, x.float(), ids, w, out=y, workspace=ws),
                     lambda: nvq.moe_experts(ex, x, ids, w, out=y, workspace=ws[:64]),
                     lambda: nvq.moe_route(x, router[:, :32], 2, out=(ids, w), workspace=rws),
                     lambda: nvq.moe_route(x, router, 2, out=(ids[:2], w), workspace=rws),
                     lambda: nvq.moe_route(x, router, 0), lambda: nvq.moe_route(x, router, 5),
                     lambda: nvq.moe_route(x, router, 2, out=(ids, w), workspace=rws[:256])):
            with pytest.raises((ValueError, nvq.NvqError)):
                call()
        monkeypatch.setattr(nvq, "_calls", None)
    assert not good.any()


@gpu
def test_tensors_of_another_device_than_the_current_one(monkeypatch):
    ex, _ = make("mxfp4", 4, 64, 32, 1)
    x, router = torch.zeros((3, 64), dtype=torch.bfloat16, device=DEV), torch.zeros((4, 64), dtype=torch.bfloat16, device=DEV)
    ids, w = torch.zeros((3, 2), dtype=torch.int32, device=DEV), torch.zeros((3, 2), device=DEV)
    y, ws, rws = torch.empty_like(x), ex.workspace(3, 2), nvq.moe_route_workspace(3, 4, DEV)
    monkeypatch.setattr(ex, "device", torch.device("cuda", 1))
    with pytest.raises(ValueError, match="the experts on"):
        nvq.moe_experts(ex, x, ids, w, out=y, workspace=ws)
    monkeypatch.undo()
    monkeypatch.setattr(nvq, "_calls", None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for call in (lambda: nvq.moe_experts(ex, x, ids, w, out=y, workspace=ws),
                 lambda: nvq.moe_route(x, router, 2, out=(ids, w), workspace=rws)):
        with pytest.raises(ValueError, match="current device"):
            call()


@gpu
@pytest.mark.parametrize("M", [1, 3, 16, 32])
def test_two_streams_at_once_and_replays(M):
    """Two layers on two streams, each with workspaces of its own; then both captured and replayed together."""
    E, K, F, k = 32, 512, 1024, 4
    g = torch.Generator().manual_seed(M)
    sides = []
    for fmt, seed in (("mxfp4", 21), ("int4", 22)):
        ex, values = make(fmt, E, K, F, seed)
        router = (torch.randn((E, K), generator=g) * 0.05).bfloat16().to(DEV)
        q, s = nvq.quant_mxfp4((torch.randn((200, K), generator=g) * 0.02).to(DEV))
        x = torch.randn((M, K), generator=g).bfloat16().to(DEV)
        out = (torch.empty((M, k), dtype=torch.int32, device=DEV), torch.empty((M, k), device=DEV))
        buf = dict(y=torch.empty((M, K), dtype=torch.bfloat16, device=DEV), z=torch.empty((M, 200), device=DEV))
        sides.append((ex, values, router, q, s, x, out, buf, nvq.moe_route_workspace(M, E, DEV), ex.workspace(M, k), torch.cuda.Stream()))

    def layer(side):
        ex, _, router, q, s, x, out, buf, rws, ews, _ = side
        nvq.moe_route(x, router, k, out=out, workspace=rws)
        nvq.moe_experts(ex, x, *out, out=buf["y"], workspace=ews)
        nvq.gemv_mxfp4(q, s, buf["y"], out=buf["z"])

    want = []
    for side in sides:
        layer(side)
        check(side[7]["y"], side[5], side[1], side[6][0].cpu().numpy(), side[6][1].cpu().numpy())
        want.append([t.clone() for t in (*side[6], side[7]["y"], side[7]["z"])])
    torch.cuda.synchronize()
    for _ in range(20):
        for side in sides:
            with torch.cuda.stream(side[10]):
                side[7]["z"].zero_()
                layer(side)
    torch.cuda.synchronize()
    for side, w in zip(sides, want):
        assert all(torch.equal(a, b) for a, b in zip((*side[6], side[7]["y"], side[7]["z"]), w))
    graphs = []
    for side in sides:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            layer(side)
        graphs.append(graph)
    for _ in range(3):
        for side in sides:
            side[5].copy_(torch.randn((M, K), generator=g).bfloat16())
        torch.cuda.synchronize()
        for side, graph in zip(sides, graphs):
            with torch.cuda.stream(side[10]):
                graph.replay()
        torch.cuda.synchronize()
        for side in sides:
            got = [t.clone() for t in (*side[6], side[7]["y"], side[7]["z"])]
            layer(side)
            assert all(torch.equal(a, b) for a, b in zip(got, (*side[6], side[7]["y"], side[7]["z"])))


# ---- logits that are no number ----
@gpu
@pytest.mark.parametrize("M,E,k", [(5, 20, 6), (1, 64, 8), (32, 130, 4), (3, 300, 2)])
def test_route_over_all_experts_leaves_out_logits_that_are_no_number(M, E, k):
    """A NaN logit counts as the smallest: of an expert that was not chosen it does not reach the weights."""
    g = torch.Generator().manual_seed(E)
    x, r = torch.randn((M, 64), generator=g).bfloat16(), torch.randn((E, 64), generator=g).bfloat16()
    r[7, 5] = r[E - 1, 63] = float("nan")
    logits = f64(x) @ f64(r).T
    logits[:, [7, E - 1]] = -np.inf
    d = 2 * (64 + 40) * np_mx.EPS32 * (np.abs(f64(x)) @ np.abs(np.nan_to_num(f64(r))).T).max(1)  # two logits' error
    for renorm in (True, False):
        ids, w = nvq.moe_route(x.to(DEV), r.to(DEV), k, renorm)
        got = ids.cpu().numpy()
        assert not np.isin(got, [7, E - 1]).any() and all(len(set(row)) == k for row in got.tolist())
        top = logits.max(1, keepdims=True)
        p = np.exp(np.take_along_axis(logits, got, 1) - top)
        p /= (p if renorm else np.exp(logits - top)).sum(1, keepdims=True)
        # as test_route_of_exact_logits_with_ties: the exponentials, their arguments (here up to 512 units), the sum
        assert (np.abs(f64(w) - p) <= p * (2 * d[:, None] + 2 * (4 + 512 + E / 64 + 22) * np_mx.EPS32)).all()


@gpu
@pytest.mark.parametrize("renorm", [True, False])
def test_route_of_fewer_numbers_than_choices(renorm):
    """Every number comes before what is none; ids stay distinct and in range."""
    r = torch.zeros((9, 32)).bfloat16()
    r[:, 0] = torch.tensor([float("nan"), 1, float("nan"), 3, float("-inf"), float("nan"), 2, float("nan"), float("nan")])
    x = torch.zeros((2, 32)).bfloat16()
    x[:, 0] = torch.tensor([1.0, 2.0])
    ids, w = nvq.moe_route(x.to(DEV), r.to(DEV), 6, renorm)
    assert ids.cpu().tolist() == [[3, 6, 1, 4, 0, 2]] * 2
    if not renorm:
        p = np.exp(np.array([[3.0, 2, 1, -np.inf], [6.0, 4, 2, -np.inf]]))
        p /= p.sum(1, keepdims=True)
        assert (np.abs(f64(w)[:, :4] - p) <= p * (2 * (4 + 8 + 22) * np_mx.EPS32)).all()
        assert bool(torch.isnan(w[:, 4:]).all())


# ---- operands that are not finite ----
def positive(fmt, rows, K, rng):
    """Weights above zero: their codes, scales and values."""
    q = rng.integers(0, 256, (rows, K // 2), dtype=np.uint8)
    if fmt == "int4":
        q |= 0x88
        q |= ((q & 0x0f) == 8).astype(np.uint8) | ((q & 0xf0) == 0x80).astype(np.uint8) << 4
        s = (2.0 ** -rng.integers(8, 11, (rows, K // 32)).astype(np.float64)).astype(np.float16).view(np.int16)
    else:
        q &= 0x77
        q |= ((q & 0x07) == 0).astype(np.uint8) | ((q & 0x70) == 0).astype(np.uint8) << 4
        s = rng.integers(115, 118, (rows, K // 32), dtype=np.uint8)
    return q, s


NOT_FINITE = [
    # products of tiles: both launches' last pass meets a column again; in the second one also with several
    # workgroups to a tile, wide tiles
    (5, 2, 2, 416, 416), (20, 4, 2, 416, 672), (32, 16, 8, 4096, 288), (9, 6, 6, 4160, 1056), (20, 60, 2, 416, 416),
    # the first launch with the activations in registers, whose last waves' blocks begin before their share
    (5, 3, 3, 2144, 11008), (22, 4, 1, 2144, 8192),
    # dot products
    (1, 8, 4, 160, 544), (2, 20, 4, 2144, 1056)]


@gpu
@pytest.mark.parametrize("M,E,k,K,F", NOT_FINITE)
def test_experts_of_infinite_activations(M, E, k, K, F):
    """Microscaled: an infinite activation beside positive weights makes its token's outputs infinite, wherever it stands."""
    rng = np.random.default_rng(K * F)
    (q, s), (dq, ds) = positive("mxfp4", E * 2 * F, K, rng), positive("mxfp4", E * K, F, rng)
    ex = nvq.Experts(dev(q.reshape(E, 2 * F, K // 2)), dev(s.reshape(E, 2 * F, K // 32)), dev(dq.reshape(E, K, F // 2)),
                     dev(ds.reshape(E, K, F // 32)))
    x = rng.integers(1, 4, (M, K)).astype(np.float32) / 64
    ids = np.stack([rng.permutation(E)[:k] for _ in range(M)]).astype(np.int32)
    w = dev(rng.random((M, k)).astype(np.float32) + 0.1)
    plain = nvq.moe_experts(ex, dev(x).bfloat16(), dev(ids), w, out_dtype=torch.float32)
    assert bool(torch.isfinite(plain).all())
    for at in (slice(None), slice(0, 1), slice(K // 2, K // 2 + 1), slice(K - 140, K - 139), slice(K - 1, K)):
        bad = x.copy()
        bad[M - 1, at] = np.inf
        y = nvq.moe_experts(ex, dev(bad).bfloat16(), dev(ids), w, out_dtype=torch.float32)
        assert bool((y[M - 1] == float("inf")).all()), at
        assert torch.equal(y[:M - 1], plain[:M - 1])


@gpu
@pytest.mark.parametrize("M,E,k,K,F", NOT_FINITE)
@pytest.mark.parametrize("fmt", ["int4", "mxfp4"])
def test_experts_with_weights_beyond_the_range(fmt, M, E, k, K, F):
    """Positive weights and activations: an infinite scale (int4) or values beyond bf16 (scale byte 253) make what they enter
    infinite, not NaN, wherever in a row the block lies (int4: an infinite h makes its outputs NaN); a scale that is no number
    makes it NaN."""
    rng = np.random.default_rng(K + F)
    up, down = positive(fmt, E * 2 * F, K, rng), positive(fmt, E * K, F, rng)
    inf, nan = (0x7c00, 0x7e00) if fmt == "int4" else (253, 255)
    x = dev(rng.integers(1, 4, (M, K)).astype(np.float32) / 64).bfloat16()
    ids = np.stack([rng.permutation(E)[:k] for _ in range(M)]).astype(np.int32)
    w = dev(rng.random((M, k)).astype(np.float32) + 0.1)
    met = np.isin(ids, [E - 1]).any(1)
    ids[~met, 0] = E - 1  # (every token has the last expert)

    def y_of(rows, at, byte, which):
        parts = []
        for (q, s), n, cols, mine in ((up, 2 * F, K, which == "up"), (down, K, F, which == "down")):
            q, s = q.reshape(E, n, cols // 2), s.reshape(E, n, cols // 32)
            if mine:
                q, s = q.copy(), s.copy()
                for r in rows:
                    s[E - 1, r, at] = byte
                    q[E - 1, r, 16 * at:16 * at + 16] = 0xff if fmt == "int4" else 0x77
            parts += [dev(q), dev(s)]
        return nvq.moe_experts(nvq.Experts(*parts), x, dev(ids), w, out_dtype=torch.float32)

    plain = y_of([], 0, 0, "")
    assert bool(torch.isfinite(plain).all())
    for at in {0, K // 64, K // 32 - 5, K // 32 - 1}:
        # one gate row, or one up row: h is infinite there, and so are all outputs
        for row in (5, F - 1, F, 2 * F - 3):
            y = y_of([row], at, inf, "up")
            assert bool((torch.isnan(y) if fmt == "int4" else y == float("inf")).all()), (at, row)
        assert bool(torch.isnan(y_of([F + 1], at, nan, "up")).all())
    for at in {0, F // 64, F // 32 - 1}:
        y = y_of([0, 7, K - 1], at, inf, "down")
        assert bool((y[:, [0, 7, K - 1]] == float("inf")).all()), at
        others = [i for i in range(K) if i not in (0, 7, K - 1)]
        assert torch.equal(y[:, others], plain[:, others])
        assert bool(torch.isnan(y_of([7], at, nan, "down")[:, 7]).all())


# ---- the general lookup of tokens (more than 16 tokens or 64 pairs) where the first launch's grid is pairs, not experts ----
@gpu
@pytest.mark.parametrize("M,E,k,K,F", [(20, 100, 3, 160, 96), (32, 300, 8, 96, 64), (17, 40, 2, 128, 64),
                                       (32, 512, 15, 64, 96), (25, 130, 5, 288, 32), (9, 160, 16, 96, 32)])
@pytest.mark.parametrize("fmt", ["int4", "mxfp4"])
def test_many_tokens_of_more_experts_than_pairs(M, E, k, K, F, fmt):
    """Few experts of many, shared by tokens in different groups of 64 pairs; slots out of range, an expert twice,
    tokens without any; a workspace of NaN."""
    assert M * k < E and (M > 16 or M * k > 64)
    rng = np.random.default_rng(E)
    ex, values = make(fmt, E, K, F, E)
    x = torch.randn((M, K), generator=torch.Generator().manual_seed(M)).bfloat16().to(DEV)
    for pool in (E, 3, 1, 40):
        # (E: hardly any shared; 1: one expert for all, in every slot)
        ids = rng.permutation(E)[:pool][rng.integers(0, pool, (M, k))].astype(np.int32)
        w = rng.random((M, k)).astype(np.float32)
        if pool != 1:
            ids[3, 0], ids[M - 1, k - 1], ids[M // 2, 0] = -1, E, ids[M // 2, k - 1]
            ids[5] = -2
        ws = ex.workspace(M, k)
        ws.fill_(255)
        y = nvq.moe_experts(ex, x, dev(ids), dev(w), out_dtype=torch.float32, workspace=ws)
        check(y, x, values, ids, w)
        assert torch.equal(y, nvq.moe_experts(ex, x, dev(ids), dev(w), out_dtype=torch.float32, workspace=ws))


# few tokens of 65 to 128 experts, nine to sixteen of 129 to 256
@gpu
@pytest.mark.parametrize("M,E,K,k", [(1, 128, 4096, 8), (3, 100, 320, 7), (8, 65, 96, 16), (9, 256, 288, 8),
                                     (16, 140, 2048, 16), (13, 129, 64, 1)])
@pytest.mark.parametrize("renorm", [True, False])
def test_route_of_exact_logits_with_ties_at_other_sizes(M, E, K, k, renorm):
    test_route_of_exact_logits_with_ties(M, E, K, k, renorm)

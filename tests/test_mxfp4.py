"""Microscaled 4-bit floating point: quantisation, its inverse and both products against plain 64-bit forms."""
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


def bits_equal(a, b):
    return np.array_equal(np.asarray(a, np.float64).view(np.uint64), np.asarray(b, np.float64).view(np.uint64))


# ---- the plain form itself, by hand ----
def test_plain_form_on_known_blocks():
    x = np.zeros((1, 64))
    x[0, :12] = [4, -4, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 7.9, -0.0, 0.2500001]
    q, s = np_mx.quant(x)
    assert s.tolist() == [[127, 0]]
    c = np.stack([q & 15, q >> 4], -1).reshape(-1)[:12]
    assert c.tolist() == [6, 14, 0, 2, 2, 4, 4, 6, 6, 7, 8, 1]
    x[0, 32] = np.inf
    assert np_mx.quant(x)[1].tolist() == [[127, 255]]
    assert np.isnan(np_mx.dequant(*np_mx.quant(x))[0, 32:]).all()


# ---- refusals (no device is touched) ----
def test_refusals_before_any_launch():
    L, a = nvq.lib(), 0x1000
    assert L.nvq_quant_mxfp4(None, 0, 4, 64, a, a, None) == 1
    assert L.nvq_quant_mxfp4(a, 2, 4, 64, a, a, None) == 1
    assert L.nvq_quant_mxfp4(a, 0, 4, 48, a, a, None) == 2
    assert L.nvq_quant_mxfp4(a, 0, 0, 64, a, a, None) == 2
    assert L.nvq_quant_mxfp4(a, 0, 1 << 62, 64, a, a, None) == 2
    assert L.nvq_quant_mxfp4(a, 1, (1 << 28) + 1, 64, a, a, None) == 2
    assert L.nvq_dequant_mxfp4(a, a, (1 << 28) + 1, 64, a, None) == 2
    assert L.nvq_gemv_mxfp4(a, a, (1 << 29) + 1, 32, a, 1, a, 0, None) == 2
    assert L.nvq_gemm_mxfp4(a, a, 1 << 30, 64, a, a, 1 << 20, a, 0, None) == 2  # (more results than a launch has lanes)
    assert L.nvq_gemm_mxfp4(a, a, 1 << 30, 512, a, a, 1 << 20, a, 0, None) == 2
    assert L.nvq_quant_mxfp4(a, 0, 4, 65568, a, a, None) == 2
    assert L.nvq_quant_mxfp4(a + 8, 0, 4, 64, a, a, None) == 3
    assert L.nvq_quant_mxfp4(a, 1, 4, 64, a, a + 2, None) == 3
    assert L.nvq_dequant_mxfp4(a, None, 4, 64, a, None) == 1
    assert L.nvq_dequant_mxfp4(a, a, 4, 40, a, None) == 2
    assert L.nvq_dequant_mxfp4(a, a, 4, 64, a + 4, None) == 3
    assert L.nvq_gemv_mxfp4(a, a, 8, 64, a, 1, None, 0, None) == 1
    assert L.nvq_gemv_mxfp4(a, a, 8, 64, a, 1, a, 2, None) == 1
    assert L.nvq_gemv_mxfp4(a, a, 8, 40, a, 1, a, 0, None) == 2
    assert L.nvq_gemv_mxfp4(a, a, 8, 64, a, 33, a, 0, None) == 2
    assert L.nvq_gemv_mxfp4(a, a, 8, 64, a, 0, a, 0, None) == 2
    assert L.nvq_gemv_mxfp4(a, a, 8, 64, a + 2, 1, a, 0, None) == 3
    assert L.nvq_gemv_mxfp4(a, a, 8, 64, a, 1, a + 2, 0, None) == 3
    assert L.nvq_gemm_mxfp4(a, a, 8, 64, a, None, 4, a, 0, None) == 1
    assert L.nvq_gemm_mxfp4(a, a, 8, 64, a, a, 0, a, 0, None) == 2
    assert L.nvq_gemm_mxfp4(a, a, 1 << 40, 64, a, a, 4, a, 0, None) == 2
    assert L.nvq_gemm_mxfp4(a, a, 8, 96 + 8, a, a, 4, a, 0, None) == 2
    assert L.nvq_gemm_mxfp4(a + 4, a, 8, 64, a, a, 4, a, 0, None) == 3
    assert L.nvq_gemm_mxfp4(a, a, 8, 64, a + 8, a, 4, a, 0, None) == 3


def test_the_binding_refuses_host_tensors():
    x = torch.zeros((2, 64))
    q, s = torch.zeros((2, 32), dtype=torch.uint8), torch.zeros((2, 2), dtype=torch.uint8)
    for call in (lambda: nvq.quant_mxfp4(x), lambda: nvq.quant_mxfp4(x, out=(q, s)), lambda: nvq.dequant_mxfp4(q, s),
                 lambda: nvq.gemv_mxfp4(q, s, x.bfloat16()), lambda: nvq.gemm_mxfp4(q, s, q, s)):
        with pytest.raises(ValueError):
            call()


@gpu
def test_the_binding_refuses_what_does_not_fit():
    q, s = torch.zeros((8, 32), dtype=torch.uint8, device=DEV), torch.zeros((8, 2), dtype=torch.uint8, device=DEV)
    x, y = torch.zeros((3, 64), dtype=torch.bfloat16, device=DEV), torch.zeros((3, 8), device=DEV)
    bad = (lambda: nvq.quant_mxfp4(x, out=(q[:2], s)), lambda: nvq.quant_mxfp4(x, out=(q, s[:2])),
           lambda: nvq.quant_mxfp4(x.half()), lambda: nvq.quant_mxfp4(x.t()),
           lambda: nvq.dequant_mxfp4(q, s, out=x), lambda: nvq.dequant_mxfp4(q, s[:4]),
           lambda: nvq.gemv_mxfp4(q, s, x[:, :32]), lambda: nvq.gemv_mxfp4(q, s[:7], x, out=y),
           lambda: nvq.gemv_mxfp4(q, s, x, out=y[:2]), lambda: nvq.gemv_mxfp4(q, s, x, out_dtype=torch.float16),
           lambda: nvq.gemm_mxfp4(q, s, q, s[:4]), lambda: nvq.gemm_mxfp4(q, s, q, s, out=y),
           lambda: nvq.gemm_mxfp4(q, s, q[:, :16], s))
    for call in bad:
        with pytest.raises(ValueError):
            call()
    with pytest.raises(nvq.NvqError):
        nvq.gemv_mxfp4(q, s, torch.zeros((33, 64), dtype=torch.bfloat16, device=DEV))


@gpu
def test_tensors_of_another_device_than_the_current_one(monkeypatch):
    q, s = torch.zeros((8, 32), dtype=torch.uint8, device=DEV), torch.zeros((8, 2), dtype=torch.uint8, device=DEV)
    x, y = torch.zeros((3, 64), dtype=torch.bfloat16, device=DEV), torch.zeros((3, 8), device=DEV)
    nvq.lib()
    monkeypatch.setattr(nvq, "_calls", None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for call in (lambda: nvq.quant_mxfp4(x, out=(q, s)), lambda: nvq.dequant_mxfp4(q[:3], s[:3], out=x),
                 lambda: nvq.gemv_mxfp4(q, s, x, out=y), lambda: nvq.gemm_mxfp4(q, s, q, s, out=y)):
        with pytest.raises(ValueError, match="current device"):
            call()


# ---- quantisation ----
@gpu
@pytest.mark.parametrize("M,K", [(1, 32), (1, 96), (3, 160), (5, 2048), (7, 1440), (33, 4096), (129, 14336), (2, 65536)])
@pytest.mark.parametrize("bf16", [False, True])
def test_quant_bit_exact(M, K, bf16):
    g = torch.Generator().manual_seed(M * K)
    x = torch.randn((M, K), generator=g) * torch.exp2(torch.randint(-20, 20, (M, 1), generator=g).float())
    x = x.bfloat16() if bf16 else x
    q, s = nvq.quant_mxfp4(x.to(DEV))
    rq, rs = np_mx.quant(f64(x))
    assert np.array_equal(s.cpu().numpy(), rs) and np.array_equal(q.cpu().numpy(), rq)
    assert bits_equal(f64(nvq.dequant_mxfp4(q, s)), np_mx.dequant(rq, rs))


@gpu
def test_quant_every_bf16_value():
    """Every bf16 number beside a largest one of 0 to 6 binades above it."""
    bits = np.arange(65536, dtype=np.uint32)
    v = (bits << 16).view(np.float32).astype(np.float64)
    with np.errstate(over="ignore"):
        for up in (0, 1, 2, 3, 4, 6):
            x = np.zeros((65536, 32))
            x[:, 0] = np.abs(v) * 2.0 ** up * (1.25 if up % 2 else 1.0)
            x[:, 17] = v
            t = torch.from_numpy(x).bfloat16()
            q, s = nvq.quant_mxfp4(t.to(DEV))
            rq, rs = np_mx.quant(f64(t))
            assert np.array_equal(s.cpu().numpy(), rs), up
            assert np.array_equal(q.cpu().numpy(), rq), up


@gpu
def test_quant_of_fp32_next_to_ties_and_at_the_ends_of_the_range():
    mids = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0], np.float32)
    near = np.concatenate([mids, np.nextafter(mids, np.float32(0)), np.nextafter(mids, np.float32(9))])
    near = np.concatenate([near, -near]).astype(np.float64)
    rows = []
    for e in list(range(-150, 126, 3)) + [-149, -148, -130, -129, -128, -127, -126, -125, -124, 124, 125]:
        row = np.zeros(64)
        row[:near.size] = near
        row[[31, 62]] = 4.0
        rows.append(row * 2.0 ** e)
    with np.errstate(over="ignore"):
        x = np.array(rows).astype(np.float32)
    x[np.isinf(x)] = 1.0
    q, s = nvq.quant_mxfp4(dev(x))
    rq, rs = np_mx.quant(x.astype(np.float64))
    assert np.array_equal(s.cpu().numpy(), rs)
    assert np.array_equal(q.cpu().numpy(), rq)


@gpu
@pytest.mark.parametrize("bf16", [False, True])
def test_quant_blocks_without_a_number(bf16):
    x = torch.randn((4, 128), generator=torch.Generator().manual_seed(1))
    x[0, 5], x[1, 40], x[2, 127], x[3, 64:96] = float("inf"), float("-inf"), float("nan"), 0.0
    x[3, 70] = -0.0
    x = x.bfloat16() if bf16 else x
    q, s = nvq.quant_mxfp4(x.to(DEV))
    rq, rs = np_mx.quant(f64(x))
    assert (rs == 255).sum() == 3
    assert np.array_equal(s.cpu().numpy(), rs) and np.array_equal(q.cpu().numpy(), rq)
    got, want = f64(nvq.dequant_mxfp4(q, s)), np_mx.dequant(rq, rs)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert bits_equal(np.nan_to_num(got), np.nan_to_num(want))


@gpu
def test_dequant_every_code_at_every_scale():
    q = np.tile(np.arange(256, dtype=np.uint8), 16 * 255).reshape(255, 4096)[:, :256 * 16]
    s = np.repeat(np.arange(255, dtype=np.uint8)[:, None], 256, 1)
    got = nvq.dequant_mxfp4(dev(q), dev(s)).float().cpu().numpy()
    with np.errstate(over="ignore"):
        want = np_mx.dequant(q, s).astype(np.float32)  # (bf16 has fp32's range)
    want[np.abs(want) >= 2.0 ** 128] = np.inf * np.sign(want[np.abs(want) >= 2.0 ** 128])
    assert np.array_equal(got.view(np.uint32), want.view(np.uint32))


@gpu
def test_quant_writes_no_further_than_its_outputs():
    x = torch.randn((3, 96), device=DEV)
    q, s = torch.full((3 * 48 + 64,), 7, dtype=torch.uint8, device=DEV), torch.full((9 + 64,), 7, dtype=torch.uint8, device=DEV)
    nvq.quant_mxfp4(x, out=(q, s))
    rq, rs = np_mx.quant(f64(x))
    assert np.array_equal(q.cpu().numpy()[:144], rq.ravel()) and bool((q[144:] == 7).all())
    assert np.array_equal(s.cpu().numpy()[:9], rs.ravel()) and bool((s[9:] == 7).all())


# ---- products ----
def exact_case(M, N, K, seed, both):
    """Operands whose sums are whole multiples of 2^-9 below 2^15: fp32 holds every partial sum, whatever the order."""
    rng = np.random.default_rng(seed)
    span = 3 if K <= 16384 else 0
    q, s = np_mx.random_mx(rng, N, K, span, 121)
    if both:
        xq, xs = np_mx.random_mx(rng, M, K, 1, 126)
        return q, s, xq, xs, np_mx.dequant(xq, xs)
    x = rng.integers(-3, 4, (M, K)).astype(np.float64)
    return q, s, x, None, x


GEMV = [(1, 1, 32), (1, 16, 64), (2, 17, 96), (1, 33, 128), (3, 70, 160), (16, 31, 224), (17, 15, 416), (32, 48, 2048),
        (5, 257, 1440), (31, 100, 4096), (8, 40, 14336), (1, 5000, 512), (7, 20, 65536), (32, 2100, 288),
        # many rows: activations in registers, in the last wave's place and not at all; K for eight and for four columns
        (1, 65523, 512), (16, 70001, 544), (17, 65537, 1440), (32, 66000, 2048), (3, 65600, 4096), (20, 65541, 3968), (9, 65539, 4128),
        (18, 65540, 480), (2, 9001, 1056), (14, 16001, 608), (24, 9001, 992),
        # ... whose results leave in groups of 256 rows, whole, short and ragged
        (32, 65536, 1024), (29, 131077, 544), (4, 135171, 512), (32, 69632, 4064),
        # one token, a lane to a block: one to two blocks of a row, a wave to it or four, ragged rows and blocks, one turn and several
        (1, 4100, 2048), (1, 9001, 2016), (1, 3, 2080), (1, 2049, 4096), (1, 4097, 4064), (1, 30000, 3968), (1, 5, 4128), (1, 1003, 8192),
        (1, 9002, 6624), (1, 6, 8224), (1, 4099, 14336), (1, 20001, 16384), (1, 50, 16416),
        # 17 to 32 tokens of few inputs and rows
        (20, 99, 2368), (25, 1236, 1760), (17, 956, 384), (32, 4090, 4064),
        # two tokens the same way, and their other ways
        (2, 3, 2080), (2, 2049, 4096), (2, 4097, 4064), (2, 9001, 3968), (2, 1003, 8192), (2, 4099, 14336), (2, 5, 4128), (2, 6, 16384),
        (2, 16400, 2112), (2, 16399, 2112),
        # all activations of a few tokens in LDS: one turn to a workgroup, two, three and more; ragged rows, columns and steps
        (1, 40, 8192), (2, 30, 12288), (3, 33, 8192), (1, 8193, 4128), (1, 40, 2080), (2, 8193, 2112), (3, 24601, 2272), (3, 17000, 4128), (1, 41000, 5152), (3, 33, 9152), (2, 40, 13856), (1, 9000, 28448),
        (1, 8200, 28576), (3, 100, 9184), (2, 30, 2944),
        # a workgroup to each row tile, to two, to four: K that ends inside a turn, and inside a column
        (16, 1003, 4128), (5, 37, 16416), (13, 4090, 6176), (12, 5001, 1568), (6, 8192, 288), (3, 8000, 320), (23, 4001, 4192),
        (19, 3900, 5152), (32, 5009, 2080), (30, 8209, 1312), (11, 8300, 1184), (8, 12003, 2272), (4, 4097, 7200)]


@gpu
@pytest.mark.parametrize("M,N,K", GEMV)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gemv_exact_sums(M, N, K, dtype):
    q, s, x, _, xv = exact_case(M, N, K, M + N + K, False)
    want = xv @ np_mx.dequant(q, s).T
    y = nvq.gemv_mxfp4(dev(q), dev(s), dev(x).bfloat16(), out_dtype=dtype)
    assert bits_equal(f64(y) + 0.0, f64(torch.from_numpy(want).float().to(dtype)) + 0.0)


GEMM = [(1, 1, 32), (1, 64, 128), (2, 17, 96), (64, 64, 256), (65, 63, 160), (77, 130, 416), (300, 257, 2080),
        (128, 513, 4096), (256, 256, 1024), (257, 1, 65536), (3, 1000, 14336), (33, 4100, 224), (1030, 70, 512), (512, 768, 1536),
        # every tile, with ragged edges and stages, some of its slices of K past the end
        (3585, 4001, 544), (4097, 3590, 1824), (2001, 2500, 800), (2304, 2305, 1312), (1000, 3001, 608), (129, 14001, 1056),
        (200, 2700, 992), (65, 8209, 544), (50, 700, 8224), (31, 2050, 8704), (10, 300, 12320)]


@gpu
@pytest.mark.parametrize("M,N,K", GEMM)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gemm_exact_sums(M, N, K, dtype):
    q, s, xq, xs, xv = exact_case(M, N, K, M + N + K, True)
    want = xv @ np_mx.dequant(q, s).T
    assert np.abs(want).max() * 2 ** 9 < 2 ** 24
    y = nvq.gemm_mxfp4(dev(q), dev(s), dev(xq), dev(xs), out_dtype=dtype)
    assert bits_equal(f64(y) + 0.0, f64(torch.from_numpy(want).float().to(dtype)) + 0.0)


@gpu
@pytest.mark.parametrize("M,N,K", [(1, 96, 4096), (20, 200, 1440), (32, 64, 14336)])
def test_products_of_ordinary_values(M, N, K):
    """Weights and activations as they come: fp32 sums of K products, each rounding at most half a step."""
    g = torch.Generator().manual_seed(K + M)
    w = torch.randn((N, K), generator=g) * 0.02
    x = torch.randn((M, K), generator=g).bfloat16()
    x[:, :K // 100] *= 20
    q, s = nvq.quant_mxfp4(w.to(DEV))
    wv = np_mx.dequant(*np_mx.quant(f64(w)))
    size = np.abs(f64(x)) @ np.abs(wv).T
    err = np.abs(f64(nvq.gemv_mxfp4(q, s, x.to(DEV))) - f64(x) @ wv.T)
    assert (err <= (K + 40) * np_mx.EPS32 * size).all()
    xq, xs = nvq.quant_mxfp4(x.to(DEV))
    xv = np_mx.dequant(*np_mx.quant(f64(x)))
    err = np.abs(f64(nvq.gemm_mxfp4(q, s, xq, xs)) - xv @ wv.T)
    assert (err <= (K + 40) * np_mx.EPS32 * (np.abs(xv) @ np.abs(wv).T)).all()


@gpu
@pytest.mark.parametrize("K", [2080, 4160, 8224])
@pytest.mark.parametrize("byte", [0, 1, 2, 60, 200, 252])
def test_one_token_at_the_ends_of_the_scales(byte, K):
    """Weights at an extreme scale, some activations that bring the result back into fp32's range, the rest zero."""
    rng = np.random.default_rng(byte)
    q = rng.integers(0, 256, (20, K // 2), dtype=np.uint8)
    s = np.full((20, K // 32), byte, np.uint8)
    x = rng.integers(-3, 4, (1, K)) * 2.0 ** min(max(127 - byte, -120), 120) * (rng.random((1, K)) < 0.05)
    want = x @ np_mx.dequant(q, s).T
    y = nvq.gemv_mxfp4(dev(q), dev(s), dev(x).bfloat16())
    assert np.array_equal(f64(y), want.astype(np.float32).astype(np.float64))
    # and the other way round: activations below bf16's normal numbers
    x = rng.integers(-3, 4, (1, K)) * 2.0 ** -131
    s[:] = 240
    want = x @ np_mx.dequant(q, s).T
    y = nvq.gemv_mxfp4(dev(q), dev(s), dev(x).bfloat16())
    assert np.array_equal(f64(y), want.astype(np.float32).astype(np.float64))


@gpu
@pytest.mark.parametrize("byte", [0, 1, 60, 200, 252])
def test_products_at_the_ends_of_the_scales(byte):
    """One block of weights at an extreme scale, activations that bring the result back into fp32's range."""
    rng = np.random.default_rng(byte)
    q = rng.integers(0, 256, (20, 16), dtype=np.uint8)
    s = np.full((20, 1), byte, np.uint8)
    back = min(max(127 - byte, -120), 120)
    x = rng.integers(-3, 4, (4, 32)) * 2.0 ** back
    want = x @ np_mx.dequant(q, s).T
    y = nvq.gemv_mxfp4(dev(q), dev(s), dev(x).bfloat16())
    assert np.array_equal(f64(y), want.astype(np.float32).astype(np.float64))
    xq, xs = np_mx.quant(x)
    want = np_mx.dequant(xq, xs) @ np_mx.dequant(q, s).T
    y = nvq.gemm_mxfp4(dev(q), dev(s), dev(xq), dev(xs))
    assert np.array_equal(f64(y), want.astype(np.float32).astype(np.float64))


@gpu
def test_a_block_without_a_number_reaches_its_row_and_token_alone():
    rng = np.random.default_rng(5)
    q, s = np_mx.random_mx(rng, 70, 288)
    xq, xs = np_mx.random_mx(rng, 33, 288)
    s[11, 3] = s[64, 8] = xs[20, 8] = xs[7, 0] = 255
    y = f64(nvq.gemm_mxfp4(dev(q), dev(s), dev(xq), dev(xs)))
    want = np_mx.dequant(xq, xs) @ np_mx.dequant(q, s).T
    assert np.array_equal(np.isnan(y), np.isnan(want))
    x = rng.integers(-3, 4, (33, 288)).astype(np.float64)[:32]
    y = f64(nvq.gemv_mxfp4(dev(q), dev(s), dev(x).bfloat16()))
    assert np.array_equal(np.isnan(y), np.isnan(x @ np_mx.dequant(q, s).T))
    x[20, 200] = np.nan
    y = f64(nvq.gemv_mxfp4(dev(q), dev(s), dev(x).bfloat16()))
    assert np.isnan(y[20]).all() and np.isnan(y[:20]).sum() == 40


@gpu
def test_quantised_nan_reaches_the_products():
    """A block that held an infinity has zero codes: its byte alone makes the results NaN."""
    g = torch.Generator().manual_seed(12)
    w, x = torch.randn((40, 288), generator=g), torch.randn((5, 288), generator=g).bfloat16()
    w[3, 100], w[33, 287] = float("inf"), float("nan")
    q, s = nvq.quant_mxfp4(w.to(DEV))
    y = nvq.gemv_mxfp4(q, s, x.to(DEV))
    z = nvq.gemm_mxfp4(q, s, *nvq.quant_mxfp4(x.to(DEV)))
    for got in (y, z):
        nan = torch.isnan(got).cpu()
        assert nan[:, [3, 33]].all() and int(nan.sum()) == 10


@gpu
def test_beyond_the_32_bit_offsets():
    """More than 4 GiB of values, codes and results: the last ones are where they belong."""
    N, K = 2 ** 21 + 5, 4160
    tail = slice(N - 37, N)
    x = torch.zeros((N, K), dtype=torch.bfloat16, device=DEV)
    ends = torch.randn((42, K), generator=torch.Generator().manual_seed(4)).bfloat16()
    x[tail], x[:5] = ends[5:].to(DEV), ends[:5].to(DEV)
    q, s = nvq.quant_mxfp4(x)
    rq, rs = np_mx.quant(f64(ends))
    assert q.numel() > 2 ** 32
    assert np.array_equal(q[tail].cpu().numpy(), rq[5:]) and np.array_equal(s[tail].cpu().numpy(), rs[5:])
    assert np.array_equal(q[:5].cpu().numpy(), rq[:5]) and not bool(q[5:N - 37].any())
    x.fill_(1)
    nvq.dequant_mxfp4(q, s, out=x)
    v = np_mx.dequant(rq, rs)
    assert bits_equal(f64(x[tail]), v[5:]) and bits_equal(f64(x[:5]), v[:5]) and not bool(x[5:N - 37].any())
    del x
    t = torch.randint(-3, 4, (32, K), generator=torch.Generator().manual_seed(5)).to(DEV).bfloat16()
    tq, ts = nvq.quant_mxfp4(t)
    tv = np_mx.dequant(*np_mx.quant(f64(t)))
    for M in (1, 32):  # (2 GiB of codes beyond the first 4)
        y = nvq.gemv_mxfp4(q, s, t[:M], out_dtype=torch.bfloat16)
        want, size = f64(t[:M]) @ v.T, np.abs(f64(t[:M])) @ np.abs(v).T
        err = np.abs(np.concatenate([f64(y[:, :5]), f64(y[:, tail])], 1) - want)
        assert (err <= (K + 40) * np_mx.EPS32 * size + np_mx.EPS16 * 1.01 * (np.abs(want) + 1e-3 * size)).all()
        assert not bool(y[:, 5:N - 37].any())
        z = nvq.gemm_mxfp4(q, s, tq[:M], ts[:M], out_dtype=torch.bfloat16)
        want, size = tv[:M] @ v.T, np.abs(tv[:M]) @ np.abs(v).T
        err = np.abs(np.concatenate([f64(z[:, :5]), f64(z[:, tail])], 1) - want)
        assert (err <= (K + 40) * np_mx.EPS32 * size + np_mx.EPS16 * 1.01 * (np.abs(want) + 1e-3 * size)).all()
        del y, z
    # as activations: rows of y beyond 4 GiB of results
    wq, ws = nvq.quant_mxfp4(torch.randn((1040, K), generator=torch.Generator().manual_seed(6)).to(DEV))
    wv = np_mx.dequant(wq.cpu().numpy(), ws.cpu().numpy())
    z = nvq.gemm_mxfp4(wq, ws, q, s, out_dtype=torch.bfloat16)
    assert z.numel() * 2 > 2 ** 32
    got = np.concatenate([f64(z[:5]), f64(z[tail])])
    want, size = v @ wv.T, np.abs(v) @ np.abs(wv).T
    assert (np.abs(got - want) <= (K + 40) * np_mx.EPS32 * size + np_mx.EPS16 * 1.01 * (np.abs(want) + 1e-3 * size)).all()
    assert not bool(z[5:N - 37].any())


@gpu
def test_scales_and_outputs_at_any_byte():
    rng = np.random.default_rng(6)
    for N, K, M in ((21, 512, 5), (130, 288, 70)):
        q, s = np_mx.random_mx(rng, N, K)
        xq, xs = np_mx.random_mx(rng, M, K, 1, 126)
        x = rng.integers(-3, 4, (M, K)).astype(np.float64)[:32]
        for off in (1, 2, 3):
            so, xso = (torch.zeros(a.size + off, dtype=torch.uint8, device=DEV) for a in (s, xs))
            so[off:], xso[off:] = dev(s.ravel()), dev(xs.ravel())
            so, xso = so[off:].view(s.shape), xso[off:].view(xs.shape)
            y = torch.zeros(M * N + 8 + off, dtype=torch.bfloat16, device=DEV)[off:]
            nvq.gemm_mxfp4(dev(q), so, dev(xq), xso, out=y)
            want = f64(torch.from_numpy(np_mx.dequant(xq, xs) @ np_mx.dequant(q, s).T).float().bfloat16())
            assert np.array_equal(f64(y[:M * N]).reshape(M, N), want) and not y[M * N:].any()
            y.zero_()
            nvq.gemv_mxfp4(dev(q), so, dev(x).bfloat16(), out=y)
            want = f64(torch.from_numpy(x @ np_mx.dequant(q, s).T).float().bfloat16())
            n = x.shape[0] * N
            assert np.array_equal(f64(y[:n]).reshape(-1, N), want) and not y[n:].any()


@gpu
def test_calls_run_on_the_current_stream_and_replay_in_a_graph():
    g = torch.Generator().manual_seed(3)
    w, x = torch.randn((200, 512), generator=g).to(DEV), torch.randn((40, 512), generator=g).bfloat16().to(DEV)
    out = (torch.empty((40, 256), dtype=torch.uint8, device=DEV), torch.empty((40, 16), dtype=torch.uint8, device=DEV))
    y, z = torch.empty((40, 200), device=DEV), torch.empty((32, 200), device=DEV)
    q, s = nvq.quant_mxfp4(w)
    side = torch.cuda.Stream()

    def once():
        nvq.quant_mxfp4(x, out=out)
        nvq.gemm_mxfp4(q, s, *out, out=y)
        nvq.gemv_mxfp4(q, s, x[:32], out=z)

    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        once()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        once()
    for k in range(3):
        x.copy_(torch.randn((40, 512), generator=g).bfloat16())
        graph.replay()
        torch.cuda.synchronize()
        yy, zz = y.clone(), z.clone()
        y.zero_()
        z.zero_()
        once()
        assert torch.equal(y, yy) and torch.equal(z, zz)
        xv = np_mx.dequant(*np_mx.quant(f64(x)))
        want = xv @ np_mx.dequant(*np_mx.quant(f64(w))).T
        assert np.abs(f64(y) - want).max() <= 1e-4 * np.abs(want).max()


@gpu
def test_calls_without_ctypes_equal_those_through_it(monkeypatch):
    rng = np.random.default_rng(9)
    q, s = [dev(a) for a in np_mx.random_mx(rng, 40, 256)]
    xq, xs = [dev(a) for a in np_mx.random_mx(rng, 5, 256)]
    x = torch.randn((5, 256), device=DEV).bfloat16()

    def all_calls():
        o = [torch.empty((5, 40), device=DEV) for _ in range(2)]
        c = (torch.empty_like(xq), torch.empty_like(xs))
        d = torch.empty((5, 256), dtype=torch.bfloat16, device=DEV)
        return [nvq.gemv_mxfp4(q, s, x, out=o[0]), nvq.gemm_mxfp4(q, s, xq, xs, out=o[1]), *nvq.quant_mxfp4(x, out=c),
                nvq.dequant_mxfp4(xq, xs, out=d)]

    nvq.lib()
    assert nvq._calls is not None
    fast = all_calls()
    monkeypatch.setattr(nvq, "_calls", None)
    for a, b in zip(fast, all_calls()):
        assert torch.equal(a, b)


# ---- operands that are not finite, at sizes that reach every kernel and whose last pass meets columns a second time ----
BEYOND = [
    # dot products: blocks past the end of the row, one wave to a row and four, one token and two
    (1, 20, 2080), (1, 3000, 2080), (1, 8200, 1056), (1, 20, 4128), (1, 20, 8224), (2, 20, 2080), (2, 20, 4128), (2, 20, 8224),
    # activations read with the weights: a row tile to a workgroup, four, and one of two token tiles
    (3, 40, 2176), (5, 8209, 2176), (20, 40, 2176),
    # all activations in LDS
    (1, 8209, 16672), (2, 17000, 4128), (3, 8209, 4224),
    # activations shared through LDS: surplus slices in the last turn, and none
    (16, 40, 4352), (6, 4100, 1440), (9, 8200, 1376), (20, 40, 4224), (20, 4100, 1440), (20, 8200, 1376), (9, 65539, 4128), (20, 65539, 4128),
    # activations in registers: a last wave whose blocks begin before its share
    (3, 65523, 544), (20, 65523, 544), (3, 65523, 2080), (20, 65523, 2080)]


def positive_weights(N, K, seed):
    """Random codes 0.5 .. 6 at scale bytes 121 .. 124, and the rows that a test looks at: the first and last forty."""
    rng = np.random.default_rng(seed)
    q = rng.integers(0, 256, (N, K // 2), dtype=np.uint8) & 0x77
    q |= ((q & 0x07) == 0).astype(np.uint8) | ((q & 0x70) == 0).astype(np.uint8) << 4
    s = rng.integers(121, 125, (N, K // 32), dtype=np.uint8)
    return q, s, np.unique(np.concatenate([np.arange(min(N, 40)), np.arange(max(0, N - 40), N)])), rng


@gpu
@pytest.mark.parametrize("M,N,K", BEYOND)
def test_gemv_of_infinite_activations(M, N, K):
    """Positive weights: a token of infinities gives infinities in every row, one at the end of another token its sign, and
    the tokens beside them their exact sums."""
    q, s, rows, rng = positive_weights(N, K, M + N + K)
    x = rng.integers(1, 4, (M, K)).astype(np.float64)
    want = x @ np_mx.dequant(q[rows], s[rows]).T
    qd, sd = dev(q), dev(s)
    for what in (np.inf, -np.inf):
        for at in (slice(None), slice(K - 1, K), slice(K // 2, K // 2 + 1), slice(0, 1), slice(K - 200, K - 199)):
            bad = x.copy()
            bad[M - 1, at] = what
            y = f64(nvq.gemv_mxfp4(qd, sd, dev(bad).bfloat16()))[:, rows]
            assert (y[M - 1] == what).all(), at
            assert np.array_equal(y[:M - 1], want[:M - 1])


@gpu
@pytest.mark.parametrize("M,N,K", BEYOND)
def test_gemv_of_weights_at_and_beyond_the_last_scales(M, N, K):
    """Scale bytes 253 and 254: values that bf16 holds are themselves, those beyond it infinite (as dequant_mxfp4 gives them);
    byte 255: no number.  Each in the first, the last or every block of a row."""
    q, s, rows, rng = positive_weights(N, K, M + N + K)
    last = N - 1
    s[3], q[3] = 254, 0x77                              # 6 * 2^127, every block
    s[5, -1], q[5, -16:] = 253, 0x77                    # 6 * 2^126, the last block
    s[6, 0], q[6, :16] = 254, 0x44                      # 2 * 2^127, the first block
    q[7], s[7, -1], q[7, -16:] = 0, 254, 0x21           # 0.5 and 1 times 2^127, the last block of a row of zeros
    q[8], s[8, 0], q[8, :16] = 0, 253, 0x53             # 1.5 and 3 times 2^126, the first one
    s[9, -1] = 255
    s[10, 0], q[10, :16] = 255, 0
    s[last, -1], q[last, -16:] = 253, 0xff              # -6 * 2^126, the last block of the last row
    x = rng.integers(1, 4, (M, K)) * 2.0 ** -30
    w = np_mx.dequant(q[rows], s[rows])
    w[np.abs(w) >= 2.0 ** 128] = np.inf * np.sign(w[np.abs(w) >= 2.0 ** 128])
    assert np.isinf(w[[3, 5, 6, -1]]).any(1).all() and np.isfinite(w[[7, 8]]).all()
    with np.errstate(invalid="ignore"):
        want = x @ np.nan_to_num(w, posinf=0.0, neginf=0.0).T
    want[:, [3, 5, 6]], want[:, [9, 10]], want[:, -1] = np.inf, np.nan, -np.inf
    y = f64(nvq.gemv_mxfp4(dev(q), dev(s), dev(x).bfloat16()))[:, rows]
    assert np.array_equal(y, want, equal_nan=True)


@gpu
@pytest.mark.parametrize("M,N,K", [(3, 20, 96), (40, 70, 288), (12, 40, 2080), (90, 370, 1056), (300, 300, 544), (700, 9000, 544),
                                   (3585, 4001, 544)])
def test_gemm_of_the_last_scales(M, N, K):
    """Scale bytes 253 and 254 on either side, small values on the other: the product itself, also of values beyond bf16."""
    rng = np.random.default_rng(M + K)
    q, s = np_mx.random_mx(rng, N, K)
    xq, xs = np_mx.random_mx(rng, M, K, 1, 96)
    # blocks of 253 and 254 alone in their rows: sums of whole multiples of 2^94 * 2^-32, below 2^24 of them
    for r, (at, byte) in enumerate(((-1, 254), (0, 253), (K // 64, 254))):
        q[r], s[r, at] = 0, byte
        q[r, 16 * (at % (K // 32)):16 * (at % (K // 32)) + 16] = rng.integers(0, 256, 16, dtype=np.uint8)
    want = np_mx.dequant(xq, xs) @ np_mx.dequant(q, s).T
    y = f64(nvq.gemm_mxfp4(dev(q), dev(s), dev(xq), dev(xs)))
    assert np.array_equal(y + 0.0, want.astype(np.float32).astype(np.float64) + 0.0)
    y = f64(nvq.gemm_mxfp4(dev(xq), dev(xs), dev(q), dev(s)))
    assert np.array_equal(y + 0.0, want.T.astype(np.float32).astype(np.float64) + 0.0)


# all activations of a few tokens in LDS: one token of more inputs than dot products take (three to seven steps to
# a row tile, the largest K that fits), two and three tokens; many row tiles and few
@gpu
@pytest.mark.parametrize("M,N,K", [(1, 40, 20480), (1, 17, 24576), (1, 8209, 16672), (1, 8200, 28416),
                                   (2, 17000, 4128), (2, 16400, 2112), (2, 16500, 8224),
                                   (3, 8193, 4128), (3, 8209, 9152), (3, 40, 8192), (3, 33000, 2080)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gemv_exact_sums_of_activations_in_lds(M, N, K, dtype):
    q, s, x, _, xv = exact_case(M, N, K, M + N + K, False)
    want = xv @ np_mx.dequant(q, s).T
    y = nvq.gemv_mxfp4(dev(q), dev(s), dev(x).bfloat16(), out_dtype=dtype)
    assert bits_equal(f64(y) + 0.0, f64(torch.from_numpy(want).float().to(dtype)) + 0.0)


# tiles of 128 x 64 in two slices of K: whole and ragged rows and tokens, windows of sixteen blocks whole, short and
# past the end
@gpu
@pytest.mark.parametrize("M,N,K", [(512, 4096, 1024), (129, 9000, 544), (450, 3700, 8224), (700, 2500, 800),
                                   (500, 4001, 1312), (64, 24577, 512)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gemm_exact_sums_of_medium_tiles(M, N, K, dtype):
    q, s, xq, xs, xv = exact_case(M, N, K, M + N + K, True)
    want = xv @ np_mx.dequant(q, s).T
    assert np.abs(want).max() * 2 ** 9 < 2 ** 24
    y = nvq.gemm_mxfp4(dev(q), dev(s), dev(xq), dev(xs), out_dtype=dtype)
    assert bits_equal(f64(y) + 0.0, f64(torch.from_numpy(want).float().to(dtype)) + 0.0)

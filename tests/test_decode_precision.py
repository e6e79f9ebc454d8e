"""Attention and adapters where what is left of large terms that cancel shows how many bits the terms had."""
import numpy as np
import pytest
import torch

from paper_2604_21026_amd import nvq
from tests import np_decode as ref
from tests.test_cache import DEV, Pool, dev, f64

gpu = pytest.mark.gpu


def cancelling(rng, B, n, D, e4m3):
    """B sequences of n tokens, one head.  Token `at` scores d below the top, and its values are cancelled, but for the
    last bits of its weight, by those of the tokens behind it, which score the top; all others score 200 below.  The
    scores are products of few bits, so exact."""
    many = 4 if e4m3 else 2  # (that many values of 4 or of 8 bits say what the weighted ones are, to 16 bits)
    pool = Pool(rng, [n] * B, 1, D, 16, e4m3)
    q = np.zeros((B, 1, D))
    d = rng.choice(np.arange(5, 33), B) / 32.0  # of the score, times the sixteenths of q
    q[:, 0, 0] = 1.0
    at = (n - 1 - many) // 32 * 32
    for b in range(B):
        k, v = np.zeros((n, 1, D)), np.zeros((n, 1, D))
        k[:, 0, 0] = -200.0
        k[at:at + many + 1, 0, 0] = 0.0
        k[at, 0, 0] = -d[b] if e4m3 else -d[b] * (1 + rng.integers(1, 16) / 128.0)
        k = ref.to_bf16(k.astype(np.float32)).astype(np.float64)
        v[at, 0] = -(1 + rng.integers(0, 8, D) / 8.0)
        pool.put(b, np.arange(n), k, v)
        held = lambda x, t: x[pool.table[b, t // 16], 0, t % 16]
        left = np.exp(held(pool.k, at)[0]) * -held(pool.v, at)
        for i in range(1, many + 1):
            row = ref.to_bf16(left.astype(np.float32)).astype(np.float64)
            pool.put(b, np.array([at + i]), k[at + i:at + i + 1], row[None, None])
            left = left - held(pool.v, at + i)
    return pool, q, many


@gpu
@pytest.mark.parametrize("n,D", [(3, 64), (5, 64), (40, 64), (70, 64), (1003, 64), (5000, 64), (40, 32), (40, 96), (1003, 128), (40, 160), (1003, 256)])
@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("dtype,eps", [(torch.float32, 0.0), (torch.bfloat16, ref.EPS16)])
def test_attention_weighs_values_with_weights_of_fp32(n, D, e4m3, dtype, eps):
    """Counted in halves of a unit of fp32 (2^-24) of the sum of the sizes.  The weight: the power of two that it is, up to
    1.62, is rounded as a product, its factor log2 e by half as much, 1.5 * 1.62 * ln 2, and the exponential is off by a
    unit, 2.  The sums: many + 1 products, each addition off by up to a unit, 2 each; the sums of the weights' parts, and of
    waves and workgroups (of which all but one weigh nothing), 4."""
    rng = np.random.default_rng(n)
    n = n + 2 if e4m3 else n
    B = 24
    pool, q, many = cancelling(rng, B, n, D, e4m3)
    y = f64(nvq.attention(pool.device(), dev(q, torch.bfloat16), dev(pool.table), dev(np.full(B, n, np.int32)), scale=1.0, out_dtype=dtype))
    halves = 1.7 + 2 + 2 * (many + 1) + 4
    t = np.arange(n)
    for b in range(B):
        k, v = (x[pool.table[b, t // 16], 0, t % 16] for x in (pool.k, pool.v))
        want, _, _, _, mean = ref.attention(q[b], k, v, 1.0, 0.0)
        assert (np.abs(want) < 2.0 ** -14 * mean).all()
        off = np.abs(y[b] - want) / (halves * ref.EPS32 * (mean + np.abs(want)) + eps * np.abs(want))
        assert off.max() <= 1, (b, off.max())


@gpu
@pytest.mark.parametrize("M,K,N,R", [(1, 2048, 50, 16), (5, 1024, 130, 32), (20, 992, 40, 24), (64, 512, 33, 64), (3, 4096, 700, 128), (70, 320, 2051, 40), (300, 96, 257, 256)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_adapters_take_h_with_all_its_bits(M, K, N, R, dtype):
    """h of 24 bits, whole numbers, and weights of one and minus one under which all but their last bits cancel: every sum is
    exact, and so is the result but for its one rounding."""
    rng = np.random.default_rng(M + N)
    n = 3
    # x: three numbers that make h's three parts, in columns of their own; ones and zeros of a say which h has them
    x, a = np.zeros((M, K)), np.zeros((n, R, K))
    col = rng.permutation(K)[:3]
    x[:, col[0]] = rng.integers(128, 256, M) * 2.0 ** 15
    x[:, col[1]] = (2 * rng.integers(64, 128, M) + 1) * 2.0 ** 7
    x[:, col[2]] = 2 * rng.integers(0, 64, M) + 1
    a[:, :, col[0]] = 1
    a[:, :, col[1:]] = rng.integers(0, 2, (n, R, 2))
    # b: as many of one as of minus one
    sign = np.repeat([1.0, -1.0], R // 2)
    b = np.stack([[rng.permutation(sign) for _ in range(N)] for _ in range(n)])
    y = rng.integers(-9, 10, (M, N)).astype(np.float64)
    ids = rng.integers(-1, n, M).astype(np.int32)
    want = y.copy()
    for m, e in enumerate(ids):
        if e >= 0:
            h = a[e] @ x[m]
            assert h.max() < 2 ** 24 and (h % 2 ** 7).any()
            want[m] += b[e] @ h
    assert np.abs(want).max() < 2 ** 24 and (M < 5 or (want % 2 ** 7).any())
    as_bf16 = lambda t: dev(t, torch.bfloat16)
    for t in (x, a, b):
        assert np.array_equal(f64(as_bf16(t)), t)
    got = nvq.adapters_add(nvq.Adapters(as_bf16(a), as_bf16(b)), as_bf16(x), dev(ids), dev(y, dtype))
    if dtype == torch.bfloat16:
        want = ref.to_bf16(want.astype(np.float32)).astype(np.float64)
    assert np.array_equal(f64(got), want)

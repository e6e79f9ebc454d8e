"""Low-rank adapters beside a layer, each token its own, against a plain form in 64 bits."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2604_21026_amd import nvq
from tests.np_decode import EPS16, EPS32

DEV = "cuda:0"
gpu = pytest.mark.gpu


def f64(t):
    return t.double().cpu().numpy()


def test_adapters_refusals_before_any_launch():
    L, a = nvq.lib(), 0x1000

    def call(x=a, ids=a, M=4, y=a, out=a, dt=1, ws=a, bytes_=1 << 24, none=False, **kw):
        v = dict(a=a, b=a, scales=a, n=3, K=64, N=50, R=16)
        v.update(kw)
        s = nvq.AdaptersStruct(*v.values())
        return L.nvq_adapters_add(None if none else C.addressof(s), x, ids, M, y, out, dt, ws, bytes_, None)

    s = nvq.AdaptersStruct(a, a, a, 3, 64, 50, 16)
    need = L.nvq_adapters_workspace_bytes(C.addressof(s), 4)
    assert need >= 4 * 16 * 4 and call(bytes_=need - 1) == 6 and call(ws=None) == 6 and call(ws=a + 64) == 6
    assert call(none=True) == 1 and call(a=None) == 1 and call(b=None) == 1 and call(x=None) == 1 and call(ids=None) == 1
    assert call(y=None) == 1 and call(out=None) == 1 and call(dt=2) == 1
    assert call(n=0) == 2 and call(n=65537) == 2 and call(K=48) == 2 and call(K=0) == 2 and call(K=65568) == 2 and call(N=0) == 2
    assert call(R=0) == 2 and call(R=12) == 2 and call(R=264) == 2 and call(M=0) == 2 and call(M=65537) == 2 and call(N=(1 << 24) + 1) == 2
    assert call(a=a + 8) == 3 and call(b=a + 2) == 3 and call(scales=a + 2) == 3 and call(x=a + 4) == 3 and call(ids=a + 1) == 3
    assert call(y=a + 8) == 3 and call(out=a + 4) == 3
    assert L.nvq_adapters_workspace_bytes(None, 4) == 0 and L.nvq_adapters_workspace_bytes(C.addressof(s), 0) == 0


def test_the_binding_refuses_adapters_that_do_not_fit():
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype)
    for args in [(z(2, 8, 64), z(2, 50, 8)), (z(2, 8, 64), z(3, 50, 8)), (z(2, 8, 64), z(2, 50, 16)), (z(8, 64), z(50, 8)),
                 (z(2, 8, 64), z(2, 50, 8), z(3, dtype=torch.float32))]:
        with pytest.raises(ValueError):
            nvq.Adapters(*args)


def plain(a, b, scales, x, ids, y):
    """The results, and the sum of the sizes of what is added up for each: of A's products under |B|."""
    want, size = y.copy(), np.abs(y)
    for m, e in enumerate(ids):
        if 0 <= e < len(a):
            want[m] += scales[e] * (b[e] @ (a[e] @ x[m]))
            size[m] += abs(scales[e]) * (np.abs(b[e]) @ (np.abs(a[e]) @ np.abs(x[m])))
    return want, size


CASES = [  # M, n, K, N, R
    (1, 1, 32, 1, 8), (1, 4, 2048, 2048, 16), (2, 3, 96, 17, 24), (15, 5, 160, 63, 40), (16, 16, 256, 64, 8), (17, 2, 1440, 1003, 64),
    (32, 7, 4096, 512, 32), (33, 40, 64, 130, 256), (70, 3, 512, 257, 136), (5, 2, 14336, 96, 128), (200, 9, 320, 1024, 16), (3, 2, 65536, 16, 8),
    (300, 9, 96, 130, 24), (600, 2, 64, 65, 16), (450, 70, 32, 1100, 40), (1300, 3, 64, 260, 8), (64, 1, 64, 50, 16), (40, 64, 96, 70, 24)]


@gpu
@pytest.mark.parametrize("M,n,K,N,R", CASES)
@pytest.mark.parametrize("dtype,eps", [(torch.float32, EPS32), (torch.bfloat16, EPS16)])
def test_adapters(M, n, K, N, R, dtype, eps):
    g = torch.Generator().manual_seed(M + K + N)
    a, b = (torch.randn((n, R, K), generator=g) * K ** -0.5).bfloat16(), (torch.randn((n, N, R), generator=g) * R ** -0.5).bfloat16()
    x, y = torch.randn((M, K), generator=g).bfloat16(), torch.randn((M, N), generator=g).to(dtype)
    scales = torch.rand((n,), generator=g) * 2 - 0.5
    handle = nvq.Adapters(a.to(DEV), b.to(DEV), scales.to(DEV))
    ws = handle.workspace(M)
    ws.fill_(255)  # (whatever it holds)
    for ids in (torch.randint(-1, n + 1, (M,), generator=g, dtype=torch.int32), torch.arange(M, dtype=torch.int32) // 5 % n,
                torch.full((M,), -1, dtype=torch.int32)):
        want, size = plain(f64(a), f64(b), f64(scales), f64(x), ids.tolist(), f64(y))
        got = nvq.adapters_add(handle, x.to(DEV), ids.to(DEV), y.to(DEV), workspace=ws)
        # fp32 sums of K products, then of R, each rounding and its like inside the matrix instructions
        bound = 2 * (K + R + 16) * EPS32 * size + eps * np.abs(want)
        assert (np.abs(f64(got) - want) <= bound).all()
        none = (ids < 0) | (ids >= n)
        assert torch.equal(got.cpu()[none], y[none])
        here = y.to(DEV)
        assert torch.equal(nvq.adapters_add(handle, x.to(DEV), ids.to(DEV), here, out=here), got) and torch.equal(here, got)


@gpu
@pytest.mark.parametrize("M", [6, 21])
def test_adapters_of_exact_sums(M):
    """Small whole numbers: every sum exact, results to the bit, with scales left out."""
    g = torch.Generator().manual_seed(M)
    n, K, N, R = 4, 480, 77, 56
    a, b = (torch.randint(-3, 4, s, generator=g).bfloat16() for s in ((n, R, K), (n, N, R)))
    x, y = torch.randint(-3, 4, (M, K), generator=g).bfloat16(), torch.randint(-9, 10, (M, N), generator=g).float()
    ids = torch.randint(-1, n, (M,), generator=g, dtype=torch.int32)
    want, size = plain(f64(a), f64(b), np.ones(n), f64(x), ids.tolist(), f64(y))
    assert size.max() < 2 ** 24
    got = nvq.adapters_add(nvq.Adapters(a.to(DEV), b.to(DEV)), x.to(DEV), ids.to(DEV), y.to(DEV))
    assert np.array_equal(f64(got), want)


@gpu
def test_adapters_of_tokens_without_a_number():
    """A NaN or an infinity of one token or of an adapter shows in its own tokens alone, as in the plain sum."""
    g = torch.Generator().manual_seed(2)
    M, n, K, N, R = 19, 4, 128, 50, 16
    a, b = torch.rand((n, R, K), generator=g).bfloat16() + 0.5, torch.rand((n, N, R), generator=g).bfloat16() + 0.5
    x, y = torch.rand((M, K), generator=g).bfloat16(), torch.zeros((M, N))
    ids = (torch.arange(M) % n).int()
    ids[18] = -1
    x[0, 5], x[17, 9], x[18, 3] = float("nan"), float("inf"), float("nan")
    b[2, 7, 3], a[3, 4, 11] = float("nan"), float("inf")
    got = f64(nvq.adapters_add(nvq.Adapters(a.to(DEV), b.to(DEV)), x.to(DEV), ids.to(DEV), y.to(DEV)))
    assert np.isnan(got[0]).all() and np.isposinf(got[17]).all() and (got[18] == 0).all()
    for m in range(1, 17):
        if ids[m] == 2:
            assert np.isnan(got[m, 7]) and np.isfinite(np.delete(got[m], 7)).all()
        elif ids[m] == 3:
            assert np.isposinf(got[m]).all()
        else:
            assert np.isfinite(got[m]).all()


@gpu
@pytest.mark.parametrize("M,N", [(3, 50), (20, 5000)])
def test_adapters_of_infinite_weights(M, N):
    """An infinite weight makes its output infinite, whatever the bits of what it meets; a zero that it meets makes it NaN."""
    n, K, R = 2, 64, 16
    a, b, x = (torch.ones(s, dtype=torch.bfloat16) for s in ((n, R, K), (n, N, R), (M, K)))
    a[:, 1] = 0
    a[:, 2] = 1 / 3  # (sums that take more than eight bits)
    b[0, 5, 0], b[0, 6, 2], b[0, 7, 1], b[1, N - 1, 3] = float("inf"), -float("inf"), float("inf"), -float("inf")
    ids = torch.arange(M, dtype=torch.int32) % n
    for dtype in (torch.float32, torch.bfloat16):
        got = f64(nvq.adapters_add(nvq.Adapters(a.to(DEV), b.to(DEV)), x.to(DEV), ids.to(DEV), torch.ones((M, N), dtype=dtype, device=DEV)))
        for m in range(M):
            at = [5, 6, 7] if m % n == 0 else [N - 1]
            assert np.isfinite(np.delete(got[m], at)).all()
            if m % n == 0:
                assert np.isposinf(got[m, 5]) and np.isneginf(got[m, 6]) and np.isnan(got[m, 7])
            else:
                assert np.isneginf(got[m, N - 1])


@gpu
@pytest.mark.parametrize("M,n,K,N,R", [(64, 64, 96, 500, 32), (64, 64, 96, 513, 32), (1, 3, 1024, 28672, 32), (1, 3, 1056, 300, 32), (16, 9, 2048, 1029, 16),
                                       (31, 2, 1984, 129, 16), (64, 5, 4096, 640, 8), (64, 5, 4128, 640, 8), (65, 5, 96, 130, 24), (9, 20, 32, 127, 24)])
def test_adapters_around_the_sizes_of_one_launch(M, n, K, N, R):
    """With weights that nothing may read: adapters that no token has hold no numbers, and x neither where a token has no adapter."""
    g = torch.Generator().manual_seed(M * K + N)
    nan = float("nan")
    a, b = (torch.randn((n, R, K), generator=g) * K ** -0.5).bfloat16(), (torch.randn((n, N, R), generator=g) * R ** -0.5).bfloat16()
    x, y = torch.randn((M, K), generator=g).bfloat16(), torch.randn((M, N), generator=g)
    scales = torch.rand((n,), generator=g) + 0.5
    ids = torch.randint(0, max(1, n - 1), (M,), generator=g, dtype=torch.int32)
    ids[torch.rand((M,), generator=g) < 0.2] = n
    none = ids == n
    want, size = plain(f64(a), f64(b), f64(scales), f64(x), ids.tolist(), f64(y))
    unused = [e for e in range(n) if e not in ids.tolist()]
    a[unused], b[unused], x[none] = nan, nan, nan
    handle = nvq.Adapters(a.to(DEV), b.to(DEV), scales.to(DEV))
    got = nvq.adapters_add(handle, x.to(DEV), ids.to(DEV), y.to(DEV))
    # fp32 sums of K products, then of R, each rounding and its like inside the matrix instructions
    bound = 2 * (K + R + 16) * EPS32 * size + EPS32 * np.abs(want)
    assert (np.abs(f64(got) - want) <= bound).all() and torch.equal(got.cpu()[none], y[none])
    here = y.to(DEV)
    assert torch.equal(nvq.adapters_add(handle, x.to(DEV), ids.to(DEV), here, out=here), got)

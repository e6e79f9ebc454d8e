"""The operators of a decode step at the largest sizes that they take."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2604_21026_amd import nvq
from tests.test_cache import DEV, Pool, bf16, check_attention, dev, f64, same_bits

gpu = pytest.mark.gpu


def test_adapters_of_the_most_tokens_and_outputs_are_not_refused():
    """2^16 tokens of 2^24 outputs: past all checks of sizes, stopped by the workspace that is not there."""
    L, a = nvq.lib(), 0x1000
    for M, N in ((1 << 16, 1 << 24), (1 << 16, (1 << 19) + 1), ((1 << 11) + 1, 1 << 24)):
        s = nvq.AdaptersStruct(a, a, a, 3, 64, N, 16)
        assert L.nvq_adapters_workspace_bytes(C.addressof(s), M) > 0
        assert L.nvq_adapters_add(C.addressof(s), a, a, M, a, a, 1, None, 0, None) == 6


@gpu
def test_adapters_of_more_than_2_35_results():
    """In place; few tokens have an adapter, the last one among them."""
    M, N, K, R = 4200, 1 << 23, 32, 8
    assert M * N > 1 << 35
    a, b = torch.ones((1, R, K), dtype=torch.bfloat16, device=DEV), torch.zeros((1, N, R), dtype=torch.bfloat16, device=DEV)
    b[0, 5], b[0, N - 1, 2] = 1.0, 1.0
    x = torch.ones((M, K), dtype=torch.bfloat16, device=DEV)
    ids = torch.full((M,), -1, dtype=torch.int32, device=DEV)
    have = [0, 63, 64, 4100, M - 1]
    ids[have] = 0
    y = torch.zeros((M, N), dtype=torch.bfloat16, device=DEV)
    assert nvq.adapters_add(nvq.Adapters(a, b), x, ids, y, out=y) is y
    want = torch.zeros(N, dtype=torch.bfloat16, device=DEV)
    want[5], want[N - 1] = R * K, K
    for m in have:
        assert torch.equal(y[m], want)
        y[m] = 0
    assert not any(bool(part.any()) for part in y.split(300))
    del y
    torch.cuda.empty_cache()


@gpu
@pytest.mark.parametrize("heads,D", [(2, 32), (2, 160), (1, 160)])
def test_cache_calls_of_the_most_rows(heads, D):
    """As many tokens as rows are allowed, or 2^24: appended, and read back by twice the rows' threads."""
    T, page = 1 << 24, 1024
    assert T * 2 * heads <= 1 << 26
    cache = nvq.Cache.empty(T // page, heads, page, D, torch.uint8, DEV)
    table = torch.arange(T // page, dtype=torch.int32, device=DEV).flip(0).contiguous().view(1, -1)
    zero, at = torch.zeros(T, dtype=torch.int32, device=DEV), torch.arange(T, dtype=torch.int32, device=DEV)
    # a token's keys are the low digits of its number, its values the high ones: four bits each, which 8 bits hold exactly
    digit = lambda t, s: (t >> s & 15).bfloat16()
    k = torch.empty((T, heads, D), dtype=torch.bfloat16, device=DEV)
    v = torch.empty((T, heads, D), dtype=torch.bfloat16, device=DEV)
    for x, shifts in ((k, (0, 4, 8)), (v, (12, 16, 20))):
        for part in range(0, T, 1 << 20):
            here = at[part:part + (1 << 20)]
            x[part:part + (1 << 20)] = digit(here, shifts[0])[:, None, None]
            x[part:part + (1 << 20), :, 1] = digit(here, shifts[1])[:, None]
            x[part:part + (1 << 20), heads - 1, D - 1] = digit(here, shifts[2])
    nvq.cache_append(cache, table, at, k, v, sequences=zero)
    back = (torch.full_like(k, -1), torch.full_like(v, -1))
    nvq.cache_read(cache, table, at, zero, out=back)
    for got, want in zip(back, (k, v)):
        assert all(torch.equal(g, w) for g, w in zip(got.split(1 << 20), want.split(1 << 20)))
    del k, v, back, cache
    torch.cuda.empty_cache()


@gpu
@pytest.mark.parametrize("H,heads,lengths", [(1024, 1, [70, 0, 1]), (1024, 1024, [70, 33]), (1024, 8, [300] * 3), (1000, 8, [40] * 70), (1024, 64, [2000])])
@pytest.mark.parametrize("e4m3", [False, True])
def test_a_step_of_the_most_heads(H, heads, lengths, e4m3):
    rng = np.random.default_rng(H + heads)
    D, page, B = 32, 16, len(lengths)
    pool = Pool(rng, lengths, heads, D, page, e4m3, room=1)
    for b, n in enumerate(lengths):
        pool.put(b, np.arange(n), bf16(rng, (n, heads, D)), bf16(rng, (n, heads, D)))
    cache, q, k, v = pool.device(), bf16(rng, (B, H, D)), bf16(rng, (B, heads, D)), bf16(rng, (B, heads, D))
    as_bf16 = lambda x: dev(x, torch.bfloat16)
    table, at = dev(pool.table), dev(np.array(lengths, np.int32))
    out = torch.empty((B, H, D), dtype=torch.bfloat16, device=DEV)
    nvq.cache_append(cache, table, at, as_bf16(k), as_bf16(v), as_bf16(q), out=out)
    assert same_bits(out, q)
    for b, n in enumerate(lengths):
        pool.put(b, np.array([n]), k[b:b + 1], v[b:b + 1])
    lse = torch.empty((B, H), dtype=torch.float32, device=DEV)
    y = nvq.attention(cache, out, table, at + 1, out_dtype=torch.float32, lse=lse)
    check_attention(f64(y), f64(lse), pool, q, [n + 1 for n in lengths], 0, 0.0, D ** -0.5, 0.0)


@gpu
@pytest.mark.parametrize("M,n,K,N,R", [(1 << 16, 3, 32, 70, 8), (40, 1 << 16, 32, 33, 8), (1000, 1 << 16, 64, 260, 16)])
def test_adapters_of_the_most_tokens_and_of_the_most_adapters(M, n, K, N, R):
    """Small whole numbers: every sum exact."""
    g = torch.Generator().manual_seed(M)
    a, b = (torch.randint(-2, 3, s, generator=g, dtype=torch.int8).to(DEV).bfloat16() for s in ((n, R, K), (n, N, R)))
    x, y = torch.randint(-2, 3, (M, K), generator=g).to(DEV).bfloat16(), torch.randint(-9, 10, (M, N), generator=g).to(DEV).float()
    ids = torch.randint(-1, n, (M,), generator=g, dtype=torch.int32).to(DEV)
    ids[0], ids[M - 1] = n - 1, n
    got = nvq.adapters_add(nvq.Adapters(a, b), x, ids, y)
    want = y.double()
    for part in range(0, M, 1024):
        e = ids[part:part + 1024].long()
        live = (e >= 0) & (e < n)
        e = e[live]
        h = (a[e].double() * x[part:part + 1024][live].double().unsqueeze(1)).sum(-1)
        want[part:part + 1024][live] += (b[e].double() * h.unsqueeze(1)).sum(-1)
    assert torch.equal(got.double(), want)

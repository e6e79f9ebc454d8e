"""The operators of a decode step at the largest sizes that they take."""
import ctypes as C

import pytest
import torch

from paper_2604_21026_amd import nvq

DEV = "cuda:0"
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

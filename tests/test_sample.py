"""The next token from logits and given random numbers, against a sorted plain form in 64 bits."""
import numpy as np
import pytest
import torch

from paper_2604_21026_amd import nvq
from tests import np_decode as ref

DEV = "cuda:0"
gpu = pytest.mark.gpu


def dev(a):
    return torch.from_numpy(np.ascontiguousarray(a)).to(DEV)


def test_sample_refusals_before_any_launch():
    L, a = nvq.lib(), 0x1000
    need = L.nvq_sample_workspace_bytes(4, 1000)
    assert need >= 4096
    for M, V in ((0, 5), (1025, 5), (4, 0), (4, (1 << 20) + 1)):
        assert L.nvq_sample_workspace_bytes(M, V) == 0

    def call(logits=a, dt=0, ld=1000, M=4, V=1000, u=a, t=a, k=a, p=a, mp=a, ids=a, ws=a, bytes_=need):
        return L.nvq_sample(logits, dt, ld, M, V, u, t, k, p, mp, ids, ws, bytes_, None)

    assert call(logits=None) == 1 and call(u=None) == 1 and call(ids=None) == 1 and call(dt=2) == 1
    assert call(M=0) == 2 and call(M=1025) == 2 and call(V=0) == 2 and call(ld=999) == 2 and call(V=(1 << 20) + 1, ld=1 << 21) == 2
    assert call(logits=a + 2) == 3 and call(logits=a + 1, dt=1) == 3 and call(u=a + 2) == 3 and call(t=a + 1) == 3
    assert call(k=a + 2) == 3 and call(p=a + 2) == 3 and call(mp=a + 2) == 3 and call(ids=a + 2) == 3
    assert call(ws=None) == 6 and call(ws=a + 128) == 6 and call(bytes_=need - 1) == 6


def check(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, workspace=None, given=None):
    """logits: a tensor on the host; the rest float32 / int32 arrays or None."""
    M = logits.shape[0]
    ask = [None if x is None else dev(x) for x in (temperature, top_k, top_p, min_p)]
    got = nvq.sample(logits.to(DEV) if given is None else given, dev(u), *ask, workspace=workspace).cpu().numpy()
    rows = logits.double().numpy()
    each = [np.full(M, d) if x is None else x for x, d in ((temperature, 1.0), (top_k, 0), (top_p, 1.0), (min_p, 0.0))]
    want = [ref.sample(rows[m], float(u[m]), *(float(x[m]) if i != 1 else int(x[m]) for i, x in enumerate(each))) for m in range(M)]
    assert got.tolist() == [int(x) for x in want]


def asks(rng, M):
    pick = lambda v, t: rng.choice(v, M).astype(t)
    return dict(temperature=pick([0.0, 0.3, 0.7, 1.0, 1.5, 20.0], np.float32), top_k=pick([0, 0, 1, 2, 40, 1000], np.int32),
                top_p=pick([1.0, 1.0, 0.1, 0.5, 0.9, 0.999], np.float32), min_p=pick([0.0, 0.0, 0.05, 0.3], np.float32))


SIZES = [(1, 1), (3, 2), (5, 63), (7, 64), (4, 65), (16, 200), (9, 1023), (8, 1025), (33, 4099), (6, 32003), (4, 128256), (2, 1 << 20)]


@gpu
@pytest.mark.parametrize("M,V", SIZES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_sample(M, V, dtype):
    rng = np.random.default_rng(M + V)
    ws = nvq.sample_workspace(40, 1 << 20, DEV)
    for spread in (0.1, 3.0, 12.0):
        logits = torch.from_numpy(rng.standard_normal((M, V)).astype(np.float32) * spread).to(dtype)
        u = rng.random(M).astype(np.float32)
        check(logits, u, workspace=ws)
        check(logits, u, workspace=ws, **asks(rng, M))
        assert int(ws[:4096].sum()) == 0
        check(logits, u, temperature=np.full(M, 0.8, np.float32), top_k=np.full(M, 50, np.int32), top_p=np.full(M, 0.95, np.float32),
              min_p=np.full(M, 0.02, np.float32))


@gpu
def test_sample_of_a_peaked_row_each_filter_by_itself():
    rng = np.random.default_rng(3)
    M, V = 12, 50000
    x = rng.standard_normal((M, V)) * 2.0
    x[:, rng.choice(V, 60, False)] += np.linspace(14, 2, 60)
    logits = torch.from_numpy(x.astype(np.float32))
    for kw in (dict(top_k=np.arange(1, M + 1)), dict(top_p=np.linspace(0.05, 0.999, M)), dict(min_p=np.geomspace(1e-6, 1.0, M)),
               dict(temperature=np.geomspace(0.05, 5.0, M)), dict(top_k=np.full(M, V)), dict(top_k=np.full(M, V - 1)),
               dict(top_k=np.full(M, 2 ** 31 - 1))):
        check(logits, rng.random(M).astype(np.float32), **{k: v.astype(np.int32 if k == "top_k" else np.float32) for k, v in kw.items()})


@gpu
def test_sample_of_equal_logits_goes_by_index():
    """All weights 1: token floor(u n) of the first n, exactly."""
    V = 3000
    u = np.array([0.0, 0.25, 0.5, 1 - 2.0 ** -24, 0.125, 0.75], np.float32)
    for value in (0.0, -3.5, 1e30):
        logits = torch.full((6, V), value)
        got = nvq.sample(logits.to(DEV), dev(u)).cpu().numpy()
        assert got.tolist() == [int(float(x) * V) for x in u]
        k = np.array([1, 8, 2999, 3000, 16, 100], np.int32)
        got = nvq.sample(logits.to(DEV), dev(u), top_k=dev(k)).cpu().numpy()
        assert got.tolist() == [int(float(x) * n) for x, n in zip(u, k)]
        # those before which less than p of the sum lies: of n equal weights ceil(p n)
        p = np.array([0.5, 0.25, 0.125, 0.5, 2.0 ** -10, 0.75], np.float32)
        got = nvq.sample(logits.to(DEV), dev(u), top_p=dev(p)).cpu().numpy()
        assert got.tolist() == [int(float(x) * np.ceil(float(y) * V)) for x, y in zip(u, p)]
        assert nvq.sample(logits.to(DEV), dev(u), temperature=torch.zeros(6, device=DEV)).tolist() == [0] * 6
    two = torch.zeros((2, V))
    two[:, 1::2] = -0.0  # equal too
    assert nvq.sample(two.to(DEV), dev(np.array([0.5, 0.0], np.float32))).tolist() == [V // 2, 0]


@gpu
def test_sample_of_rows_without_a_number():
    inf, nan = float("inf"), float("nan")
    V = 500
    x = torch.full((7, V), -inf)
    x[1] = nan
    x[2, 77] = -4.0
    x[3, 10], x[3, 400] = inf, inf
    x[4, ::2], x[4, 1::2] = nan, 1.0
    x[5, 3], x[5, 9] = 2.0, 2.0
    x[6, 20:40] = -3e38
    u = np.array([0.3, 0.3, 0.999, 0.9, 0.5, 0.6, 0.51], np.float32)
    for dtype in (torch.float32, torch.bfloat16):
        got = nvq.sample(x.to(dtype).to(DEV), dev(u)).tolist()
        assert got == [-1, -1, 77, 10, 2 * 125 + 1, 9, 30]


@gpu
def test_sample_of_arguments_at_their_ends():
    nan, inf = float("nan"), float("inf")
    g = torch.Generator().manual_seed(1)
    x = torch.randn((1, 700), generator=g).repeat(10, 1)
    order = torch.argsort(-x[0], stable=True).tolist()
    f = lambda *v: dev(np.array(v, np.float32))
    first = [order[0]] * 10
    half = f(*[0.5] * 10)
    assert nvq.sample(x.to(DEV), f(0.0, -1.0, nan, -inf, -0.0, 0.0, 0.0, 0.0, 0.0, 0.0)).tolist() == first
    assert nvq.sample(x.to(DEV), f(1.0, 2.0, inf, *[1.0] * 7)).tolist() == [order[-1]] * 10
    assert nvq.sample(x.to(DEV), half, f(0.0, -1.0, nan, -inf, -0.0, 1e-30, 1e-40, 0.0, 0.0, 0.0)).tolist() == first
    assert nvq.sample(x.to(DEV), half, top_p=f(0.0, -1.0, nan, -inf, 1e-30, 1e-40, 0.0, 0.0, 0.0, 0.0)).tolist() == first
    assert nvq.sample(x.to(DEV), half, min_p=f(1.0, 2.0, inf, 1.5, *[1.0] * 6)).tolist() == first
    free = nvq.sample(x.to(DEV), half).tolist()
    assert nvq.sample(x.to(DEV), half, top_p=f(1.0, 2.0, inf, *[1.0] * 7), min_p=f(0.0, -1.0, nan, -inf, *[0.0] * 6),
                      top_k=dev(np.array([0, -1, -2 ** 31, 700, 701, 0, 0, 0, 0, 0], np.int32))).tolist() == free
    # temperature without end: every token alike, in the order of the logits
    assert nvq.sample(x.to(DEV), half, f(*[inf] * 10)).tolist() == [order[350]] * 10


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_sample_of_rows_that_lie_apart_at_any_alignment(dtype):
    rng = np.random.default_rng(8)
    for M, V, ld, first in ((4, 1001, 1003, 1), (3, 4096, 5000, 3), (2, 30001, 30002, 1)):
        flat = torch.from_numpy(rng.standard_normal(M * ld + 8).astype(np.float32) * 4).to(dtype)
        view = lambda t: t[first:first + M * ld].view(M, ld)[:, :V]
        check(view(flat).contiguous(), rng.random(M).astype(np.float32), given=view(flat.to(DEV)), **asks(rng, M))


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_sample_of_rows_that_are_mostly_masked(dtype):
    """All but a few tokens at the type's lowest value, or far below: filters that reach into them."""
    rng = np.random.default_rng(21)
    M, V = 8, 60000
    x = np.full((M, V), torch.finfo(dtype).min, np.float64)
    x[4:] = -80.0
    for m in range(M):
        x[m, rng.choice(V, 3 + 5 * m, False)] = rng.standard_normal(3 + 5 * m) * 3
    logits, u = torch.from_numpy(x).to(dtype), rng.random(M).astype(np.float32)
    f = lambda v, t=np.float32: np.full(M, v, t)
    for kw in ({}, dict(top_k=f(50, np.int32)), dict(top_p=f(0.9999)), dict(min_p=f(1e-30)), dict(top_k=f(50, np.int32), top_p=f(0.95), min_p=f(1e-25)),
               dict(temperature=f(0.2), top_k=f(1000, np.int32)), dict(temperature=f(3.0), top_k=f(20, np.int32), min_p=f(0.01))):
        check(logits, u, **kw)


@gpu
@pytest.mark.parametrize("spread", [0.02, 2.5, 40.0])
def test_sample_of_low_and_high_temperatures(spread):
    """Filters that end in every part of the bins, behind them, and rows that no bins serve."""
    rng = np.random.default_rng(22)
    M, V = 10, 40000
    logits = torch.from_numpy((rng.standard_normal((M, V)) * spread).astype(np.float32))
    for t in (0.01, 0.1, 0.3, 2.0, 30.0):
        u = rng.random(M).astype(np.float32)
        kw = dict(temperature=np.full(M, t, np.float32))
        check(logits, u, **kw)
        check(logits, u, top_k=np.geomspace(1, V - 1, M).astype(np.int32), **kw)
        check(logits, u, top_k=np.full(M, 50, np.int32), top_p=np.linspace(0.1, 0.99, M).astype(np.float32), min_p=np.full(M, 0.02, np.float32), **kw)


@gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_sample_of_many_equal_logits_among_others(dtype):
    """bf16 values of both signs around powers of two, where their distance changes, many of each: lists of hundreds of equal ones."""
    rng = np.random.default_rng(23)
    M, V = 12, 30000
    for centre, spread in ((0.0, 1.0), (4.0, 0.3), (-4.0, 0.3), (-8.0, 0.5), (16.0, 1.0), (-0.25, 0.02), (-1.0, 0.05)):
        logits = torch.from_numpy((centre + rng.standard_normal((M, V)) * spread).astype(np.float32)).bfloat16().to(dtype)
        u = rng.random(M).astype(np.float32)
        check(logits, u, temperature=np.full(M, 1.5, np.float32))
        check(logits, u, top_k=np.geomspace(2, V - 1, M).astype(np.int32), top_p=np.full(M, 0.9, np.float32))
        # (one value among them that bf16 does not hold)
        if dtype == torch.float32:
            logits[:, 7] += 2.0 ** -12
            check(logits, u, temperature=np.full(M, 1.5, np.float32), top_p=np.full(M, 0.97, np.float32))


@gpu
@pytest.mark.parametrize("V", [700, 40000, 128256])
def test_sample_at_the_end_of_what_is_kept(V):
    """u = 1: the last kept token, whichever filter ends there, however the sums of its bin and of its tokens were rounded."""
    rng = np.random.default_rng(V)
    M = 24
    x = rng.standard_normal((M, V)) * 2.0
    x[:, rng.choice(V, 60, False)] += np.linspace(14, 2, 60)
    logits, one = torch.from_numpy(x.astype(np.float32)), np.ones(M, np.float32)
    f = lambda a: a.astype(np.float32)
    for kw in (dict(min_p=f(np.geomspace(1e-7, 0.5, M))), dict(top_k=np.geomspace(1, 0.9 * V, M).astype(np.int32)),
               dict(top_p=f(np.linspace(0.05, 0.999, M))), dict(min_p=f(np.full(M, 1e-3)), top_k=np.full(M, 40, np.int32)),
               dict(min_p=f(np.full(M, 1e-3)), top_p=f(np.full(M, 0.99)), temperature=f(np.full(M, 1.3))), {}):
        check(logits, one, **kw)
        check(logits, one * 3, **kw)


@gpu
def test_sample_at_the_end_passes_over_tokens_without_a_weight():
    """Below half of 2^-43 a weight counts for nothing: 30.6 below the largest 0.45 of it, as bins of a part's own largest have it."""
    V, few = 128256, 3000
    x = torch.full((4, V), -100.0)
    x[:, 5] = 0.0
    x[0, -few:] = -30.6
    x[1, -few:] = -30.6
    x[1, 40000] = -29.0
    x[2, -50:] = -30.6
    x[3, 100:100 + few] = -30.6
    u = torch.ones(4, device=DEV)
    want = [5, 40000, 5, 5]
    for dtype in (torch.float32, torch.bfloat16):  # (in 16 bits -30.625)
        logits = x.to(dtype).to(DEV)
        assert nvq.sample(logits, u).tolist() == want
        assert nvq.sample(logits, u, top_k=torch.full((4,), 30, dtype=torch.int32, device=DEV)).tolist() == want
        assert nvq.sample(logits, u, min_p=torch.full((4,), 1e-30, device=DEV)).tolist() == want


@gpu
@pytest.mark.parametrize("M,V", [(3, 8192), (3, 8193), (5, 10001), (2, 16384), (3, 16385), (257, 9001), (300, 1000), (270, 20001), (1024, 700)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_sample_of_rows_that_one_workgroup_takes(M, V, dtype):
    """Around one and two blocks of 8192 logits, and of batches with a row to every compute unit; rows that no bins serve among them."""
    rng = np.random.default_rng(M + V)
    ws = nvq.sample_workspace(M, V, DEV)
    for spread in (0.02, 2.5):
        x = rng.standard_normal((M, V)) * spread
        x[0] = 700000.0 + rng.standard_normal(V) * 1000
        x[1, rng.choice(V, V // 2, False)] = -np.inf
        x[2 % M, 1:] = np.nan
        logits = torch.from_numpy(x.astype(np.float32)).to(dtype)
        u = rng.random(M).astype(np.float32)
        check(logits, u, workspace=ws)
        check(logits, u, workspace=ws, **asks(rng, M))
        check(logits, np.ones(M, np.float32), workspace=ws, top_k=rng.integers(1, 60, M).astype(np.int32))
        assert int(ws[:4096].sum()) == 0


@gpu
@pytest.mark.parametrize("M,V", [(86, 32768), (86, 32769), (85, 24577), (256, 30011), (257, 30011), (256, 40011), (255, 40011)])
def test_sample_around_the_rows_of_four_blocks_that_one_workgroup_takes(M, V):
    rng = np.random.default_rng(M + V)
    ws = nvq.sample_workspace(M, V, DEV)
    logits, u = torch.from_numpy((rng.standard_normal((M, V)) * 2.5).astype(np.float32)).bfloat16(), rng.random(M).astype(np.float32)
    check(logits, u, workspace=ws)
    check(logits, u, workspace=ws, **asks(rng, M))
    assert int(ws[:4096].sum()) == 0


@gpu
@pytest.mark.parametrize("M,V", [(28, 128256), (48, 50000), (100, 50001), (3, 270000), (130, 41000)])
def test_sample_of_parts_of_several_blocks(M, V):
    rng = np.random.default_rng(M + V)
    ws = nvq.sample_workspace(M, V, DEV)
    logits, u = torch.from_numpy((rng.standard_normal((M, V)) * 3.0).astype(np.float32)), rng.random(M).astype(np.float32)
    check(logits, u, workspace=ws)
    check(logits, u, workspace=ws, **asks(rng, M))
    assert int(ws[:4096].sum()) == 0


@gpu
@pytest.mark.parametrize("V", [900, 4000, 4096, 128256])
def test_sample_of_many_equal_logits_that_bf16_does_not_hold(V):
    """Lists of up to thousands of equal tokens, alone, in crowds, beside others: by index, whatever their bits."""
    rng = np.random.default_rng(V)
    M = 6
    few = min(V, 4000)
    x = np.full((M, V), -50.0, np.float32)
    x[0, :few] = 0.1
    x[1, rng.choice(V, few, False)] = np.float32(0.1) + np.float32(2.0 ** -20) * rng.integers(0, 3, few).astype(np.float32)
    x[2, :few] = rng.standard_normal(few).astype(np.float16) * np.float16(0.01)
    x[3, rng.choice(V, few, False)] = np.where(rng.random(few) < 0.5, np.float32(0.7), rng.random(few).astype(np.float32))
    x[4, :few] = 0.125  # (one that bf16 holds, and one among them that it does not)
    x[4, 7] = 0.1250001
    x[5, :few] = (4 + rng.standard_normal(few) * 0.02).astype(np.float32)
    logits = torch.from_numpy(x)
    for _ in range(3):
        u = rng.random(M).astype(np.float32)
        check(logits, u)
        check(logits, u, top_k=rng.integers(1, few, M).astype(np.int32), top_p=np.full(M, 0.9, np.float32))
    check(logits, np.ones(M, np.float32))


@gpu
def test_sample_of_many_equal_logits_takes_no_time_out_of_proportion():
    """4000 equal logits, and 4000 different ones: a slot with all of them was ranked in thirty times the time, token by token."""
    def time_of(x):
        out, ws, u = torch.empty(1, dtype=torch.int32, device=DEV), nvq.sample_workspace(1, 4000, DEV), torch.full((1,), 0.5, device=DEV)
        x = x.to(DEV)
        least = float("inf")
        for _ in range(10):
            start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            start.record()
            for _ in range(50):
                nvq.sample(x, u, out=out, workspace=ws)
            end.record()
            torch.cuda.synchronize()
            least = min(least, start.elapsed_time(end))
        return least

    g = torch.Generator().manual_seed(1)
    assert time_of(torch.full((1, 4000), 0.1)) < 10 * time_of(torch.randn((1, 4000), generator=g) * 0.02)

"""A decode step: a layer, adapters beside it, its keys and values into the cache, attention, the next token; call by call,
in graphs, on two streams at once, and each call at the ends of what it takes."""
import numpy as np
import pytest
import torch

from paper_2604_21026_amd import nvq
from tests import np_decode as ref
from tests.test_adapters import plain
from tests.test_cache import DEV, Pool, bf16, check_attention, dev, f64, same_bits

gpu = pytest.mark.gpu


def angles(n, rot):
    a = np.arange(n)[:, None] * 10000.0 ** (-np.arange(0, rot, 2) / rot)
    return np.concatenate((np.cos(a), np.sin(a)), 1).astype(np.float32)


class Step:
    """B sequences that go on from what is in their caches: `x` of the last token, the layer that makes q, k and v of it side
    by side, an adapter per sequence, the head."""

    def __init__(self, seed, B, e4m3=False, H=8, heads=2, D=64, page=16, V=5000, steps=4, workspaces=None):
        rng = np.random.default_rng(seed)
        g = torch.Generator().manual_seed(seed)
        self.B, self.H, self.heads, self.D, self.rng = B, H, heads, D, rng
        self.held = rng.integers(0, 300, B)
        self.pool = Pool(rng, self.held, heads, D, page, e4m3, room=steps)
        for b, n in enumerate(self.held):
            self.pool.put(b, np.arange(n), bf16(rng, (n, heads, D)), bf16(rng, (n, heads, D)))
        K, N = 256, (H + 2 * heads) * D
        self.cache, self.table = self.pool.device(), dev(self.pool.table)
        self.layer = nvq.pack_int4((torch.randn((N, K), generator=g) * K ** -0.5).to(DEV))
        self.head = nvq.pack_int4((torch.randn((V, H * D), generator=g) * 3 * (H * D) ** -0.5).to(DEV))
        self.a, self.b = (torch.randn((3, 16, K), generator=g) * K ** -0.5).bfloat16(), (torch.randn((3, N, 16), generator=g) * 0.25).bfloat16()
        self.adapters = nvq.Adapters(self.a.to(DEV), self.b.to(DEV), torch.tensor([1.0, 0.5, -2.0], device=DEV))
        self.who = dev(rng.integers(-1, 3, B).astype(np.int32))
        self.angles = angles(512, D)
        self.cos_sin = dev(self.angles)
        self.tokens = torch.randn((V, K), generator=g).bfloat16().to(DEV)
        self.ask = [dev(rng.choice(v, B).astype(t)) for v, t in (([0.0, 0.7, 1.0], np.float32), ([0, 20, 400], np.int32), ([1.0, 0.9], np.float32),
                                                                ([0.0, 0.05], np.float32))]
        z = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype, device=DEV)
        self.x, self.p, self.q, self.y = z(B, K), z(B, N), z(B, H, D), z(B, H, D)
        self.logits, self.u, self.ids = z(B, V, dtype=torch.float32), z(B, dtype=torch.float32), z(B, dtype=torch.int32)
        self.at, self.lengths = dev(self.held.astype(np.int32)), z(B, dtype=torch.int32)
        self.ws = workspaces or (self.adapters.workspace(B), self.cache.workspace(B, H), nvq.sample_workspace(B, V, DEV))
        self.start = [t.clone() for t in self.kept()]

    def kept(self):
        return [t for t in self.cache.keep if t is not None] + [self.ids, self.at]

    def rewind(self):
        for t, s in zip(self.kept(), self.start):
            t.copy_(s)

    def run(self):
        H, heads, D = self.H, self.heads, self.D
        torch.index_select(self.tokens, 0, self.ids, out=self.x)
        nvq.gemv_w4a16(*self.layer, self.x, out=self.p)
        nvq.adapters_add(self.adapters, self.x, self.who, self.p, out=self.p, workspace=self.ws[0])
        rows = self.p.view(self.B, -1, D)
        nvq.cache_append(self.cache, self.table, self.at, rows[:, H:H + heads], rows[:, H + heads:], rows[:, :H], self.cos_sin, out=self.q)
        torch.add(self.at, 1, out=self.lengths)
        nvq.attention(self.cache, self.q, self.table, self.lengths, out=self.y, workspace=self.ws[1])
        nvq.gemv_w4a16(*self.head, self.y.view(self.B, H * D), out=self.logits)
        nvq.sample(self.logits, self.u, *self.ask, out=self.ids, workspace=self.ws[2])
        self.at.add_(1)

    def outcome(self):
        """As bits: the cache holds NaN where nothing has been written."""
        return [t.view(torch.uint8).clone() for t in self.kept() + [self.p, self.q, self.y, self.logits]]

    def check(self):
        """The step that has just run, stage by stage."""
        H, heads, D, B = self.H, self.heads, self.D, self.B
        at = self.at.cpu().numpy() - 1
        layer = nvq.gemv_w4a16(*self.layer, self.x, out_dtype=torch.bfloat16)
        want, size = plain(f64(self.a), f64(self.b), f64(self.adapters.keep[2]), f64(self.x), self.who.tolist(), f64(layer))
        assert (np.abs(f64(self.p) - want) <= 2 * (256 + 32) * ref.EPS32 * size + ref.EPS16 * np.abs(want)).all()
        rows = f64(self.p).reshape(B, -1, D)
        turned = ref.rotate(rows[:, :H + heads], self.angles, at, False)
        assert same_bits(self.q, turned[:, :H])
        for b in range(B):
            self.pool.put(b, at[b:b + 1], turned[b:b + 1, H:].astype(np.float64), rows[b:b + 1, H + heads:])
        for got, held in zip(self.pool.raw(self.cache), self.pool.raw(self.pool.device())):
            assert got is None or np.array_equal(got, held)
        check_attention(f64(self.y), None, self.pool, f64(self.q), at + 1, 0, 0.0, D ** -0.5, ref.EPS16)
        ask = [t.cpu().numpy() for t in self.ask]
        rows, u = f64(self.logits), f64(self.u)
        assert self.ids.tolist() == [int(ref.sample(rows[b], u[b], *(x[b].item() for x in ask))) for b in range(B)]
        assert all(int(w[:4096].sum()) == 0 for w in self.ws[1:])


@gpu
@pytest.mark.parametrize("B", [1, 5, 32])
@pytest.mark.parametrize("e4m3", [False, True])
def test_steps(B, e4m3):
    s = Step(B, B, e4m3)
    for _ in range(4):
        s.u.uniform_()
        s.run()
        s.check()


@gpu
@pytest.mark.parametrize("B", [1, 7])
def test_graphs_that_share_workspaces(B):
    """Steps of two sets of sequences, captured over the same workspaces and replayed in turn, eager work between."""
    one = Step(40 + B, B)
    sides = [one, Step(50 + B, B, workspaces=one.ws)]
    draws = [[torch.rand(B, device=DEV) for _ in range(4)] for _ in sides]
    want = []
    for s, us in zip(sides, draws):
        want.append([])
        for u in us:
            s.u.copy_(u)
            s.run()
            want[-1].append(s.outcome())
    graphs = []
    torch.cuda.synchronize()
    for s in sides:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s.run()
        graphs.append(graph)
    for s in sides:
        s.rewind()
    for i in range(4):
        for s, graph, us, w in zip(sides, graphs, draws, want):
            s.u.copy_(us[i])
            graph.replay()
            if i % 2:
                torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(s.outcome(), w[i]))
            # (and a call of other sizes with these workspaces)
            nvq.sample(s.logits[:1, :777], s.u[:1], workspace=s.ws[2])
            nvq.attention(s.cache, s.q[:1, :2 * s.heads], s.table[:1], s.lengths[:1], workspace=s.ws[1])


@gpu
def test_two_streams_at_once():
    sides = [(Step(60, 4), torch.cuda.Stream()), (Step(61, 9, True), torch.cuda.Stream())]
    for s, _ in sides:
        s.u.fill_(0.6)
    want = []
    for s, _ in sides:
        s.run()
        want.append(s.outcome())
        s.rewind()
    torch.cuda.synchronize()
    for _ in range(10):
        for s, stream in sides:
            with torch.cuda.stream(stream):
                s.rewind()
                s.run()
    torch.cuda.synchronize()
    for (s, _), w in zip(sides, want):
        assert all(torch.equal(a, b) for a, b in zip(s.outcome(), w))


@gpu
def test_both_ways_into_the_library_agree(monkeypatch):
    s = Step(70, 3)
    s.u.fill_(0.3)
    s.run()
    want = s.outcome()
    k, v = nvq.cache_read(s.cache, s.table, s.at - 1, out=(torch.empty_like(s.q[:, :2]), torch.empty_like(s.q[:, :2])))
    s.rewind()
    monkeypatch.setattr(nvq, "_calls", None)
    s.run()
    assert all(torch.equal(a, b) for a, b in zip(s.outcome(), want))
    assert all(torch.equal(a, b) for a, b in zip(nvq.cache_read(s.cache, s.table, s.at - 1), (k, v)))


@gpu
@pytest.mark.parametrize("fast", [True, False])
def test_a_window_beyond_the_library_s_numbers_is_refused(fast, monkeypatch):
    s = Step(71, 2)
    if not fast:
        monkeypatch.setattr(nvq, "_calls", None)
    for window in (1 << 31, 1 << 32):
        with pytest.raises(ValueError, match="window is out of range"):
            nvq.attention(s.cache, s.q, s.table, s.lengths, window=window, out=s.y, workspace=s.ws[1])
    with pytest.raises(nvq.NvqError):
        nvq.attention(s.cache, s.q, s.table, s.lengths, window=-1, out=s.y, workspace=s.ws[1])


@gpu
def test_tensors_of_another_device_than_the_current_one(monkeypatch):
    s = Step(72, 2)
    calls = [lambda: nvq.adapters_add(s.adapters, s.x, s.who, s.p, out=s.p, workspace=s.ws[0]),
             lambda: nvq.cache_append(s.cache, s.table, s.at, s.q[:, :2], s.q[:, :2]),
             lambda: nvq.cache_read(s.cache, s.table, s.at, out=(s.q[:, :2].contiguous(), s.q[:, :2].contiguous())),
             lambda: nvq.attention(s.cache, s.q, s.table, s.lengths, out=s.y, workspace=s.ws[1]),
             lambda: nvq.sample(s.logits, s.u, out=s.ids, workspace=s.ws[2])]
    for handle in (s.adapters, s.cache):
        monkeypatch.setattr(handle, "device", torch.device("cuda", 1))
        monkeypatch.setattr(handle, "index", 1)
    for call in calls[:4]:
        with pytest.raises(ValueError, match="current device"):
            call()
    monkeypatch.undo()
    monkeypatch.setattr(nvq, "_calls", None)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    for call in calls:
        with pytest.raises(ValueError, match="current device"):
            call()


# ---- sizes at their ends ----
@gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.uint8])
def test_a_cache_whose_places_pass_32_bits(dtype):
    """Pages beyond 2^32 elements, 40 tokens over the borders of the first and the last."""
    heads, D, page, pages = 8, 128, 1024, 4100
    assert (pages - 1) * heads * D * page > 1 << 32
    rng = np.random.default_rng(1)
    cache = nvq.Cache.empty(pages, heads, page, D, dtype, DEV)
    table = np.array([[pages - 1, 0, pages - 2]], np.int32)
    n, first = 1100, 1000
    pool = Pool(rng, [n], heads, D, page, dtype == torch.uint8, room=page)
    pool.table[:, :3] = np.arange(3)
    k, v = bf16(rng, (n, heads, D)), bf16(rng, (n, heads, D))
    pool.put(0, np.arange(n), k, v)
    zero, at = torch.zeros(n, dtype=torch.int32, device=DEV), torch.arange(n, dtype=torch.int32, device=DEV)
    nvq.cache_append(cache, dev(table), at, dev(k, torch.bfloat16), dev(v, torch.bfloat16), sequences=zero)
    got = nvq.cache_read(cache, dev(table), at[first:], zero[first:])
    held = lambda x: np.stack([x[t // page, :, t % page] for t in range(first, n)])
    assert same_bits(got[0], held(pool.k)) and same_bits(got[1], held(pool.v))
    q = bf16(rng, (1, 16, D))
    y = nvq.attention(cache, dev(q, torch.bfloat16), dev(table), torch.tensor([n], dtype=torch.int32, device=DEV), out_dtype=torch.float32)
    check_attention(f64(y), None, pool, q, [n], 0, 0.0, D ** -0.5, 0.0)


@gpu
@pytest.mark.parametrize("n,H,heads,D", [(140000, 1, 1, 32), (30000, 6, 2, 64), (140000, 4, 1, 256)])
def test_attention_of_a_sequence_shared_by_many_workgroups(n, H, heads, D):
    rng = np.random.default_rng(n + D)
    pool = Pool(rng, [n], heads, D, 1024, False)
    pool.put(0, np.arange(n), bf16(rng, (n, heads, D)), bf16(rng, (n, heads, D)))
    q = bf16(rng, (1, H, D))
    lse = torch.empty((1, H), dtype=torch.float32, device=DEV)
    y = nvq.attention(pool.device(), dev(q, torch.bfloat16), dev(pool.table), torch.tensor([n], dtype=torch.int32, device=DEV),
                      out_dtype=torch.float32, lse=lse)
    check_attention(f64(y), f64(lse), pool, q, [n], 0, 0.0, D ** -0.5, 0.0)


@gpu
def test_attention_of_as_many_sequences_as_it_takes():
    """4096 sequences of sixteen heads to a key head: all the memory that a workgroup has."""
    rng = np.random.default_rng(2)
    B, H, D, page = 4096, 16, 128, 8
    lengths = rng.integers(0, 40, B)
    lengths[[0, 4095]] = 0, 300
    pool = Pool(rng, lengths, 1, D, page, False)
    for b, n in enumerate(lengths):
        pool.put(b, np.arange(n), bf16(rng, (n, 1, D)), bf16(rng, (n, 1, D)))
    q = bf16(rng, (B, H, D))
    y = nvq.attention(pool.device(), dev(q, torch.bfloat16), dev(pool.table), dev(lengths.astype(np.int32)), out_dtype=torch.float32)
    check_attention(f64(y), None, pool, q, lengths, 0, 0.0, D ** -0.5, 0.0)


@gpu
@pytest.mark.parametrize("times", [8, 60])
def test_a_token_read_twice_and_pages_that_sequences_share(times):
    rng = np.random.default_rng(3)
    n, heads, D, page = 40, 2, 64, 16
    pool = Pool(rng, [n, n], heads, D, page, False)
    pool.table[1, :2] = pool.table[0, :2]  # the same beginning
    k, v = bf16(rng, (n, heads, D)), bf16(rng, (n, heads, D))
    pool.put(0, np.arange(n), k, v)
    pool.put(1, np.arange(32, n), ref.to_bf16((k[32:] + 1.0).astype(np.float32)).astype(np.float64), v[32:])
    cache, table = pool.device(), dev(pool.table)
    at, of = np.array([5, 5, 6, 7, 6, 0, 39, 38, 39, 31, 32, 33] * times, np.int32), np.array([0, 1, 1, 1, 0, 0, 0, 0, 0, 1, 1, 1] * times, np.int32)
    got = nvq.cache_read(cache, table, dev(at), dev(of))
    page_of = pool.table[of, at // page]
    assert same_bits(got[0], pool.k[page_of, :, at % page]) and same_bits(got[1], pool.v[page_of, :, at % page])
    q = bf16(rng, (2, 4, D))
    y = nvq.attention(cache, dev(q, torch.bfloat16), table, torch.tensor([n, n], dtype=torch.int32, device=DEV), out_dtype=torch.float32)
    check_attention(f64(y), None, pool, q, [n, n], 0, 0.0, D ** -0.5, 0.0)


@gpu
def test_rows_of_logits_beyond_32_bits():
    M, V, ld = 4, 4500, (1 << 30) + 64
    rng = np.random.default_rng(4)
    logits = torch.empty((M, ld), dtype=torch.bfloat16, device=DEV)[:, :V]
    x = torch.from_numpy(rng.standard_normal((M, V)).astype(np.float32) * 3).bfloat16()
    logits.copy_(x)
    u = rng.random(M).astype(np.float32)
    assert nvq.sample(logits, dev(u)).tolist() == [int(ref.sample(x[m].double().numpy(), float(u[m]))) for m in range(M)]


@gpu
def test_adapters_beyond_32_bits():
    """Weights of the last of three adapters behind 2^32 elements, results behind 2^31 bytes."""
    n, N, K, R, M = 3, 1 << 23, 32, 256, 70
    b = torch.zeros((n, N, R), dtype=torch.bfloat16, device=DEV)
    a = torch.zeros((n, R, K), dtype=torch.bfloat16, device=DEV)
    a[2], b[2, N - 2] = 1.0, 1.0
    b[2, 5, 7] = 2.0
    x, y = torch.ones((M, K), dtype=torch.bfloat16, device=DEV), torch.ones((M, N), dtype=torch.bfloat16, device=DEV)
    ids = torch.full((M,), 2, dtype=torch.int32, device=DEV)
    ids[3] = -1
    got = nvq.adapters_add(nvq.Adapters(a, b), x, ids, y, out=y)
    want = torch.ones(N, dtype=torch.bfloat16, device=DEV)
    want[N - 2], want[5] = 1 + 256 * 32, 1 + 2 * 32  # (8193 is 8192 in bf16)
    for m in range(M):
        assert torch.equal(got[m], want) if m != 3 else bool((got[m] == 1).all())

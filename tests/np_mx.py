"""Plain 64-bit forms of the microscaled 4-bit format and of the mixture-of-experts layer (numpy), for
tests: written from the definitions, without the package's code."""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
VALUES = np.concatenate([GRID, -GRID])
EPS32 = 2.0 ** -24  # half a step of fp32, relative
EPS16 = 2.0 ** -8   # of bf16


def quant(x):
    """x float64 [M,K] -> q uint8 [M,K/2], scales uint8 [M,K/32]."""
    M, K = x.shape
    v = x.reshape(M, K // 32, 32)
    mag = np.abs(v)
    top = mag.max(-1)
    bad = ~np.isfinite(top)
    e = np.frexp(np.where(bad, 1.0, top))[1] - 1  # floor(log2)
    byte = np.where(top == 0, 0, np.clip(e + 125, 0, 254))
    with np.errstate(invalid="ignore", over="ignore"):
        a = mag / 2.0 ** (byte - 127.0)[..., None]
        far = np.abs(a[..., None] - GRID)
    near = far.min(-1, keepdims=True) == far
    code = near.argmax(-1)                       # the lower of two as near
    tie = near.sum(-1) == 2
    code = np.where(tie & (code % 2 == 1), code + 1, code)
    code = np.where(a >= 6.0, 7, code)
    code = code + 8 * np.signbit(v)
    code[bad] = 0
    code = code.reshape(M, K).astype(np.uint8)
    return code[:, 0::2] | (code[:, 1::2] << 4), np.where(bad, 255, byte).astype(np.uint8)


def dequant(q, s):
    """-> float64 [..., K] (scale byte 255: NaN)."""
    v = np.empty(q.shape[:-1] + (q.shape[-1] * 2,))
    v[..., 0::2] = VALUES[q & 15]
    v[..., 1::2] = VALUES[q >> 4]
    scale = np.where(s == 255, np.nan, 2.0 ** (s.astype(np.float64) - 127.0))
    return v * np.repeat(scale, 32, -1)


def dequant_int4(q, s):
    """int4 codes in groups of 32 (inputs j and 16 + j in byte j), fp16 scales given as their bits."""
    g = q.reshape(q.shape[:-1] + (-1, 16))
    c = np.concatenate([g & 15, g >> 4], -1).astype(np.float64) - 8.0
    return (c * s.view(np.float16).astype(np.float64)[..., None]).reshape(q.shape[:-1] + (-1,))


def random_mx(rng, rows, K, spread=3, middle=121):
    """Random codes, scale bytes middle .. middle + spread."""
    return (rng.integers(0, 256, (rows, K // 2), dtype=np.uint8),
            rng.integers(middle, middle + spread + 1, (rows, K // 32), dtype=np.uint8))


def best(logits, k):
    """ids of the k largest, descending, the lowest index first among equals (NaN last)."""
    key = np.where(np.isnan(logits), -np.inf, logits)
    return np.argsort(-key, axis=1, kind="stable")[:, :k]


def silu(g):
    return g / (1.0 + np.exp(-g))


def experts(x, gate_up, down, ids, weights):
    """x [M,K], gate_up [E,2F,K], down [E,K,F], ids, weights [M,k] (all float64 but ids) -> y [M,K] and a bound on
    what fp32 sums in any order, approximations good to a few units of fp32 in silu, and one rounding of h to
    bf16 can differ from it (before y's own rounding)."""
    M, K = x.shape
    E, F = gate_up.shape[0], down.shape[2]
    y, tol = np.zeros((M, K)), np.zeros((M, K))
    for m in range(M):
        for e, w in zip(ids[m], weights[m]):
            if not 0 <= e < E:
                continue
            gu = gate_up[e] @ x[m]
            d_gu = (K + 40) * EPS32 * (np.abs(gate_up[e]) @ np.abs(x[m]))
            g, u, dg, du = gu[:F], gu[F:], d_gu[:F], d_gu[F:]
            h = silu(g) * u
            # |silu'| < 1.1; exp2, its argument, the reciprocal and two products: below (8 + 2 |g|) units
            dh = 1.1 * dg * (np.abs(u) + du) + np.abs(silu(g)) * du + np.abs(h) * (8 + 2 * np.abs(g)) * 2 * EPS32
            dh = dh + EPS16 * (np.abs(h) + dh)
            y[m] += w * (down[e] @ h)
            # products with h, the weight and the sums over waves and slots
            tol[m] += abs(w) * (np.abs(down[e]) @ dh + (F + 64) * EPS32 * (np.abs(down[e]) @ (np.abs(h) + dh)))
    return y, tol

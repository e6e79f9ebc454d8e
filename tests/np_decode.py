"""Plain forms, in 64 bits where numbers are computed, of the paged cache, attention over it, sampling and adapters
(numpy), for tests: written from the definitions, without the package's code."""
import numpy as np

EPS32 = 2.0 ** -24  # half a step of fp32, relative
EPS16 = 2.0 ** -8   # of bf16

_E4M3 = np.array([c % 8 * 2.0 ** -9 if c < 8 else (1 + c % 8 / 8) * 2.0 ** (c // 8 - 7) for c in range(127)])
E4M3 = np.concatenate([_E4M3, [np.nan], -_E4M3, [np.nan]])  # value of each code


def to_bf16(x):
    """float32 -> the nearest bf16 values, ties to even, as float32 (finite values)."""
    b = np.ascontiguousarray(x, np.float32).view(np.uint32)
    return ((b + 0x7fff + (b >> 16 & 1)) & np.uint32(0xffff0000)).view(np.float32)


def rotate(x, cos_sin, positions, interleaved):
    """float32 [T,H,D] -> float32, every product and sum rounded to binary32, then to bf16."""
    rot = cos_sin.shape[1]
    x = x.astype(np.float32).copy()
    c, s = (cos_sin[positions][:, None, i * rot // 2:(i + 1) * rot // 2].astype(np.float32) for i in (0, 1))
    at = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b = x[..., at[0]].copy(), x[..., at[1]].copy()
    with np.errstate(all="ignore"):
        x[..., at[0]], x[..., at[1]] = a * c - b * s, b * c + a * s
    return to_bf16(x)


def quant_e4m3(x):
    """float64 [..., D] (finite) -> codes u8, scale bytes u8 [...]."""
    top = np.abs(x).max(-1)
    byte = np.ones(top.shape, np.int64)
    for b in range(1, 255):  # the smallest power of two that does
        byte = np.where((top <= 448 * 2.0 ** (byte - 127.0)), byte, np.minimum(byte + 1, 254))
    v = np.abs(x) / 2.0 ** (byte - 127.0)[..., None]
    up = np.clip(np.searchsorted(_E4M3, v), 0, 126)
    lo = np.maximum(up - 1, 0)
    du, dl = _E4M3[up] - v, v - _E4M3[lo]
    code = np.where((du < dl) | ((du == dl) & (up % 2 == 0)), up, lo)
    code = np.where(_E4M3[up] == v, up, code)
    return (code + 128 * np.signbit(x)).astype(np.uint8), byte.astype(np.uint8)


def scale_of(byte):
    return np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127))


def attention(q, k, v, scale, softcap):
    """q [g,D], k, v [n,D] of one sequence and key head -> out [g,D], log of the sum of exp [g], and what the errors of
    a computation are measured by: the largest sum of |q||k| and |score|, the mean |v| under the weights."""
    s = scale * (q @ k.T)
    size = abs(scale) * (np.abs(q) @ np.abs(k).T).max(1)
    if softcap:
        s = softcap * np.tanh(s / softcap)
    m = s.max(1, keepdims=True)
    p = np.exp(s - m)
    l = p.sum(1, keepdims=True)
    return p @ v / l, (m + np.log(l))[:, 0], size, (m - s.min(1, keepdims=True))[:, 0], p @ np.abs(v) / l


def sample(logits, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One row (float64): the id."""
    live = np.flatnonzero(logits > -np.inf)  # (not NaN either)
    if len(live) == 0:
        return -1
    order = live[np.argsort(-logits[live], kind="stable")]
    if not temperature > 0 or np.isinf(logits[order[0]]):
        return order[0]
    if top_k > 0:
        order = order[:top_k]
    w = np.exp((logits[order] - logits[order[0]]) / temperature)
    upto = np.cumsum(w)
    n = len(order)
    if not top_p >= 1:
        n = 1 + int((upto[:-1] < max(top_p, 0) * upto[-1]).sum())
    if min_p > 0:
        n = min(n, max(1, int((w >= min_p).sum())))
    u = u if u > 0 else 0.0
    last = max(1, int((w[:n] >= 2.0 ** -44).sum())) - 1  # (smaller weights count for nothing: such a token is never chosen)
    return order[min(last, int((upto[:n] <= u * upto[n - 1]).sum()))]

"""Plain 64-bit statements of the long-context serving operators, written from
include/mlkv.h independently of the binding and the kernels: the 4-bit cache's
values and layout, attention over any set of positions with its rounding bound,
norm and rotation."""
import numpy as np

import synth
from gpu_util import U, softmax_rounding_bound

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def f64(bits):
    return synth.bf16_to_f32(bits).astype(np.float64)


# ------------------------------------------------------------- 4-bit cache ---

def quantise(bits: np.ndarray):
    """bf16 patterns [..., D] -> (codes [..., D], exponent bytes [..., D/32])."""
    x = f64(bits)
    blocks = x.reshape(*x.shape[:-1], -1, 32)
    top = np.abs(blocks).max(axis=-1)
    odd = ~np.isfinite(top)
    safe = np.where(odd | (top == 0), 1.0, top)
    e = np.floor(np.log2(safe)).astype(np.int64) - 3
    for _ in range(3):  # the least e with top < 7 * 2^e
        e = np.where(safe >= 7 * 2.0 ** e, e + 1, e)
    e = np.where(top == 0, -124, np.clip(e, -124, 125))
    y = np.where(odd[..., None], 0.0, blocks) / 2.0 ** e[..., None].astype(np.float64)
    mag = np.abs(y)
    # Nearest of the grid; a tie goes to the even place.
    dist = np.abs(mag[..., None] - GRID)
    near = dist.min(axis=-1, keepdims=True)
    tied = dist == near
    even = tied & (np.arange(8) % 2 == 0)
    place = np.where(even.any(axis=-1), even.argmax(axis=-1), tied.argmax(axis=-1))
    sign = (bits.reshape(blocks.shape) >> 15).astype(np.int64)
    codes = np.where(odd[..., None], 0, place | (sign << 3)).astype(np.uint8)
    exps = np.where(odd, 255, e + 127).astype(np.uint8)
    return codes.reshape(x.shape), exps


def values(codes: np.ndarray, exps: np.ndarray) -> np.ndarray:
    """What codes and exponent bytes stand for, float64 [..., D]."""
    v = GRID[codes & 7] * np.where(codes & 8, -1.0, 1.0)
    scale = np.where(exps == 255, np.nan, 2.0 ** (exps.astype(np.float64) - 127))
    return v * np.repeat(scale, 32, axis=-1)


def held(bits: np.ndarray) -> np.ndarray:
    return values(*quantise(bits))


def places(D: int):
    """Byte offsets inside a record, for token u and channel d: (key byte, key
    nibble, value byte, value nibble) [32][D], (key exponent, value exponent)
    [32][D/32]."""
    K = D // 32
    u, d = np.meshgrid(np.arange(32), np.arange(D), indexing="ij")
    i = ((u >> 2) & 1) * K + (d >> 5)
    lane = ((d >> 3) & 3) * 16 + ((u >> 3) << 2) + (u & 3)
    kb = (i >> 2) * 1024 + lane * 16 + (i & 3) * 4 + ((d & 7) >> 1)
    j = d >> 4
    lane = (u >> 3) * 16 + (d & 15)
    vb = 16 * D + (j >> 2) * 1024 + lane * 16 + (j & 3) * 4 + ((u & 7) >> 1)
    u, b = np.meshgrid(np.arange(32), np.arange(K), indexing="ij")
    ke = 32 * D + (((u >> 3) << 2) + (u & 3)) * 2 * K + ((u >> 2) & 1) * K + b
    ve = 33 * D + (u >> 3) * 8 * K + b * 8 + (u & 7)
    u, d = np.meshgrid(np.arange(32), np.arange(D), indexing="ij")
    return kb, d & 1, vb, u & 1, ke, ve


def store(data: np.ndarray, kv: int, b: int, start: int, k_bits: np.ndarray, v_bits: np.ndarray):
    """Rows [T][D] to slots start .. of data [n_kv][B][S/32][34 D], in place."""
    D = data.shape[-1] // 34
    S = data.shape[2] * 32
    kb, kn, vb, vn, ke, ve = places(D)
    ck, ek = quantise(k_bits)
    cv, ev = quantise(v_bits)
    for t in range(k_bits.shape[0]):
        slot = start + t
        if not 0 <= slot < S:
            continue
        rec, u = data[kv, b, slot // 32], slot % 32
        for codes, byte, nib, exps, eb in ((ck, kb, kn, ek, ke), (cv, vb, vn, ev, ve)):
            for n in (0, 1):  # the two nibbles of a byte, one after the other
                sel = nib[u] == n
                at = byte[u][sel]
                keep = 0xF0 if n == 0 else 0x0F
                rec[at] = (rec[at] & keep) | (codes[t][sel] << (4 * n))
            rec[eb[u]] = exps[t]


def load(data: np.ndarray):
    """data -> the values held, (k, v) float64 [n_kv][B][S][D]."""
    n_kv, B, tiles, record = data.shape
    D = record // 34
    kb, kn, vb, vn, ke, ve = places(D)
    out = []
    for byte, nib, eb in ((kb, kn, ke), (vb, vn, ve)):
        codes = (data[..., byte] >> (4 * nib)) & 15
        out.append(values(codes, data[..., eb]).reshape(n_kv, B, tiles * 32, D))
    return out


# --------------------------------------------------------------- attention ---

def attended(n: int, window: int, sinks: int) -> np.ndarray:
    """Positions a query at position n attends (none for n < 0)."""
    p = np.arange(n + 1)
    return p if window == 0 else p[(p < sinks) | (p > n - window)]


def attend(q: np.ndarray, K: np.ndarray, V: np.ndarray, at: np.ndarray):
    """Rows q [r][D] over the positions `at` of K, V [S][D] (float64): the
    exact outputs and the bound of what bf16 weights and fp32 sums may be off."""
    if at.size == 0:
        return np.zeros(q.shape), np.zeros(q.shape)
    k, v = K[at], V[at]
    s = q @ k.T / np.sqrt(q.shape[1])
    w = np.exp(s - s.max(axis=1, keepdims=True))
    ref = (w / w.sum(axis=1, keepdims=True)) @ v
    return ref, softmax_rounding_bound(q, k, v, ref, np.full(q.shape[0], at.size))


# ------------------------------------------------------- norm and rotation ---

def norm_rope(bits: np.ndarray, weight, eps: float, dims: int, base: float, pos: np.ndarray):
    """bf16 rows [..., heads][D] at pos [...] -> (exact, bound on the rounded
    result): half a bf16 step of the result (2^-8 of it), and of the two
    numbers it is made of at most (D + 40) half steps of fp32: the sum of D
    squares (D / 2 of its root), its root and quotient (3), three products, the
    angle's fraction of a turn (2 pi half steps of a number up to 1/2), sine and
    cosine (4 each) and the rotation's products and sum."""
    x = f64(bits)
    D = x.shape[-1]
    if weight is not None:
        x = x * f64(weight) / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps)
    out, parts = x.copy(), np.abs(x)
    if dims:
        half = dims // 2
        angle = pos[..., None, None] * base ** (-2.0 * np.arange(half) / dims)
        c, s = np.cos(angle), np.sin(angle)
        lo, hi = x[..., :half], x[..., half:dims]
        out[..., :half], out[..., half:dims] = lo * c - hi * s, hi * c + lo * s
        both = np.abs(lo) + np.abs(hi)
        parts[..., :half] = parts[..., half:dims] = both
    return out, 2.0 ** -8 * np.abs(out) + U * (D + 40) * parts

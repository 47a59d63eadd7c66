"""CPU oracle of the 4-bit K/V cache: the format by its definition, in fp64 (numpy only, slow and plain)."""
from __future__ import annotations

import numpy as np

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
MAX_SCALE, MAX_VALUE = 10240.0, 61440.0


def scale_values() -> np.ndarray:
    """The 256 unsigned 8-bit floats: 5 exponent bits (bias 15), 3 mantissa bits; exponent 0 is subnormal."""
    out = []
    for c in range(256):
        e, m = c >> 3, c & 7
        out.append(m / 8 * 2.0 ** -14 if e == 0 else (1 + m / 8) * 2.0 ** (e - 15))
    return np.array(out)


SCALES = scale_values()
N_SCALES = int(np.searchsorted(SCALES, MAX_SCALE)) + 1     # codes that are written


def nearest(x: np.ndarray, grid: np.ndarray) -> np.ndarray:
    """Index of the grid value next to x >= 0 (saturating); halfway between two, the even index."""
    hi = np.minimum(np.searchsorted(grid, x), len(grid) - 1)
    lo = np.maximum(hi - 1, 0)
    up, down = grid[hi] - x, x - grid[lo]
    return np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)


def encode(x: np.ndarray):
    """x [..., 128] (fp64 values of bf16 numbers) -> code of every channel [..., 128] (0 .. 15), scale codes [..., 8]."""
    x = np.where(np.isnan(x), 0.0, np.clip(x, -MAX_VALUE, MAX_VALUE)).reshape(*x.shape[:-1], 8, 16)
    s = nearest(np.abs(x).max(-1) / 6.0, SCALES[:N_SCALES])
    v = SCALES[s][..., None]
    ratio = np.divide(np.abs(x), v, out=np.zeros_like(x), where=v > 0)
    code = nearest(ratio, E2M1) + 8 * (x < 0)
    return code.reshape(*x.shape[:-2], 128).astype(np.uint8), s.astype(np.uint8)


def decode(code: np.ndarray, s: np.ndarray) -> np.ndarray:
    """Codes [..., 128] and scale codes [..., 8] -> fp64 values [..., 128]."""
    v = E2M1[code & 7] * np.where(code & 8, -1.0, 1.0)
    return (v.reshape(*v.shape[:-1], 8, 16) * SCALES[s][..., None]).reshape(v.shape)


def pack(code: np.ndarray) -> np.ndarray:
    """Two channels a byte, the even one in the low half: [..., 128] -> [..., 64]."""
    return (code[..., 0::2] | (code[..., 1::2] << 4)).astype(np.uint8)


def unpack(packed: np.ndarray) -> np.ndarray:
    return np.stack([packed & 15, packed >> 4], -1).reshape(*packed.shape[:-1], 128)


def attention(q: np.ndarray, k: np.ndarray, v: np.ndarray, sm_scale: float):
    """One query [128] over keys [n, 128]: output, natural-log-sum-exp, sum p |v| and the largest sum |q k| sm_scale (the
    last two for error bounds)."""
    if len(k) == 0:
        return np.zeros(128), -np.inf, np.zeros(128), 0.0
    z = k @ q * sm_scale
    m = z.max()
    e = np.exp(z - m)
    p = e / e.sum()
    return p @ v, m + np.log(e.sum()), p @ np.abs(v), float((np.abs(k) @ np.abs(q)).max() * sm_scale)

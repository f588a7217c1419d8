"""Oracle of the AdamW step and its 8-bit states -- TEST INFRASTRUCTURE ONLY.

Only `tests/` may import this module.  Plain numpy.  `step` is the definition in float64; `Codes8` restates the storage
of 8-bit states (blocks of 256, e4m3 codes, a power of two for a scale, random rounding by a hash) in integer and exact
arithmetic, element by element tables instead of bit tricks.
"""
from __future__ import annotations

from typing import Tuple

import numpy as np

BLOCK = 256


def step(w, m, v, g, *, lr: float, beta1: float, beta2: float, eps: float, weight_decay: float, t: int):
    """One step with decoupled weight decay, t = 1 for the first; returns (w, m, v)."""
    w, m, v, g = (np.asarray(a, np.float64) for a in (w, m, v, g))
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    w = w * (1 - lr * weight_decay) - lr * (m / (1 - beta1 ** t)) / (np.sqrt(v / (1 - beta2 ** t)) + eps)
    return w, m, v


def moments_f32(m, v, g, beta1: float, beta2: float):
    """The moments in fp32, every product and sum rounded, as the library states it."""
    f = np.float32
    m, v, g = (np.asarray(a, f) for a in (m, v, g))
    return m * f(beta1) + g * f(1 - beta1), v * f(beta2) + (g * g) * f(1 - beta2)


def _code_values() -> np.ndarray:
    """The 127 magnitudes of e4m3 (exponents 1..15 with bias 7 and three bits below, the gradual ones underneath)."""
    out = [c / 512 for c in range(8)]
    out += [(8 + c) / 8 * 2.0 ** (e - 7) for e in range(1, 16) for c in range(8)]
    return np.array(out[:127])                                     # the last pattern is not a number


VALUES = _code_values()


def decode(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """Values of the codes [n], fp64; scales [ceil(n / BLOCK)]."""
    codes = np.asarray(codes, np.uint8)
    v = np.where(codes & 0x80, -1.0, 1.0) * VALUES[codes & 0x7f]
    return v * np.repeat(np.asarray(scales, np.float64), BLOCK)[:len(v)]


def mix(x: np.ndarray) -> np.ndarray:
    x = np.asarray(x, np.uint64) & np.uint64(0xffffffff)
    for mult, shift in ((0x6A09E667, 16), (0xBB67AE85, 15)):
        x = ((x ^ (x >> np.uint64(shift))) * np.uint64(mult)) & np.uint64(0xffffffff)
    return x ^ (x >> np.uint64(16))


def random_words(seed: int, t: int, first_block: int, n: int) -> np.ndarray:
    """32 random bits for each of n weights of a tensor whose first block of the plan is first_block, at step t."""
    key = mix(np.array([(seed + t * 0x9E3779B9) & 0xffffffff]))[0]
    return mix(np.arange(n, dtype=np.uint64) + np.uint64(first_block * BLOCK) + key)


def scales_of(x: np.ndarray) -> np.ndarray:
    """The power of two of each block of magnitudes x that brings its largest into (224, 448]; 0 for a block of zeros."""
    x = np.abs(np.asarray(x, np.float64))
    most = np.array([x[i:i + BLOCK].max() for i in range(0, len(x), BLOCK)])
    out = np.zeros(len(most))
    some = most > 0
    k = np.floor(np.log2(np.where(some, most, 1.0)))
    k = np.where(most > 1.75 * 2.0 ** k, k + 1, k)
    k = np.where(most <= 1.75 * 2.0 ** (k - 1), k - 1, k)          # (log2 of a power of two may round either way)
    out[some] = 2.0 ** (k[some] - 8)
    return out


def encode(x: np.ndarray, scales: np.ndarray, r: np.ndarray) -> np.ndarray:
    """Codes of x: the magnitude lies between two codes, the upper one is taken where r < 2^20 says so."""
    x = np.asarray(x, np.float64)
    s = np.repeat(np.asarray(scales, np.float64), BLOCK)[:len(x)]
    y = np.minimum(np.abs(x) / np.where(s > 0, s, 1.0), 448.0)
    low = np.searchsorted(VALUES, y, side="right") - 1
    high = np.minimum(low + 1, len(VALUES) - 1)
    gap = np.where(high > low, VALUES[high] - VALUES[low], 1.0)
    share = np.rint((y - VALUES[low]) / gap * 2.0 ** 20)           # the float's bits below the code's
    up = share + np.asarray(r, np.float64) >= 2.0 ** 20
    code = np.where(up, high, low)
    return (code | np.where(x < 0, 0x80, 0)).astype(np.uint8)


def states8(m: np.ndarray, v: np.ndarray, words: np.ndarray) -> Tuple[np.ndarray, np.ndarray, np.ndarray, np.ndarray]:
    """(codes of m, codes of sqrt v, scales of m, scales of sqrt v)."""
    u = np.sqrt(np.asarray(v, np.float64))
    ms, us = scales_of(m), scales_of(u)
    words = np.asarray(words, np.uint64)
    mc = encode(m, ms, words >> np.uint64(12))
    uc = encode(u, us, words & np.uint64(0xfffff))
    return mc, np.where((np.asarray(v) > 0) & (uc == 0), 1, uc).astype(np.uint8), ms, us

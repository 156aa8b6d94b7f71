"""Plain CPU oracle of caches held in 8 bits: scales and codes of a block, their values, attention over them.

TEST INFRASTRUCTURE ONLY (see pced_oracle). NumPy and the plain definitions, one block at a time. The
roundings that are part of the definition (a scale in bf16, a product in fp32) are done in fp32; all else is
float64.
"""
from __future__ import annotations

import math

import numpy as np

PAGE = 16
LARGEST = {"e4m3": 448.0, "int8": 127.0}


def e4m3_values() -> np.ndarray:
    """The value of every byte as a float of 4 exponent bits (bias 7) and 3 of the significand, without infinities;
    0x7F and 0xFF are NaN."""
    out = np.zeros(256)
    for b in range(256):
        e, m = b >> 3 & 15, b & 7
        x = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        out[b] = (math.nan if b & 127 == 127 else x) * (-1.0 if b & 128 else 1.0)
    return out


E4M3 = e4m3_values()


def scale_of(x: np.ndarray, code: str) -> np.float32:
    """A block's scale."""
    a = np.abs(np.asarray(x, dtype=np.float32))
    top = np.float32(min(max(float(np.where(np.isnan(a), 0, a).max()), 2.0 ** -100), 2.0 ** 127))
    t = np.float32(top / np.float32(LARGEST[code]))
    s = np.array([t]).view(np.uint32)[0]
    return np.array([(int(s) + 0xFFFF) >> 16 << 16], dtype=np.uint32).view(np.float32)[0]


def encode(x: np.ndarray, code: str):
    """(bytes of the block's values, scale); x any shape, values of bf16."""
    x = np.asarray(x, dtype=np.float32)
    s = scale_of(x, code)
    with np.errstate(invalid="ignore", over="ignore"):
        y = (x * np.float32(np.float32(1) / s)).astype(np.float64)
    y = np.where(np.isnan(x), 0.0, np.clip(y, -LARGEST[code], LARGEST[code]))
    if code == "int8":
        return np.rint(y).astype(np.int8).view(np.uint8), s
    up = E4M3[:127]  # the values from 0 on, ascending
    a = np.abs(y)
    hi = np.searchsorted(up, a)  # the first value not below
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - up[lo], up[hi] - a
    b = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    return (b | np.where(np.signbit(y), 128, 0)).astype(np.uint8), s


def decode(b: np.ndarray, s, code: str) -> np.ndarray:
    """The values of a block's bytes."""
    v = E4M3[b] if code == "e4m3" else b.view(np.int8).astype(np.float64)
    return v * float(s)


def held(rows: np.ndarray, complete: int, code: str) -> np.ndarray:
    """rows [tokens][Hkv][D] as a cache in 8 bits holds them: the first `complete` tokens (whole pages) by codes."""
    out = np.array(rows, dtype=np.float64)
    for p in range(complete // PAGE):
        for h in range(out.shape[1]):
            at = (slice(PAGE * p, PAGE * (p + 1)), h)
            b, s = encode(out[at], code)
            out[at] = decode(b, s, code)
    return out


def attend(q: np.ndarray, k: np.ndarray, v: np.ndarray) -> np.ndarray:
    """q [G][D], k and v [tokens][D]: softmax(q k^T / sqrt(D)) v."""
    z = q @ k.T / math.sqrt(q.shape[1])
    w = np.exp(z - z.max(1, keepdims=True))
    return w @ v / w.sum(1, keepdims=True)

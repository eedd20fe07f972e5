"""CPU oracle: the 4-bit KV cache's number format and page layout.  TEST INFRASTRUCTURE ONLY.

E2M1 as the OCP microscaling formats specification defines it: 1 sign bit, 2 exponent bits with bias 1, 1 mantissa bit;
exponent field 0 holds 0 and 0.5; no infinities, no NaN; the largest value is 6.  32 consecutive head dims of one token share
a scale 2^(byte - 127); byte 255 makes all of them NaN.

Encoding picks the scale 2^(e - 2) for a largest absolute value in [1, 1.75] 2^e and 2^(e - 1) above that, within 2^-125 ..
2^125, and rounds x / scale to the nearest value, ties to the even code, saturating at +-6.

Layout of one page (block_size slots of head_dim elements), written out element by element:
  K  code of (slot, d) in byte ((d // 32) * bs + slot) * 16 + (d % 32) // 2, scale in byte bs * D // 2 + slot * (D // 32) + d // 32
  V  code in byte ((slot // 8) * (D // 4) + d // 4) * 16 + (slot % 8) * 2 + (d % 4) // 2, scale in bs * D // 2 + (d // 32) * bs + slot
with the even head dim's code in the byte's low half.
"""
from __future__ import annotations

import math

import numpy as np

BLOCK = 32


def decode_one(code: int) -> float:
    sign = -1.0 if code & 8 else 1.0
    e, m = (code >> 1) & 3, code & 1
    return sign * (m * 0.5 if e == 0 else (1.0 + m / 2.0) * 2.0 ** (e - 1))


TABLE = np.array([decode_one(c) for c in range(16)], np.float64)


def scale_value(byte: int) -> float:
    return float("nan") if byte == 255 else 2.0 ** (int(byte) - 127)


def scale_byte(block) -> int:
    """The scale byte of 32 values."""
    a = [abs(float(x)) for x in block]
    if any(x != x for x in a):
        return 255
    top = max(a)
    if top == 0.0:
        return 2
    if math.isinf(top):
        return 252
    e = math.frexp(top)[1] - 1                  # 2^e <= top < 2^(e + 1)
    s = e - 1 if top > 1.75 * 2.0 ** e else e - 2
    return min(max(s, -125), 125) + 127


def encode_one(x: float, byte: int) -> int:
    if byte == 255:
        return 0
    sign = 8 if math.copysign(1.0, x) < 0 else 0
    y = abs(x) / scale_value(byte)
    best = min(range(8), key=lambda c: (abs(min(y, 8.0) - TABLE[c]), c % 2))
    return sign | best


def encode(x):
    """x [..., D] -> codes [..., D], scale bytes [..., D // 32]."""
    x = np.asarray(x, np.float64)
    blocks = x.reshape(-1, BLOCK)
    scales = np.array([scale_byte(b) for b in blocks], np.uint8)
    codes = np.array([[encode_one(float(v), int(s)) for v in b] for b, s in zip(blocks, scales)], np.uint8)
    return codes.reshape(x.shape), scales.reshape(x.shape[:-1] + (x.shape[-1] // BLOCK,))


def decode(codes, scales):
    size = np.array([scale_value(int(s)) for s in range(256)])[np.asarray(scales, np.int64)]
    return TABLE[np.asarray(codes, np.int64)] * np.repeat(size, BLOCK, -1)


def page_bytes(bs, D):
    return bs * D // 2 + bs * D // BLOCK


def code_byte(which, slot, d, bs, D):
    if which == "k":
        return ((d // 32) * bs + slot) * 16 + (d % 32) // 2
    return ((slot // 8) * (D // 4) + d // 4) * 16 + (slot % 8) * 2 + (d % 4) // 2


def scale_at(which, slot, d, bs, D):
    return bs * D // 2 + (slot * (D // 32) + d // 32 if which == "k" else (d // 32) * bs + slot)


def put_row(page, which, slot, codes, scales, bs):
    """One token's row (codes [D], scales [D // 32]) into a page (uint8, page_bytes)."""
    D = len(codes)
    for d in range(D):
        at, shift = code_byte(which, slot, d, bs, D), 4 * (d % 2)
        page[at] = (int(page[at]) & (0xF0 if shift == 0 else 0x0F)) | (int(codes[d]) << shift)
        page[scale_at(which, slot, d, bs, D)] = scales[d // BLOCK]


def decode_pages(pages, which, bs, D):
    """pages [nb, H, page_bytes] uint8 -> float64 [nb, H, bs, D]."""
    slot, d = np.meshgrid(np.arange(bs), np.arange(D), indexing="ij")
    code = (pages[:, :, code_byte(which, slot, d, bs, D)] >> (4 * (d % 2))) & 15
    size = np.array([scale_value(s) for s in range(256)])[pages[:, :, scale_at(which, slot, d, bs, D)]]
    return TABLE[code] * size

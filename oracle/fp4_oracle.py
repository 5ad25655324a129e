"""Rows held in 4 bits and blocks of a paged cache, from their definitions in float64 (numpy), one value or one request at a time
where that is the definition.

  quantise, values    E2M1 codes with a power-of-two scale for every 32 elements
  block_tables        requests in order, blocks from a free list, slots of the new tokens
"""
from __future__ import annotations

from fractions import Fraction

import numpy as np

BLOCK = 32
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
NAN_BYTE = 255


def scale_exponent(top: float) -> int:
    """The smallest e >= -126 with top <= 7 * 2^e, 125 at most, in exact arithmetic."""
    e = -126
    top = Fraction(float(top))
    while e < 125 and top > 7 * Fraction(2) ** e:
        e += 1
    return e


def nearest_code(y: float) -> int:
    """The magnitude code nearest to y >= 0; ties to the even code; beyond the largest, the largest."""
    off = [abs(Fraction(float(y)) - Fraction(m)) for m in MAGNITUDES]
    least = min(off)
    best = [c for c in range(8) if off[c] == least]
    return best[0] if len(best) == 1 else [c for c in best if c % 2 == 0][0]


def quantise(x: np.ndarray):
    """Rows x [..., d] -> (codes uint8 [..., d / 2], two a byte, element 2 i in the low half; scale bytes uint8 [..., d / 32])."""
    x = np.asarray(x, dtype=np.float64)
    blocks = x.reshape(-1, BLOCK)
    top = np.abs(blocks).max(axis=1)
    bad = ~np.isfinite(blocks).all(axis=1)
    with np.errstate(invalid="ignore"):
        mantissa, exponent = np.frexp(np.where(bad, 0.0, top))
    e = np.where(mantissa <= 0.875, exponent - 3, exponent - 2)      # top = mantissa 2^exponent <= 7 2^(exponent - 3) iff mantissa <= 7/8
    e = np.clip(np.where(top == 0.0, -126, e), -126, 125)
    y = np.abs(np.where(bad[:, None], 0.0, blocks)) * np.ldexp(1.0, -e)[:, None]
    edges = (np.array(MAGNITUDES[1:]) + np.array(MAGNITUDES[:-1])) / 2
    code = np.zeros(y.shape, dtype=np.uint8)
    for i, edge in enumerate(edges):                     # on an edge the even one of the codes i and i + 1
        code += (y > edge) if i % 2 == 0 else (y >= edge)
    code |= (np.signbit(blocks) & ~bad[:, None]).astype(np.uint8) << 3
    code = code.reshape(x.shape)
    byte = np.where(bad, NAN_BYTE, e + 127).astype(np.uint8)
    return code[..., 0::2] | code[..., 1::2] << 4, byte.reshape(x.shape[:-1] + (x.shape[-1] // BLOCK,))


def values(codes: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """Codes [..., d / 2] and scale bytes [..., d / 32] -> float64 [..., d]."""
    half = np.stack((codes & 15, codes >> 4), axis=-1).reshape(codes.shape[:-1] + (2 * codes.shape[-1],))
    size = np.array(MAGNITUDES)[half & 7]
    x = np.where(half & 8, -size, size).reshape(scales.shape + (BLOCK,))
    unit = np.where(scales == NAN_BYTE, np.nan, np.ldexp(1.0, scales.astype(np.int64) - 127))
    return (x * unit[..., None]).reshape(half.shape)


def block_tables(length, n_kv_heads: int, block_rows: int, blocks_per_seq: int, free, n_slots=None, held=None, table=None):
    """(table [batch, n_kv_heads, blocks_per_seq], live [batch], slots [n_kv_heads, n_slots] or None, (taken, wanted, tokens)).
    Requests one after the other (n_slots None or 0: no slots are asked for); `table` is the table so far (its entries of held blocks are read)."""
    B, H, R = len(length), n_kv_heads, block_rows
    n_slots = n_slots or None
    fresh = held is None
    held = [0] * B if fresh else [max(int(x), 0) for x in held]
    length = [max(int(n), h) for n, h in zip(length, held)]
    out = np.zeros((B, H, blocks_per_seq), dtype=np.int32) if fresh else np.array(table, dtype=np.int32)
    live = np.zeros(B, dtype=np.int32)
    slots = None if n_slots is None else np.full((H, n_slots), -1, dtype=np.int64)
    wanted = tokens = taken = 0
    up = lambda n: -(-n // R)
    for b in range(B):
        new, first = length[b] - held[b], tokens
        tokens += new
        too_long = up(length[b]) > blocks_per_seq
        need = 0 if too_long else H * (up(length[b]) - up(held[b]))
        at = wanted
        wanted += need
        ok = not too_long and (need == 0 or wanted <= len(free)) and (n_slots is None or new == 0 or tokens <= n_slots)
        live[b] = length[b] if ok else held[b]
        if not ok:
            continue
        if need:
            taken = wanted
        for h in range(H):
            for c in range(up(held[b]), up(length[b])):
                out[b, h, c] = free[at]
                at += 1
            if slots is not None:
                pos = np.arange(held[b], length[b])
                slots[h, first:first + new] = out[b, h, pos // R].astype(np.int64) * R + pos % R
    return out, live, slots, (taken, wanted, min(tokens, 2 ** 31 - 1))

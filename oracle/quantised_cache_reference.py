"""TEST INFRASTRUCTURE ONLY -- what the 4-bit cache must hold and what it stands for, from the definition in the library's header.

Numbers have a sign and one of eight magnitudes; a key's block of 32 channels shares a power of two, the values of a (position, KV
head) a float of four significant bits.  Scales and codes are found here by search over all candidates in double precision, in which every
comparison is exact: magnitudes, scales and their products with a code have a few significant bits each.  Records are filled byte by byte.
The comparison bar is bit-exact.
"""
from __future__ import annotations

import numpy as np

PAGE = 16
BLOCK = 32
MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
LOWEST, HIGHEST = -100, 124


def _f64(bits: np.ndarray) -> np.ndarray:
    return (np.asarray(bits, np.uint16).astype(np.uint32) << np.uint32(16)).view(np.float32).astype(np.float64)


def _bits(x: np.ndarray) -> np.ndarray:
    """bf16 bits of values that bf16 represents."""
    f = np.ascontiguousarray(x, np.float32)
    b = (f.view(np.uint32) >> np.uint32(16)).astype(np.uint16)
    nan = np.isnan(x)
    assert (nan | (_f64(b) == x)).all(), "not representable"
    return np.where(nan, np.uint16(0x7FC0), b)


def record_bytes(head_dim: int) -> int:
    return 16 * head_dim + head_dim // 2 + 64


KEY_SCALES = np.exp2(np.arange(LOWEST, HIGHEST + 1, dtype=np.float64))
VALUE_SCALES = np.sort(np.concatenate([np.arange(8, 16) * 2.0 ** (e - 3) for e in range(LOWEST, HIGHEST)] + [[2.0 ** HIGHEST]]))


def smallest_scale(top: np.ndarray, scales: np.ndarray) -> np.ndarray:
    """The smallest of ``scales`` (ascending) with top <= 6 * scale; the largest where there is none."""
    i = np.searchsorted(6.0 * scales, top, side="left")
    return scales[np.minimum(i, len(scales) - 1)]


def nearest_code(x: np.ndarray, scale: np.ndarray) -> np.ndarray:
    """Codes of ``x`` in units of ``scale``: nearest magnitude, of two as near the one with the even code; the sign in bit 3."""
    far = np.abs(np.abs(x)[..., None] - MAGNITUDES * scale[..., None])
    order = np.array([0, 2, 4, 6, 1, 3, 5, 7])
    return (order[np.argmin(far[..., order], axis=-1)] + 8 * np.signbit(x)).astype(np.uint8)


def quantise_keys(bits: np.ndarray):
    """Codes [..., D] and scale bytes [..., D / 32] of bf16 rows."""
    x = _f64(bits).reshape(bits.shape[:-1] + (-1, BLOCK))
    bad = ~np.isfinite(x).all(-1)
    x = np.where(bad[..., None], 0.0, x)
    scale = smallest_scale(np.abs(x).max(-1), KEY_SCALES)
    byte = np.where(bad, 255, np.rint(np.log2(scale)) + 127).astype(np.uint8)
    return nearest_code(x, np.broadcast_to(scale[..., None], x.shape)).reshape(bits.shape), byte


def quantise_values(bits: np.ndarray):
    """Codes [..., D] and scales [...] (float32, exact) of bf16 rows."""
    x = _f64(bits)
    bad = ~np.isfinite(x).all(-1)
    x = np.where(bad[..., None], 0.0, x)
    scale = smallest_scale(np.abs(x).max(-1), VALUE_SCALES)
    codes = nearest_code(x, np.broadcast_to(scale[..., None], x.shape))
    return codes, np.where(bad, np.nan, scale).astype(np.float32)


def key_places(head_dim: int):
    """(byte, shift) inside a record of every [slot, channel] of the keys."""
    slot, c = np.meshgrid(np.arange(PAGE), np.arange(head_dim), indexing="ij")
    return (c // BLOCK * PAGE + slot) * 16 + c % BLOCK // 2, 4 * (c % 2)


def value_places(head_dim: int):
    slot, c = np.meshgrid(np.arange(PAGE), np.arange(head_dim), indexing="ij")
    return 8 * head_dim + ((slot // 4 * 16 + c % 16) * (head_dim // 16) + c // 16) * 2 + slot % 4 // 2, 4 * (slot % 2)


def append(pool: np.ndarray, k_new: np.ndarray, v_new: np.ndarray, block_table, q_start, q_len, ctx_len) -> None:
    """Writes rows [T, Hkv, D] of bf16 bits into the pool, uint8 [pages, Hkv, record], in place."""
    d = k_new.shape[-1]
    k_code, k_byte = quantise_keys(k_new)
    v_code, v_scale = quantise_values(v_new)
    places = (key_places(d), k_code), (value_places(d), v_code)
    for s in range(len(q_len)):
        for j in range(int(q_len[s])):
            pos, t = int(ctx_len[s]) - int(q_len[s]) + j, int(q_start[s]) + j
            page, slot = int(block_table[s][pos // PAGE]), pos % PAGE
            for h in range(k_new.shape[1]):
                rec = pool[page, h]
                for (at, shift), code in places:
                    a, sh = at[slot], shift[slot].astype(np.uint8)
                    for parity in (0, 4):       # a byte may take two of the row's channels
                        c = np.nonzero(sh == parity)[0]
                        rec[a[c]] = (rec[a[c]] & np.uint8(0xF0 >> parity)) | (code[t, h, c] << np.uint8(parity))
                rec[16 * d + np.arange(d // BLOCK) * PAGE + slot] = k_byte[t, h]
                rec[16 * d + d // 2 + 4 * slot:16 * d + d // 2 + 4 * slot + 4] = v_scale[t, h].reshape(1).view(np.uint8)


def held_page(rec: np.ndarray, head_dim: int):
    """Keys and values [16, D] (float64) that records [..., record] stand for."""
    grid = np.concatenate([MAGNITUDES, -MAGNITUDES])
    (ka, ks), (va, vs) = key_places(head_dim), value_places(head_dim)
    k = grid[(rec[..., ka] >> ks.astype(np.uint8)) & 15]
    v = grid[(rec[..., va] >> vs.astype(np.uint8)) & 15]
    byte = rec[..., 16 * head_dim:16 * head_dim + head_dim // 2].reshape(rec.shape[:-1] + (-1, PAGE)).swapaxes(-1, -2)
    unit = np.where(byte == 255, np.nan, np.exp2(byte.astype(np.float64) - 127))
    scale = np.ascontiguousarray(rec[..., 16 * head_dim + head_dim // 2:]).view(np.float32).astype(np.float64)
    return k * np.repeat(unit, BLOCK, axis=-1), v * scale[..., None]


def read(pool: np.ndarray, block_table, q_len, ctx_len, head_dim: int):
    """bf16 bits [T, Hkv, D] of positions ctx_len - q_len .. ctx_len - 1 of each sequence."""
    ks, vs = [], []
    for s in range(len(q_len)):
        first, end = int(ctx_len[s]) - int(q_len[s]), int(ctx_len[s])
        lo, hi = first // PAGE, (end - 1) // PAGE + 1
        k, v = held_page(pool[np.asarray(block_table[s][lo:hi])], head_dim)      # [pages, Hkv, 16, D]
        for x, out in ((k, ks), (v, vs)):
            rows = x.transpose(0, 2, 1, 3).reshape(-1, pool.shape[1], head_dim)
            out.append(rows[first - lo * PAGE:end - lo * PAGE])
    return _bits(np.concatenate(ks)), _bits(np.concatenate(vs))


def stands_for(k_bits: np.ndarray, v_bits: np.ndarray):
    """bf16 bits of what rows become by being held in 4 bits."""
    code, byte = quantise_keys(k_bits)
    grid = np.concatenate([MAGNITUDES, -MAGNITUDES])
    unit = np.where(byte == 255, np.nan, np.exp2(byte.astype(np.float64) - 127))
    k = grid[code] * np.repeat(unit, BLOCK, axis=-1)
    code, scale = quantise_values(v_bits)
    return _bits(k), _bits(grid[code] * scale.astype(np.float64)[..., None])

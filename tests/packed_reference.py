"""The 4-bit cache in plain numpy, from its description: every element by trying all sixteen values, every record byte
by byte.  Nothing of the library is used."""
import numpy as np

VALUES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
RECORD = 2176


def power_of_block(x):
    """e for 32 numbers (binary64), or None where one is infinite or NaN."""
    if not np.isfinite(x).all():
        return None
    top, e = np.abs(x).max(), -126
    while top > 7 * 2.0 ** e:
        e += 1
    return e


def pack_row(x):
    """128 numbers to 128 codes and 4 power bytes."""
    codes, powers = np.zeros(128, np.uint8), np.zeros(4, np.uint8)
    for b in range(4):
        block = x[32 * b:32 * b + 32]
        e = power_of_block(block)
        powers[b] = 255 if e is None else e + 127
        if e is None:
            continue
        for i, v in enumerate(block):
            off = np.abs(abs(v) / 2.0 ** e - VALUES)
            near = np.flatnonzero(off == off.min())
            code = near[0] if near[0] % 2 == 0 else near[-1]           # a tie goes to the even code
            codes[32 * b + i] = code | (8 if np.signbit(v) else 0)
    return codes, powers


def pack_record(k, v):
    """Keys and values [16][128] (binary64) to one record."""
    rec = np.zeros(RECORD, np.uint8)
    for t in range(16):
        for x, is_value in ((k[t], False), (v[t], True)):
            codes, powers = pack_row(x)
            for c in range(128):
                at = 1024 + ((t // 4 * 16 + c // 8) * 4 + t % 4) * 4 + c % 8 // 2 if is_value else t * 64 + c // 2
                rec[at] |= codes[c] << (4 * (c % 2))
            for b in range(4):
                rec[2112 + b * 16 + t if is_value else 2048 + t * 4 + b] = powers[b]
    return rec


def unpack(pool):
    """Records [..., 2176] to keys and values [..., 16, 128] in binary64."""
    t, c = np.arange(16)[:, None], np.arange(128)[None]
    signed = np.concatenate([VALUES, -VALUES])
    got = []
    for at, e in ((t * 64 + c // 2, 2048 + t * 4 + c // 32),
                  (1024 + ((t // 4 * 16 + c // 8) * 4 + t % 4) * 4 + c % 8 // 2, 2112 + c // 32 * 16 + t)):
        power = pool[..., e].astype(np.float64)
        got.append(signed[pool[..., at] >> (4 * (c % 2)) & 15] * np.where(power == 255, np.nan, 2.0 ** (power - 127)))
    return got

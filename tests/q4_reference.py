"""The 4-bit cache in plain numpy: coding in 64 bits and the layout of a slab, byte by byte, as sv.h states them."""
import numpy as np

SLAB = 9216


def bf16(x):
    """Rounded once to bfloat16 (nearest, ties to even), as float64: by way of fp32 cut towards zero, whose last bit says that there was more
    (rounded to fp32 instead, a number next to a tie becomes one)."""
    x = np.asarray(x, np.float64)
    with np.errstate(over="ignore", invalid="ignore"):
        y = x.astype(np.float32)
        y = np.where(np.abs(y) > np.abs(x), np.nextafter(y, np.float32(0)), y)
        b = (y.view(np.uint32) | (y != x)).astype(np.uint64)
    r = ((b + 0x7fff + ((b >> 16) & 1)) >> 16 << 16).astype(np.uint32)
    return np.where(np.isnan(x), np.float32(np.nan), r.view(np.float32)).astype(np.float64)


def code(rows):
    """Codes, scales and offsets of rows [...][128] of bfloat16 values."""
    g = np.asarray(rows, np.float64).reshape(*rows.shape[:-1], 2, 64)
    odd = ~np.isfinite(g).all(-1)
    g = np.where(odd[..., None], 0.0, g)
    low, high = g.min(-1), g.max(-1)
    f = lambda x: np.float64(np.float32(x))                      # each step rounded to fp32
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        scale = bf16(f(f(f(high - low) / 15) * 16))
        offset = bf16(f(low - scale))
        c = np.rint(f(f(f(f(g - offset[..., None]) / scale[..., None]) * 16) - 16))
    c = np.where(scale[..., None] > 0, np.clip(np.nan_to_num(c), 0, 15), 0).astype(np.int64)
    return np.where(odd[..., None], 0, c).reshape(rows.shape), np.where(odd, np.nan, scale), np.where(odd, np.nan, offset)


def stands_for(c, scale, offset):
    """(1 + c / 16) scale + offset, rounded once.  The product has 13 bits; of the sum, what 64 bits cut off goes into the last of them, so
    that nothing next to a tie becomes one."""
    with np.errstate(invalid="ignore", over="ignore"):
        a, m = (1 + c / 16) * scale, np.asarray(offset, np.float64) + 0 * scale
        s = np.asarray(a + m)
        b = s - a
        cut = (a - (s - b)) + (m - b)
        even = (s.view(np.int64) & 1) == 0
        return bf16(np.where((cut != 0) & np.isfinite(cut) & even, np.nextafter(s, np.sign(cut) * np.inf), s))


def value(codes, scale, offset):
    c = codes.reshape(*codes.shape[:-1], 2, 64)
    return stands_for(c, scale[..., None], offset[..., None]).reshape(codes.shape)


def _bits(x):
    return np.where(np.isnan(x), np.uint16(0x7fff), (np.asarray(x, np.float32).view(np.uint32) >> 16).astype(np.uint16))


def put(slab, t, k, v):
    """Token t (0..63) of a slab (uint8 [SLAB], in place): one row of keys, one of values."""
    for first, row in ((0, k), (4096, v)):
        c, scale, offset = code(row)
        for d in range(128):
            if first:
                byte, e = 4096 + (t // 32) * 2048 + d * 16 + (t % 32) // 8 * 4, t % 8
            else:
                byte, e = (d // 32) * 1024 + t * 16 + (d % 32) // 8 * 4, d % 8
            n = e // 2 if e % 2 == 0 else 4 + e // 2                 # its nibble of the word
            byte, shift = byte + n // 2, 4 * (n % 2)
            slab[byte] = (int(slab[byte]) & ~(15 << shift) & 0xff) | int(c[d]) << shift
        for g in range(2):
            for i, x in enumerate((scale[g], offset[g])):
                at = 8704 + g * 256 + i * 128 + t * 2 if first else 8192 + t * 8 + g * 4 + i * 2
                slab[at:at + 2] = np.frombuffer(np.uint16(_bits(x)).tobytes(), np.uint8)


def get(slab):
    """Keys and values [64][128] that a slab stands for."""
    t, d = np.meshgrid(np.arange(64), np.arange(128), indexing="ij")

    def nibble(byte, e):
        n = np.where(e % 2 == 0, e // 2, 4 + e // 2)
        return slab[byte + n // 2] >> (4 * (n % 2)) & 15

    num = lambda at: (slab[at].astype(np.uint32) << 16 | slab[at + 1].astype(np.uint32) << 24).view(np.float32).astype(np.float64)
    kc = nibble((d // 32) * 1024 + t * 16 + (d % 32) // 8 * 4, d % 8)
    vc = nibble(4096 + (t // 32) * 2048 + d * 16 + (t % 32) // 8 * 4, t % 8)
    g = d // 64
    return (stands_for(kc, num(8192 + t * 8 + g * 4), num(8192 + t * 8 + g * 4 + 2)),
            stands_for(vc, num(8704 + g * 256 + t * 2), num(8704 + g * 256 + 128 + t * 2)))

"""Plain definitions of the 8-bit cache in 64 bits (numpy): the e4m3 value list,
rounding to it, and the append."""
import numpy as np

LEAST = 87  # scale byte of 2^-40


def e4m3_values():
    """What byte codes 0 .. 126 stand for (127 is NaN; the sign bit mirrors them)."""
    c = np.arange(127)
    e, m = c >> 3, c & 7
    return np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))


VALUES = e4m3_values()


def decode(b):
    b = np.asarray(b, dtype=np.uint8)
    v = np.append(VALUES, np.nan)[b & 0x7f]
    return np.where(b & 0x80, -v, v)


def encode(x):
    """Codes of the nearest values (the even code among two equally near); NaN
    and infinities give 0x7f.  |x| may not exceed 448."""
    x = np.asarray(x, dtype=np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    assert a.size == 0 or a.max() <= 448.0
    hi = np.clip(np.searchsorted(VALUES, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = VALUES[hi] - a, a - VALUES[lo]
    code = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    code = np.where(VALUES[hi] == a, hi, code)
    code = code | np.where(np.signbit(x), 0x80, 0)
    return np.where(np.isfinite(x), code, 0x7f).astype(np.uint8)


def least_byte(top):
    b = LEAST
    while top > 448.0 * 2.0 ** (b - 127):
        b += 1
    return b


def append(pages, scale, rows, slots):
    """One run: rows [n, Hkv, 128] at consecutive slots of one page's bytes
    [Hkv, 16, 128] with scale bytes [Hkv]; both changed in place."""
    s0 = slots[0]
    for h in range(pages.shape[0]):
        x = rows[:, h].astype(np.float64)
        fine = np.abs(x[np.isfinite(x)])
        b = least_byte(fine.max() if fine.size else 0.0)
        if s0:
            was = int(scale[h])
            b = max(b, was)
            if b != was:
                pages[h, :s0] = encode(decode(pages[h, :s0]) * 2.0 ** (was - b))
        pages[h, slots] = encode(x * 2.0 ** (127 - b)) if b != 255 else 0x7f
        scale[h] = b


def same_bytes(a, b):
    """Equal codes, any NaN equal to any other."""
    return bool(np.all((a == b) | (((a & 0x7f) == 0x7f) & ((b & 0x7f) == 0x7f))))

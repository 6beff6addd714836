"""Plain 64-bit implementations of the block formats and of the rotation, written from their definitions: every element is compared with every level."""
import numpy as np

BITS = {"mxfp4": 4, "mxfp8": 8}


def levels(fmt):
    """Values of the codes without a sign, in their order."""
    if fmt == "mxfp4":
        return np.array([(1 + m / 2) * 2.0 ** (e - 1) if e else m / 2 for e in range(4) for m in range(2)])
    return np.array([(1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6 for e in range(16) for m in range(8)][:-1])     # the last code is NaN


def encode(x, fmt):
    """Rows x [..., d]: (codes as elements [..., d] uint8, scales [..., d / 32] uint8)."""
    x = np.asarray(x, dtype=np.float64)
    lv, bits = levels(fmt), BITS[fmt]
    top, lowest = (7.0, -125) if fmt == "mxfp4" else (464.0, -117)
    mid = (lv[1:] + lv[:-1]) / 2
    b = x.reshape(x.shape[:-1] + (x.shape[-1] // 32, 32))
    fine = np.isfinite(b).all(-1)
    most = np.abs(np.where(fine[..., None], b, 0)).max(-1)
    E = np.full(most.shape, lowest)
    for e in range(128, lowest, -1):                       # the smallest exponent that reaches
        E = np.where(most > top * 2.0 ** (e - 1), np.maximum(E, e), E)
    y = np.abs(np.where(fine[..., None], b, 0)) / 2.0 ** E[..., None].astype(np.float64)
    code = np.searchsorted(mid, y, side="left")            # middles below y: the nearer level, a tie goes to the lower one
    tie = (code < len(mid)) & (mid[np.minimum(code, len(mid) - 1)] == y) & (code % 2 == 1)
    code = code + tie                                      # ... unless that one's code is odd
    code = np.where(np.signbit(b) & fine[..., None], code | 1 << (bits - 1), code)
    return code.astype(np.uint8).reshape(x.shape), np.where(fine, E + 127, 255).astype(np.uint8)


def pack(code, fmt):
    return code if fmt == "mxfp8" else (code[..., 0::2] | code[..., 1::2] << 4).astype(np.uint8)


def unpack(codes, fmt):
    return codes if fmt == "mxfp8" else np.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[:-1] + (2 * codes.shape[-1],))


def decode(codes, scales, fmt):
    """Values of packed codes [..., bytes] and scales."""
    lv, bits = levels(fmt), BITS[fmt]
    c = unpack(codes, fmt).astype(np.int64)
    mag = c & ((1 << (bits - 1)) - 1)
    value = np.append(lv, np.nan)[np.minimum(mag, len(lv))]
    value = np.where(c >> (bits - 1), -value, value)
    s = scales.astype(np.int64)
    unit = np.where(s == 255, np.nan, 2.0 ** (np.minimum(s, 254) - 127.0))
    return value * np.repeat(unit, 32, axis=-1)


def held(x, fmt):
    """What rows x read back as."""
    code, scale = encode(x, fmt)
    return decode(pack(code, fmt), scale, fmt)


def rope(x, pos, inv_freq, axis, layout, inverse=False):
    """x [n, H, d], pos [axes, n].  layout: "half" or "interleaved".  A pair whose axis does not exist stays."""
    x = np.array(x, dtype=np.float64)
    pairs = len(inv_freq)
    for i in range(pairs):
        a = 0 if axis is None else int(axis[i])
        if a >= len(pos):
            continue
        angle = np.asarray(pos[a], dtype=np.longdouble) * np.longdouble(float(inv_freq[i]))
        c, s = np.cos(angle).astype(np.float64)[:, None], np.sin(angle).astype(np.float64)[:, None]
        if inverse:
            s = -s
        p, q = (i, i + pairs) if layout == "half" else (2 * i, 2 * i + 1)
        x[:, :, p], x[:, :, q] = x[:, :, p] * c - x[:, :, q] * s, x[:, :, q] * c + x[:, :, p] * s
    return x

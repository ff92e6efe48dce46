"""fp64 reference of the quantised cache: the two element formats, their group scales, the layout of a page's slab.

Everything goes element by element from the definitions: the scale by trying exponents, an element by its distance from
every value of its format, a byte's place by its formula.
"""
import numpy as np

GROUP, PAGE = 32, 16
TOP = {4: 7.0, 8: 464.0}
RANGE = {4: (-125, 125), 8: (-117, 119)}


def magnitudes(bits):
    """The values of codes 0, 1, 2, ... without their sign."""
    man, bias, count = (1, 1, 8) if bits == 4 else (3, 7, 127)
    out = []
    for c in range(count):
        e, f = c >> man, c & ((1 << man) - 1)
        out.append((f / 2 ** man if e == 0 else 1 + f / 2 ** man) * 2.0 ** (max(e, 1) - bias))
    return np.array(out)


def exponent(size, bits):
    """Least e of the format's range with size <= top * 2^e (the largest e where there is none)."""
    lo, hi = RANGE[bits]
    for e in range(lo, hi):
        if size <= TOP[bits] * 2.0 ** e:
            return e
    return hi


def quantise(row, bits):
    """row [d] -> (codes [d], scale bytes [d / 32]), uint8."""
    row = np.asarray(row, dtype=np.float64)
    codes, scales = np.zeros(len(row), np.uint8), np.zeros(len(row) // GROUP, np.uint8)
    table = magnitudes(bits)
    for g in range(len(row) // GROUP):
        x = row[g * GROUP:(g + 1) * GROUP]
        if not np.all(np.isfinite(x)):
            scales[g] = 255
            continue
        e = exponent(np.abs(x).max(), bits)
        scales[g] = e + 127
        dist = np.abs(np.minimum(np.abs(x) / 2.0 ** e, table[-1])[:, None] - table)
        best = dist.min(1, keepdims=True)
        near = dist == best
        pick = near.argmax(1)                                     # the lower of two at the same distance
        tie = near.sum(1) == 2
        pick = np.where(tie & (pick % 2 == 1), pick + 1, pick)    # ties to the even code
        codes[g * GROUP:(g + 1) * GROUP] = pick + np.signbit(x) * (1 << (bits - 1))
    return codes, scales


def values(codes, scales, bits):
    """What codes [..., d] and scale bytes [..., d / 32] stand for."""
    table = magnitudes(bits)
    table = np.concatenate([table, np.full((1 << (bits - 1)) - len(table), np.nan)])
    v = np.concatenate([table, -table])[codes]
    s = np.where(scales == 255, np.nan, 2.0 ** (np.minimum(scales, 254).astype(np.float64) - 127))
    return v * np.repeat(s, GROUP, axis=-1)


def slab_bytes(d, kb, vb):
    return PAGE * d * (kb + vb) // 8 + 2 * PAGE * d // GROUP


def code_place(t, e, d, bits, is_v):
    """(byte within the part's codes, first bit within the byte) of element e of token t."""
    if is_v:
        lane, element = (t // 4) * 16 + e // (d // 16), (t % 4) * (d // 16) + e % (d // 16)
    else:
        lane, element = (e // (d // 4)) * 16 + t, e % (d // 4)
    byte, bit = element * bits // 8, element * bits % 8
    width = min(16, d // 4 * bits // 8)                           # bytes of a lane in a plane
    return (byte // width) * 64 * width + lane * width + byte % width, bit


def scale_place(t, g, d, is_v):
    return (t // 4) * 4 * (d // GROUP) + g * 4 + t % 4 if is_v else g * PAGE + t


class Places:
    """Where the parts of every token lie in a slab: byte and bit of its codes, byte of its scales."""

    def __init__(self, d, kb, vb):
        starts = np.cumsum([0, PAGE * d * kb // 8, PAGE * d * vb // 8, PAGE * d // GROUP])
        self.parts = []
        for is_v, bits in ((False, kb), (True, vb)):
            byte, bit = np.zeros((PAGE, d), int), np.zeros((PAGE, d), int)
            scale = np.zeros((PAGE, d // GROUP), int)
            for t in range(PAGE):
                for e in range(d):
                    byte[t, e], bit[t, e] = code_place(t, e, d, bits, is_v)
                for g in range(d // GROUP):
                    scale[t, g] = scale_place(t, g, d, is_v)
            self.parts.append((bits, byte + starts[int(is_v)], bit, scale + starts[2 + int(is_v)]))
        self.bytes = slab_bytes(d, kb, vb)

    def store(self, slab, t, k, v):
        """Token t's rows quantised into slab [bytes] (uint8, changed in place)."""
        for x, (bits, byte, bit, scale) in zip((k, v), self.parts):
            codes, scales = quantise(x, bits)
            for e, c in enumerate(codes):
                keep = 0xff ^ (((1 << bits) - 1) << bit[t, e])
                slab[byte[t, e]] = (slab[byte[t, e]] & keep) | (int(c) << bit[t, e])
            slab[scale[t]] = scales

    def rows(self, slabs):
        """K and V [n * 16][d] of slabs [n][bytes], in 64 bits."""
        out = []
        for bits, byte, bit, scale in self.parts:
            codes = (slabs[:, byte] >> bit) & ((1 << bits) - 1)
            v = values(codes, slabs[:, scale], bits)
            out.append(v.reshape(-1, v.shape[-1]))
        return out

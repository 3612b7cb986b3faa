"""CPU oracle (test infrastructure only): the 8-bit KV cache, e4m3 codes with a power-of-two scale for every 64 tokens of a KV head.

Numbers are fp64 throughout; a code is a byte and its value comes from the definition of the format: sign, four bits of exponent
(bias 7), three of fraction; exponent 0 holds the multiples of 2^-9; 0x7f and 0xff are NaN; there are no infinities.
"""
import numpy as np

from oracle import forward as ofwd

BLOCK = 64


def _value(code):
    sign = -1.0 if code & 0x80 else 1.0
    e, f = (code >> 3) & 15, code & 7
    if e == 15 and f == 7:
        return float("nan")
    return sign * (f * 2.0 ** -9 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7))


VALUES = np.array([_value(c) for c in range(256)])
_UP = VALUES[:127]                                           # 0 .. 448, ascending with the code


def encode(x):
    """The code of the nearest value, of two equally near the one with the even fraction; beyond 448: 448; no number: NaN."""
    x = np.asarray(x, np.float64)
    a = np.minimum(np.where(np.isfinite(x), np.abs(x), 0.0), 448.0)
    hi = np.clip(np.searchsorted(_UP, a), 1, 126)            # _UP[hi - 1] < a <= _UP[hi], but for a = 0
    below, above = a - _UP[hi - 1], _UP[hi] - a
    code = np.where((below < above) | ((below == above) & (hi % 2 == 1)), hi - 1, hi)
    code = np.where(np.isfinite(x), code, 127)
    return (code | np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def decode(codes):
    return VALUES[codes]


def scale_for(x):
    """The smallest power of two s, 2^-40 <= s <= 2^40, with max |x| <= 448 s over the numbers among x."""
    x = np.abs(np.asarray(x, np.float64))
    top = np.max(x[np.isfinite(x)], initial=0.0)
    e = -40
    while e < 40 and top > 448.0 * 2.0 ** e:
        e += 1
    return 2.0 ** e


class Plane:
    """K or V of one sequence and KV head: codes [max_len, d], scales [max_len / 64]."""

    def __init__(self, max_len, d):
        self.codes = np.full((max_len, d), 255, np.uint8)
        self.scale = np.full(max_len // BLOCK, np.nan)

    def append(self, s0, rows):
        end = s0 + len(rows)
        for block in range(s0 // BLOCK, (end - 1) // BLOCK + 1):
            lo, hi = max(s0, block * BLOCK), min(end, (block + 1) * BLOCK)
            new = np.asarray(rows[lo - s0:hi - s0], np.float64)
            scale = scale_for(new)
            if lo > block * BLOCK:                           # older tokens in the block
                before = self.scale[block]
                scale = max(scale, before)
                if scale > before:
                    old = self.codes[block * BLOCK:lo]
                    self.codes[block * BLOCK:lo] = encode(decode(old) * (before / scale))
            self.codes[lo:hi] = encode(new / scale)
            self.scale[block] = scale

    def numbers(self, n):
        return decode(self.codes[:n]) * np.repeat(self.scale, BLOCK)[:n, None]


class KVCache8(ofwd.KVCache):
    """The oracle's cache, in 8 bits: forward() reads back what the codes stand for."""

    def __init__(self, cfg, batch, max_len):
        super().__init__(cfg, batch, max_len)
        self.planes = [[[(Plane(max_len, cfg.d_head), Plane(max_len, cfg.d_head)) for _ in range(cfg.n_kv_heads)]
                        for _ in range(batch)] for _ in range(cfg.n_layers)]

    def append(self, l, b, s0, k, v):
        end = s0 + k.shape[0]
        first = s0 // BLOCK * BLOCK
        for h, (pk, pv) in enumerate(self.planes[l][b]):
            pk.append(s0, k[:, h])
            pv.append(s0, v[:, h])
            self.k[l][b, h, first:end] = pk.numbers(end)[first:]
            self.v[l][b, h, first:end] = pv.numbers(end)[first:]

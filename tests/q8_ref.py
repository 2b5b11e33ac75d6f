"""Plain 64-bit implementation of the 8-bit cache (numpy, written from the format's
definition): blocks of 32 elements with one exponent, in granules of 16 tokens."""
import numpy as np

from window_ref import P

BAD = 255  # exponent of a block that is NaN


def encode(x):
    """(codes uint8 [..., d], exponents uint8 [..., d / 32]) of fp32-representable numbers."""
    x = np.asarray(x, dtype=np.float64)
    b = x.reshape(*x.shape[:-1], -1, 32)
    fine = np.isfinite(b).all(-1)
    b = np.where(fine[..., None], b, 0.0)
    most = np.abs(b).max(-1)
    E = np.full(most.shape, 8)
    while True:  # the smallest exponent for which no magnitude rounds to 128
        over = np.rint(most * 2.0 ** (133.0 - E)) > 127
        if not over.any():
            break
        E = E + over
    fine &= E <= 253
    m = np.where(fine[..., None], np.rint(b * 2.0 ** (133.0 - E[..., None])), 0.0)
    codes = np.where(m < 0, 128 - m, m).astype(np.uint8)
    return codes.reshape(x.shape), np.where(fine, E, BAD).astype(np.uint8)


def decode(codes, exps):
    """fp64 numbers of codes [..., d] and exponents [..., d / 32]."""
    c = np.asarray(codes).astype(np.int64)
    m = np.where(c < 128, c, 128 - c).reshape(*c.shape[:-1], -1, 32).astype(np.float64)
    e = np.asarray(exps).astype(np.float64)
    step = np.where(e >= 254, np.nan, 2.0 ** (e - 133.0))
    return (m * step[..., None]).reshape(c.shape)


def half_step(most):
    """The largest rounding error of a block whose largest magnitude is `most`."""
    return 0.5 * 2.0 ** (encode(np.repeat(np.asarray(most, dtype=np.float64)[..., None], 32, -1))[1][..., 0] - 133.0)


class Cache8:
    """A paged 8-bit cache of `layers` layers, its pages scattered; what is not written is NaN (every byte 255)."""

    def __init__(self, requests, max_pages, Hkv, d, seed, layers=1, layer=0, fill=255, gap=0):
        self.R, self.max_pages, self.Hkv, self.d, self.layer = requests, max_pages, Hkv, d, layer
        self.layer_page_bytes = Hkv * 132 * d + gap
        page = layers * self.layer_page_bytes
        n = requests * max_pages + 1  # the last page is nobody's: entries of unread pages point at it
        self.bytes = np.full(n * page, fill, dtype=np.uint8)
        order = np.random.default_rng(seed).permutation(requests * max_pages)
        self.table = (order.reshape(requests, max_pages) * page).astype(np.int64)
        self.nobody = (n - 1) * page

    def slot(self, r, j, which):
        """Indices of (codes [Hkv][d], exponents [Hkv][d / 32]) of request r's position j (or positions [n], first)."""
        d, j = self.d, np.asarray(j)
        t = j % 16
        at = self.table[r, j // P] + self.layer * self.layer_page_bytes
        at = at[..., None] + (np.arange(self.Hkv) * 4 + (j % P // 16)[..., None]) * 33 * d  # [..., Hkv]
        i = np.arange(d)
        inside = (i // 16 ^ (t * d // 128 % (d // 16))[..., None]) * 16 + i % 16  # [..., d]
        codes = at[..., None] + which * 16 * d + ((t * d)[..., None] + inside)[..., None, :]
        exps = at[..., None] + 32 * d + which * (d // 2) + (t * (d // 32))[..., None, None] + np.arange(d // 32)
        return codes, exps

    def put(self, r, j, k, v):
        """k, v: numbers [..., Hkv][d], rounded to what the cache holds."""
        for which, x in ((0, k), (1, v)):
            (ic, ie), (c, e) = self.slot(r, j, which), encode(np.float32(x))
            self.bytes[ic], self.bytes[ie] = c, e

    def fill_request(self, r, positions, seed, scale=1.0, lean=None):
        rng = np.random.default_rng(seed)
        js = np.asarray(list(positions), dtype=np.int64)
        if not len(js):
            return
        k, v = rng.standard_normal((2, len(js), self.Hkv, self.d)) * scale
        for i, j in enumerate(js):
            if lean is not None and int(j) in lean:
                k[i] += 0.6 * lean[int(j)]
        self.put(r, js, k, v)

    def gather(self, r, js):
        out = []
        for which in (0, 1):
            ic, ie = self.slot(r, np.asarray(js), which)
            out.append(decode(self.bytes[ic], self.bytes[ie]))
        return out

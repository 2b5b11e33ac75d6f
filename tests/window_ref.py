"""Plain 64-bit implementation of the windowed-serving operators and the paged
caches they are tested on (numpy, written from the definitions)."""
import numpy as np

P = 64
U = 2.0 ** -24  # fp32 unit roundoff


def bf16_round(a):
    """fp32 -> the nearest bf16 (ties to even), as fp32.  Finite inputs."""
    u = np.ascontiguousarray(a, dtype=np.float32).view(np.uint32)
    u = (u + 0x7FFF + ((u >> 16) & 1)) & np.uint32(0xFFFF0000)
    return u.view(np.float32)


def bf16_bits(a):
    return (bf16_round(a).view(np.uint32) >> 16).astype(np.uint16)


def bits_f64(b):
    return (np.asarray(b, dtype=np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def visible(pos, j, window, sinks):
    """Whether the query at `pos` sees the cached position `j`."""
    return (j <= pos) & ((j > pos - window) | (j < sinks))


def seen_positions(rows, window, sinks):
    """The cached positions that a query at one of the positions `rows` sees, in order."""
    rows = np.asarray(list(rows), dtype=np.int64).reshape(-1, 1)
    j = np.arange(max(int(rows.max(initial=-1)) + 1, 0))[None, :]
    return np.flatnonzero(visible(rows, j, window, sinks).any(0)).tolist()


class Cache:
    """A paged cache of `layers` layers, its pages scattered; every element that is
    not written keeps `fill`."""

    def __init__(self, requests, max_pages, Hkv, d, seed, layers=1, layer=0, fill=0x7FC0, gap=0):
        self.R, self.max_pages, self.Hkv, self.d, self.layer = requests, max_pages, Hkv, d, layer
        self.layer_page_bytes = 2 * Hkv * P * d * 2 + gap
        page = layers * self.layer_page_bytes
        n = requests * max_pages + 1  # the last page is nobody's: entries of unread pages point at it
        self.bits = np.full(n * page // 2, fill, dtype=np.uint16)
        order = np.random.default_rng(seed).permutation(requests * max_pages)
        self.table = (order.reshape(requests, max_pages) * page).astype(np.int64)
        self.nobody = (n - 1) * page

    def slot(self, r, j, which):
        """Index of [Hkv][d] elements (as an index array) of request r's position j."""
        at = (self.table[r, j // P] + self.layer * self.layer_page_bytes) // 2 + which * self.Hkv * P * self.d
        return at + (np.arange(self.Hkv)[:, None] * P + j % P) * self.d + np.arange(self.d)[None, :]

    def put(self, r, j, k, v):
        """k, v: bf16 bits [Hkv][d]."""
        self.bits[self.slot(r, j, 0)] = k
        self.bits[self.slot(r, j, 1)] = v

    def fill_request(self, r, positions, seed, scale=1.0, lean=None):
        rng = np.random.default_rng(seed)
        for j in positions:
            k = rng.standard_normal((self.Hkv, self.d)) * scale
            if lean is not None and j in lean:
                k = k + 0.6 * lean[j]
            self.put(r, j, bf16_bits(k), bf16_bits(rng.standard_normal((self.Hkv, self.d)) * scale))

    def gather(self, r, js):
        js = np.asarray(js)
        at = (self.table[r, js // P] + self.layer * self.layer_page_bytes) // 2
        at = at[:, None] + (np.arange(self.Hkv)[None, :] * P + (js % P)[:, None]) * self.d
        at = at[:, :, None] + np.arange(self.d)
        return bits_f64(self.bits[at]), bits_f64(self.bits[at + self.Hkv * P * self.d])  # [n][Hkv][d]


def attend(cache, r, pos, q, window, sinks):
    """One row: (o, tol32, tolbf) with q [Hq][d] fp64; tol* bound the error of the two types.

    The scores carry delta = 2 (d + 16) U scale sum|q||k| (products summed in fp32,
    the tensor cores truncating), so a weight is off by a factor within exp(+-2 delta)
    and the 8 U of its exponential's argument; n terms are then summed in fp32.  A
    bf16 row's weights are rounded once (2^-9) and so is its output."""
    Hq, d = q.shape
    js = seen_positions([pos], window, sinks)
    if not js:
        return np.zeros((Hq, d)), np.zeros((Hq, d)), np.zeros((Hq, d))
    k, v = cache.gather(r, js)
    G = Hq // cache.Hkv
    K, V = k.transpose(1, 0, 2), v.transpose(1, 0, 2)  # [Hkv][n][d]
    Q = q.reshape(cache.Hkv, G, d)
    s = Q @ K.transpose(0, 2, 1) / np.sqrt(d)
    w = np.exp(s - s.max(-1, keepdims=True))
    w /= w.sum(-1, keepdims=True)
    o, mass = w @ V, w @ np.abs(V)
    top = (np.abs(Q) @ np.abs(K).transpose(0, 2, 1)).max(-1, keepdims=True) / np.sqrt(d)
    delta = 2 * (d + 16) * U * top + 8 * U * (1 + np.abs(s).max(-1, keepdims=True))
    t32 = mass * (np.expm1(2 * delta) + 2 * (len(js) + 64) * U) + 1e-30
    tbf = t32 + mass * 2.0 ** -8 + np.abs(o) * 2.0 ** -8
    return o.reshape(Hq, d), t32.reshape(Hq, d), tbf.reshape(Hq, d)


def append_row(x, pos, Hq, Hkv, d, g_q, g_k, eps, theta):
    """(q [Hq][d], k, v [Hkv][d], a bound of the fp32 error of q and k) of one fp64 row."""
    y = x.reshape(Hq + 2 * Hkv, d).copy()
    for lo, hi, g in ((0, Hq, g_q), (Hq, Hq + Hkv, g_k)):
        if g is not None:
            z = y[lo:hi]
            y[lo:hi] = z / np.sqrt((z * z).mean(-1, keepdims=True) + eps) * g
    a, b = y[:Hq + Hkv, :d // 2].copy(), y[:Hq + Hkv, d // 2:].copy()
    if theta:
        ang = pos * np.float64(theta) ** (-2.0 * np.arange(d // 2) / d)
        c, s = np.cos(ang), np.sin(ang)
        y[:Hq + Hkv, :d // 2], y[:Hq + Hkv, d // 2:] = a * c - b * s, b * c + a * s
    # the angle is held to 2^-32 of a turn and sincospi to 2 ulp; the norm sums d squares
    size = np.abs(a) + np.abs(b)
    tol = np.concatenate([size, size], -1) * (16 + (d if g_q is not None else 0)) * U
    return y[:Hq], y[Hq:Hq + Hkv], y[Hq + Hkv:], tol[:Hq], tol[Hq:]

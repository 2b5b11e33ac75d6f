"""Inputs on which each bf16 plane of the windowed attentions' operands counts, their exact
answers, and bounds that a lost plane breaks (numpy).

Every request sees two positions whose keys have one element each, so that a score is one
product and next to nothing is lost in sums:
  queries   scores of about 100 that differ by less than 2: o = tanh((s0 - s1) / 2)
  weights   weights 1 and e^-x with values 0 and 256:       o = 256 / (e^x + 1)
  opposed   weights 1 and e^-x with values 256 and -256:    o = 256 tanh(x / 2), x small
"""
import numpy as np

import window_ref as W
from window_ref import U, Cache

KINDS = ("queries", "weights", "opposed")


def case(kind, requests, Hq, Hkv, d, seed):
    """(cache, q [requests][Hq][d] fp32); the opposed case has bf16 queries."""
    rng = np.random.default_rng(seed)
    c = Cache(requests, 1, Hkv, d, seed, fill=0)
    q = np.zeros((requests, Hq, d))
    key = 16.0 if kind == "queries" else 1.0
    for r in range(requests):
        for j in range(2):
            k = np.zeros((Hkv, d))
            k[:, j] = key
            v = {"queries": (1.0, -1.0), "weights": (0.0, 256.0), "opposed": (256.0, -256.0)}[kind][j]
            c.put(r, j, W.bf16_bits(k), W.bf16_bits(np.full((Hkv, d), v)))
    if kind == "queries":
        q[..., 0] = 64 + 32 * rng.random((requests, Hq))
        q[..., 1] = q[..., 0] + 0.5 * rng.standard_normal((requests, Hq))
    else:
        x = rng.uniform(0.1, 3, (requests, Hq)) if kind == "weights" else rng.uniform(0.005, 0.03, (requests, Hq))
        q[..., 1] = -x * np.sqrt(d)
    q = q.astype(np.float32)
    return c, (W.bf16_round(q) if kind == "opposed" else q)


def scores(kind, q):
    """Exact scores [..., 2]."""
    return q[..., :2].astype(np.float64) * (16.0 if kind == "queries" else 1.0) / np.sqrt(q.shape[-1])


def exact(kind, q):
    s = scores(kind, q)
    x = s[..., 0] - s[..., 1]
    return {"queries": np.tanh(x / 2), "weights": 256 / (np.exp(x) + 1), "opposed": 256 * np.tanh(x / 2)}[kind]


def bound(kind, q, dtype):
    """A score is summed from its planes (two sums that may truncate: 4 U), scaled and taken from the
    rounded maximum (2 U); the exponential is good to 4 U beside its argument; a sum over planes and
    positions, the division and the output are 16 U of the mass.  Two planes of a weight: 2^-16."""
    s = scores(kind, q)
    o = exact(kind, q)
    delta = 6 * U * np.abs(s).sum(-1) + 8 * U  # of ln(w0 / w1)
    mass = {"queries": 1.0, "weights": np.abs(o), "opposed": 256.0}[kind]
    slope = {"queries": 0.5, "weights": 1.0, "opposed": 0.5}[kind]  # |do| <= slope mass delta
    t = mass * (slope * delta + 16 * U)
    return t if dtype == "f32" else t + 2.0 ** -16 * mass + 2.0 ** -8 * np.abs(o)

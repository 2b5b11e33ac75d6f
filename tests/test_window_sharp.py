"""The sharp inputs of window_sharp.py tell a lost plane: a host emulation of the attention on
bf16 planes stays within the bounds with all of them and leaves them with one taken out."""
import numpy as np
import pytest

import window_ref as W
import window_sharp as S


def planes(v, n, rounded_last=True):
    """n bf16 planes of fp32 numbers: each the largest below what is left, the last one rounded."""
    out, v = [], np.asarray(v, dtype=np.float32)
    for i in range(n):
        if i == n - 1 and rounded_last:
            p = W.bf16_round(v)
        else:
            p = ((v * np.float32(1 - 2.0 ** -24)).view(np.uint32) & np.uint32(0xFFFF0000)).view(np.float32)
        out.append(p)
        v = (v - p).astype(np.float32)
    return out


def emulate(kind, q, q_planes, w_planes):
    """q [..., d]; how many planes of the queries and of the weights are multiplied (of three)."""
    key = np.float32(16 if kind == "queries" else 1)
    f = np.float32
    s = np.zeros(q.shape[:-1] + (2,), dtype=f)
    for p in reversed(planes(q[..., :2], 3)[:q_planes]):
        s = (s + p * key).astype(f)
    a = (s * f(1.4426950408889634 / np.sqrt(q.shape[-1]))).astype(f)
    w = np.exp2((a - a.max(-1, keepdims=True)).astype(f).astype(np.float64)).astype(f)
    v = np.array({"queries": (1, -1), "weights": (0, 256), "opposed": (256, -256)}[kind], dtype=f)
    o = np.zeros(q.shape[:-1], dtype=f)
    for p in reversed(planes(w, 3)[:w_planes] if w_planes != 2 else planes(w, 2)):
        o = (o + (p * v).sum(-1, dtype=f)).astype(f)
    return (o / w.sum(-1, dtype=f)).astype(np.float64)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind,dtype,good,lost", [
    ("queries", "f32", (3, 3), (2, 3)), ("weights", "f32", (3, 3), (3, 2)), ("opposed", "f32", (3, 3), (3, 2)),
    ("opposed", "bf16", (1, 2), (1, 1))])
def test_a_lost_plane_breaks_the_bound(kind, dtype, good, lost, d):
    _, q = S.case(kind, 4, 16, 2, d, 5)
    want, tol = S.exact(kind, q), S.bound(kind, q, dtype)

    def off(n):
        o = emulate(kind, q, *n)
        return np.abs((W.bf16_round(o.astype(np.float32)) if dtype == "bf16" else o) - want) / tol

    if dtype == "bf16":  # bf16 queries are their own first plane
        assert np.array_equal(W.bf16_round(q), q)
    ratio = off((3, good[1]) if dtype == "bf16" else good)
    assert ratio.max() <= 1
    ratio = off((3, lost[1]) if dtype == "bf16" else lost)
    assert ratio.max() > 1  # one element suffices for the test to fail


@pytest.mark.parametrize("kind", S.KINDS)
def test_the_exact_answers_are_the_definition(kind):
    c, q = S.case(kind, 2, 4, 2, 64, 6)
    for r in range(2):
        want, _, _ = W.attend(c, r, 1, q[r].astype(np.float64), 2, 0)
        assert np.allclose(want, S.exact(kind, q)[r][:, None], rtol=1e-12, atol=1e-12)

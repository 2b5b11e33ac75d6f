"""The plain decoder of plain_decoder.py against the oracle's, with the oracle's rounding of the cache (host only),
and what the 8-bit cache's rounding changes."""
import numpy as np
import pytest

import plain_decoder as D
import q8_ref as Q
from paper_2512_21835_gb300 import configs, inputs


@pytest.mark.parametrize("model", ["tiny", "tiny-mha", "tiny-qk"])
def test_it_is_the_oracles(orc, model):
    m = configs.MODELS[model]
    toks = inputs.token_ids(7, 40, m["vocab"])
    desc = orc.ModelDesc(**m)
    ref = orc.forward(desc, orc.Weights(desc, configs.WEIGHT_SEED), toks, n_prefill=40, prefill_flags=0, decode_flags=0,
                      want_logits=True)
    z, logits = D.forward(orc, m, configs.WEIGHT_SEED, toks, lambda a: a, 1000, 0)
    assert np.max(np.abs(z - ref["hidden"])) < 1e-9 and np.max(np.abs(logits - ref["logits"])) < 1e-9
    ref = orc.forward(desc, orc.Weights(desc, configs.WEIGHT_SEED), toks, n_prefill=40, prefill_flags=orc.KV_BF16,
                      decode_flags=orc.KV_BF16)
    # rounded once, as the oracle does: by way of fp32 a number next to a border may come out on its other side
    z, _ = D.forward(orc, m, configs.WEIGHT_SEED, toks, orc.round_bf16, 1000, 0)
    assert np.max(np.abs(z - ref["hidden"])) < 1e-9


def q8(a):
    return Q.decode(*Q.encode(a))


@pytest.mark.parametrize("model", ["tiny", "tiny-mha", "tiny-qk"])
def test_another_cache_is_told_apart(orc, model):
    """A cache that does not round, one that makes every second block half as large and one that turns heads around
    are all outside the bound of test_gpu_q8_generation.py; 1e-6 of noise before the rounding is inside."""
    from test_gpu_q8_generation import BOUND
    m = configs.MODELS[model]
    toks = inputs.token_ids(7, 90, m["vocab"])
    want = D.forward(orc, m, configs.WEIGHT_SEED, toks, q8, 1000, 0)[0][79:]

    def off(f):
        return float(np.max(np.abs(D.forward(orc, m, configs.WEIGHT_SEED, toks, f, 1000, 0)[0][79:] - want)))

    def half(a):  # every second block at half its size
        b = q8(a).reshape(*a.shape[:-1], -1, 32).copy()
        b[..., ::2, :] *= 0.5
        return b.reshape(a.shape)

    assert off(half) > 2 * BOUND
    assert off(lambda a: np.flip(q8(a), -1)) > 2 * BOUND
    assert 0.02 < off(lambda a: a) < 0.04
    assert off(lambda a: q8(a * (1 + 1e-6))) < BOUND / 2

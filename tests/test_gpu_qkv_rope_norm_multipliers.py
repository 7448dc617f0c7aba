"""The common exponent of a head norm's multipliers where the largest factor lies next to a bound."""
import numpy as np
import pytest

import generation_reference as ref
from gpu_util import assert_same, ctx, dev, host

TOP = [(32767 / 64, 6), (np.nextafter(32767 / 64, np.inf), 5), (np.nextafter(32767 / 64, 0), 6), (32767 / 16384, 14),
       (np.nextafter(32767 / 16384, 4), 13), (32767.0, 0), (np.nextafter(32767.0, 4e4), -1), (32767 * 128.0, -7)]


def _factors(top):
    """One factor at the top; the others smaller, so that a bit more or less of them shows in the results."""
    gamma = np.random.default_rng(5).uniform(0.05, 0.2, 64) * top
    gamma[11] = -top
    return gamma


def _x(rng, T):
    return np.clip(np.rint(rng.standard_normal((T, 3 * 64)) * 5000), -32767, 32767).astype(np.int16)


@pytest.mark.parametrize("top,g", TOP)
def test_the_exponent_of_the_plain_form(top, g):
    """The largest g up to 16 with |gamma| (128 / S) 2^g <= 32767."""
    assert ref.head_norm_multipliers(_factors(top), 128.0)[1] == g


@pytest.mark.gpu
@pytest.mark.parametrize("top,g", TOP)
def test_factors_next_to_a_bound(top, g):
    T, S = 4000, 128.0
    x, gamma = _x(np.random.default_rng(1), T), _factors(top)
    out, _ = ctx().ibert_qkv_rope_i8(dev(x), 1.0, 1, 1, S, S, 200.0, gamma, gamma[::-1])
    ctx().check()
    q, k, v = ref.qkv_rope(x, 1, 1, 1.0, S, S, 200.0, gamma, gamma[::-1], None, None, False)
    assert_same(host(out), np.concatenate([q, k, v], 1).reshape(T, -1))

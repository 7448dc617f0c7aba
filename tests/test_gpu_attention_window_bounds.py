"""Windowed attention of sequences longer than the call says: reported, and still a defined result."""
import numpy as np
import pytest

import generation_reference as ref
from gpu_util import assert_same, ctx, dev, host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window,sinks,kept", [(33000, 40000, 32536), (59000, 60000, 6536), (70000, 60000, 5536), (5000, 300, 300)])
def test_overlong_sequences_see_at_most_65536_keys(window, sinks, kept):
    """The last min(window, max_len) keys and as many of the first ones as 65536 leave room for: the sums of weighted values
    stay in 32 bits however long the sequence is.  (Values near 127 everywhere: 73000 of them would not.)"""
    rng = np.random.default_rng(window)
    T, max_len, scales = 80000, 60000, (0.05, 0.04, 0.03, 0.03)
    qkv = np.empty((T, 3 * 64), np.int8)
    qkv[:, :128] = 3
    qkv[:, 128:] = rng.integers(120, 128, (T, 64))
    out, _ = ctx().ibert_attention_window_i8(dev(qkv), dev(np.array([0, T], np.int32)), max_len, 1, 1, *scales, window=window, sinks=sinks)
    assert ctx().ibert_last_status() == -8
    got = host(out)
    for row in (0, 100, 32999, 45000, 65535, 65536, 73000, T - 1):
        j = ref.visible(row + 1, min(window, max_len), kept)
        want = ref.weighted(np.full(j.size, 9 * 64), qkv[j, 128:].astype(np.int64), *scales, 255)
        assert_same(got[row], want.astype(np.int8), f"row {row}")

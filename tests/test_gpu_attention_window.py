"""Causal attention of packed sequences with window and sinks on the GPU against the plain 64-bit form."""
import numpy as np
import pytest
import torch

import generation_reference as ref
from gpu_util import assert_same, ctx, dev, host
from paper_2101_01321_b200 import binding

pytestmark = pytest.mark.gpu
SC = (0.05, 0.04, 0.03, 0.01)


def _run(rng, lens, heads, kv, window=0, sinks=0, p_max=255, max_len=None, scales=SC, behind=0, qkv=None, spread=35):
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    T = int(cu[-1]) + behind
    if qkv is None:
        qkv = np.clip(np.rint(rng.standard_normal((T, (heads + 2 * kv) * 64)) * spread), -127, 127).astype(np.int8)
    out = torch.full((T, heads * 64), 77, dtype=torch.int8, device="cuda")
    got, S = ctx().ibert_attention_window_i8(dev(qkv), dev(cu), max_len or max(1, max(lens)), heads, kv, *scales, window=window,
                                             sinks=sinks, p_max=p_max, out=out)
    ctx().check()
    assert S == scales[3] and got is out
    want = ref.attention_window(qkv, cu, heads, kv, window, sinks, scales, p_max)
    want[cu[-1]:] = 77                                             # rows behind the last sequence
    assert_same(host(out), want, "window")
    return want


@pytest.mark.parametrize("lens", [[1], [2], [63], [64], [65], [127], [128], [129], [200], [256], [300], [1] * 130, [0, 5, 0, 0, 128, 0], [0, 0, 1],
                                  [3] * 50, [120, 1, 7, 128, 2], [1, 0, 255, 64, 31], [40] * 9])
@pytest.mark.parametrize("p_max", [255, 127])
def test_causal(lens, p_max):
    _run(np.random.default_rng(len(lens) + sum(lens)), lens, 2, 1, p_max=p_max)


@pytest.mark.parametrize("heads,kv", [(1, 1), (3, 3), (12, 12), (8, 2), (6, 1)])
def test_heads(heads, kv):
    want = _run(np.random.default_rng(heads), [70, 150, 9], heads, kv)
    assert np.abs(want).max() > 5


@pytest.mark.parametrize("window", [1, 2, 31, 63, 64, 65, 128, 200, 1000])
@pytest.mark.parametrize("sinks", [0, 1, 4, 63, 64, 65, 130, 1000])
def test_window_and_sinks(window, sinks):
    _run(np.random.default_rng(window + sinks), [500, 33, 1, 290], 1, 1, window, sinks)


def test_long_sequences():
    rng = np.random.default_rng(1)
    _run(rng, [2600], 1, 1)
    _run(rng, [700, 2100], 2, 1, 600, 5)
    _run(rng, [4500], 1, 1, 64, 1)


def test_rows_behind_the_last_sequence_are_left_alone():
    rng = np.random.default_rng(2)
    for behind in (1, 60, 128, 400):
        _run(rng, [100, 29], 2, 2, behind=behind)
    _run(rng, [0, 0], 2, 2, behind=5)


def test_extreme_values():
    rng = np.random.default_rng(3)
    for k, v, q in ((127, 127, 127), (-127, -127, 127), (0, 127, 127), (-128, -128, 127), (-128, -128, -128)):
        qkv = np.empty((200, 3 * 64), np.int8)
        qkv[:, :64], qkv[:, 64:128], qkv[:, 128:] = q, k, v
        qkv[::7, 64:128] = (-qkv[::7, 64:128].astype(np.int16)).clip(-127, 127)
        _run(rng, [150, 50], 1, 1, qkv=qkv, scales=(0.05, 0.04, 0.03, 0.03))


@pytest.mark.parametrize("scales", [(1e-4, 1e-4, 1.0, 1.0), (0.3, 0.3, 1e-6, 1.0), (1.0, 1.0, 5.0, 0.001), (1e-5, 1e-5, 0.02, 0.02),
                                    (0.9, 0.9, 0.1, 0.1), (0.0123, 0.077, 0.5, 0.25),
                                    (0.02, 0.02, 0.1, 0.1), (0.003, 0.003, 0.1, 0.1), (0.04, 0.02, 0.1, 0.05), (0.35, 0.23, 0.1, 0.1)])
def test_scales(scales):
    _run(np.random.default_rng(4), [3, 177, 90], 2, 1, scales=scales)
    _run(np.random.default_rng(5), [300], 1, 1, 50, 3, scales=scales)


def test_too_long_sequences_are_reported():
    rng = np.random.default_rng(6)
    qkv = rng.integers(-127, 128, (260, 3 * 64)).astype(np.int8)
    cu = np.array([0, 200, 260], np.int32)
    out, _ = ctx().ibert_attention_window_i8(dev(qkv), dev(cu), 150, 1, 1, *SC)
    assert ctx().ibert_last_status() == -8
    want = ref.attention_window(qkv, cu, 1, 1, 150, 0, SC, 255)       # at most the last 150 keys
    assert_same(host(out), want)


def test_many_sequences_of_random_lengths():
    rng = np.random.default_rng(7)
    for B, top in ((300, 9), (40, 130), (9, 400)):
        lens = rng.integers(0, top + 1, B).tolist()
        _run(rng, lens, 4, 2, max_len=top)
        _run(rng, lens, 2, 2, 17, 2, max_len=top)


@pytest.mark.parametrize("scales", [(0.05, 0.04, 0.03, 0.01), (0.02, 0.02, 0.1, 0.1), (0.003, 0.003, 0.1, 0.1), (1e-4, 1e-4, 1.0, 1.0)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (70, 3)])
def test_more_ctas_than_the_gpu_holds(scales, window, sinks):
    """600 CTAs: one thread per row, every form of the exponential."""
    _run(np.random.default_rng(9), [300, 1, 250, 64, 0, 365, 200], 60, 4, window, sinks, scales=scales)


def test_sequences_past_the_tensor_are_reported():
    rng = np.random.default_rng(11)
    qkv = rng.integers(-127, 128, (100, 3 * 64)).astype(np.int8)
    out, _ = ctx().ibert_attention_window_i8(dev(qkv), dev(np.array([0, 60, 130], np.int32)), 130, 1, 1, *SC)
    assert ctx().ibert_last_status() == -8
    assert_same(host(out), ref.attention_window(qkv, np.array([0, 60, 100]), 1, 1, 0, 0, SC, 255))


def test_tensors_past_2_gib():
    """Row offsets past 2^31 elements: the last rows of a packed tensor of 2.2e9 bytes."""
    T, heads, kv = 700001, 40, 5
    qkv = torch.randint(-100, 101, (T, (heads + 2 * kv) * 64), dtype=torch.int8, device="cuda")
    lens = np.full(T // 70, 70)
    cu = np.concatenate([[0], np.cumsum(lens), [T]]).astype(np.int32)
    out, _ = ctx().ibert_attention_window_i8(qkv, dev(cu), 100, heads, kv, *SC, window=20, sinks=2)
    ctx().check()
    for b in (0, 5000, len(cu) - 3, len(cu) - 2):
        rows = slice(int(cu[b]), int(cu[b + 1]))
        n = rows.stop - rows.start
        want = ref.attention_window(host(qkv[rows]), np.array([0, n]), heads, kv, 20, 2, SC, 255)
        assert_same(host(out[rows]), want, f"sequence {b}")


def test_near_the_first_operator_of_its_kind():
    """One sequence, its last query: the weighted mean against ibert_attention_i8's divide-first form on the same keys.  There
    every probability is floored to a 255th, so L keys lose up to L/255 of their weight; here each weight is rounded to half
    a 510th of the largest.  With L = 16 keys both are within 16/255 * 2 + 16/510 of the mean's largest magnitude."""
    rng = np.random.default_rng(8)
    L, scales = 16, (0.05, 0.04, 0.03, 0.03)
    qkv = np.clip(np.rint(rng.standard_normal((L, 3 * 64)) * 20), -127, 127).astype(np.int8)
    a, _ = ctx().ibert_attention_i8(dev(qkv), 1, L, 64, 1, *scales)
    b, _ = ctx().ibert_attention_window_i8(dev(qkv), dev(np.array([0, L], np.int32)), L, 1, 1, *scales)
    ctx().check()
    top = np.abs(qkv[:, 128:].astype(int)).max()
    assert np.abs(host(a)[-1].astype(int) - host(b)[-1]).max() <= top * (16 / 255 * 2 + 16 / 510) + 1

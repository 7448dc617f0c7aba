"""Attention of single tokens over a paged cache on the GPU against the plain 64-bit form."""
import numpy as np
import pytest
import torch

import generation_reference as ref
from gpu_util import assert_same, ctx, dev, host
from paper_2101_01321_b200 import binding

pytestmark = pytest.mark.gpu
SC = (0.05, 0.04, 0.03, 0.01)


def _cache(rng, lens, kv, P, max_pages=None, spread=35):
    used = -(-np.asarray(lens) // P)
    n_pages = int(used.sum()) + 3
    ids = rng.permutation(n_pages).astype(np.int32)
    tables = np.full((len(lens), max_pages or max(1, int(used.max()))), -1, np.int32)
    at = 0
    for b, u in enumerate(used):
        tables[b, :u] = ids[at:at + u]
        at += u
    kc, vc = (np.clip(np.rint(rng.standard_normal((n_pages, kv, P, 64)) * spread), -127, 127).astype(np.int8) for _ in range(2))
    return tables, kc, vc


def _run(rng, lens, heads, kv, P, window=0, sinks=0, p_max=255, max_len=None, scales=SC, cache=None, q=None, max_pages=None):
    lens = np.asarray(lens, np.int32)
    tables, kc, vc = cache or _cache(rng, lens, kv, P, max_pages)
    if q is None:
        q = np.clip(np.rint(rng.standard_normal((lens.size, heads * 64)) * 35), -127, 127).astype(np.int8)
    max_len = max_len or max(1, int(lens.max()))
    out, S = ctx().ibert_attention_decode_i8(dev(q), dev(kc), dev(vc), dev(tables), dev(lens), max_len, heads, *scales, window=window,
                                             sinks=sinks, p_max=p_max)
    ctx().check()
    assert S == scales[3]
    want = ref.attention_decode(q, kc, vc, tables, lens, window, sinks, scales, p_max)
    assert_same(host(out), want, "decode")
    return want


@pytest.mark.parametrize("P", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("heads,kv", [(1, 1), (12, 12), (6, 2), (8, 1), (32, 4), (9, 1), (24, 1), (20, 4)])
def test_heads_and_pages(P, heads, kv):
    rng = np.random.default_rng(P + heads)
    want = _run(rng, [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 100, 257, 300], heads, kv, P)
    assert np.abs(want).max() > 5


@pytest.mark.parametrize("n", [1, 7, 32, 255, 256, 257, 511, 513, 1000, 2049, 4100, 9000, 20011])
@pytest.mark.parametrize("p_max", [255, 127])
def test_one_sequence(n, p_max):
    _run(np.random.default_rng(n), [n], 4, 2, 16 if n % 2 else 64, p_max=p_max)


@pytest.mark.parametrize("window", [1, 2, 31, 32, 33, 64, 100, 1000])
@pytest.mark.parametrize("sinks", [0, 1, 4, 31, 32, 33, 70])
def test_window_and_sinks(window, sinks):
    rng = np.random.default_rng(window * 100 + sinks)
    lens = [1, 2, sinks + 1, window, window + 1, window + sinks, window + sinks + 1, window + sinks + 33, 500, 64, 96, 1300]
    _run(rng, lens, 4, 2, 16, window, sinks)


def test_pages_behind_the_window_are_not_looked_at():
    rng = np.random.default_rng(1)
    lens = [400, 333]
    tables, kc, vc = _cache(rng, lens, 2, 16)
    gone = tables.copy()
    for b, n in enumerate(lens):
        gone[b, 1:(n - 50) // 16] = 10 ** 9                    # pages between the sinks and the window
    q = rng.integers(-127, 128, (2, 4 * 64)).astype(np.int8)
    _run(rng, lens, 4, 2, 16, 50, 4, cache=(gone, kc, vc), q=q)
    assert ctx().ibert_last_status() == 0


def test_empty_sequences_give_zero_and_rows_are_independent():
    rng = np.random.default_rng(2)
    want = _run(rng, [0, 5, 0, 40, 0], 4, 4, 16)
    assert not want[[0, 2, 4]].any() and want[[1, 3]].any()
    _run(rng, [0], 2, 1, 16, max_len=700, max_pages=64)


def test_batches_of_ragged_lengths():
    rng = np.random.default_rng(3)
    for B, top in ((3, 5000), (40, 900), (200, 130)):
        lens = rng.integers(0, top + 1, B)
        _run(rng, lens, 6, 3, 32, max_len=max(int(lens.max()), top), max_pages=-(-top // 32) + 1)


def test_longest_visible_context():
    rng = np.random.default_rng(4)
    _run(rng, [65536], 2, 1, 256)
    _run(rng, [65530], 8, 1, 128)
    _run(rng, [70001], 3, 1, 64, window=65000, sinks=536)


def test_extreme_values():
    """All keys alike, scores at both ends of their range, and -128, which only a cache written by others holds."""
    rng = np.random.default_rng(5)
    for k, v, q in ((127, 127, 127), (-127, -127, 127), (0, 127, 127), (-128, -128, 127), (-128, -128, -128)):
        tables, kc, vc = _cache(rng, [300], 1, 16)
        kc[:], vc[:] = k, v
        kc[tables[0, 3], 0, 5] = -kc[tables[0, 3], 0, 5].clip(-127)
        _run(rng, [300], 2, 1, 16, cache=(tables, kc, vc), q=np.full((1, 128), q, np.int8), scales=(0.05, 0.04, 0.03, 0.03))


@pytest.mark.parametrize("scales", [(1e-4, 1e-4, 1.0, 1.0), (0.3, 0.3, 1e-6, 1.0), (1.0, 1.0, 5.0, 0.001), (1e-5, 1e-5, 0.02, 0.02),
                                    (0.9, 0.9, 0.1, 0.1), (0.0123, 0.077, 0.5, 0.25),
                                    (0.02, 0.02, 0.1, 0.1), (0.003, 0.003, 0.1, 0.1), (0.04, 0.02, 0.1, 0.05), (0.35, 0.23, 0.1, 0.1)])
def test_scales(scales):
    _run(np.random.default_rng(6), [3, 77, 500], 4, 2, 16, scales=scales)


def test_bad_pages_and_lengths_are_reported_and_harmless():
    rng = np.random.default_rng(7)
    lens = [100, 64, 40]
    tables, kc, vc = _cache(rng, lens, 2, 16)
    tables[0, 2], tables[1, 0], tables[1, 3] = -1, kc.shape[0], 2 ** 31 - 1
    q = rng.integers(-127, 128, (3, 4 * 64)).astype(np.int8)
    out, _ = ctx().ibert_attention_decode_i8(dev(q), dev(kc), dev(vc), dev(tables), dev(np.array(lens, np.int32)), 100, 4, *SC)
    assert ctx().ibert_last_status() == -8
    assert_same(host(out), ref.attention_decode(q, kc, vc, tables, lens, 0, 0, SC, 255), "keys on bad pages are left out")
    tables[:] = -5
    out, _ = ctx().ibert_attention_decode_i8(dev(q), dev(kc), dev(vc), dev(tables), dev(np.array(lens, np.int32)), 100, 4, *SC)
    assert ctx().ibert_last_status() == -8 and not host(out).any()
    tables, kc, vc = _cache(rng, [112, 64, 48], 2, 16)
    for odd, taken in (([101, 64, 40], [100, 64, 40]), ([2 ** 31 - 1, -5, 40], [100, 0, 40])):
        out, _ = ctx().ibert_attention_decode_i8(dev(q), dev(kc), dev(vc), dev(tables), dev(np.array(odd, np.int32)), 100, 4, *SC)
        assert ctx().ibert_last_status() == -8
        assert_same(host(out), ref.attention_decode(q, kc, vc, tables, taken, 0, 0, SC, 255))


def test_rows_of_a_packed_step():
    """Row offsets of a step in which some sequences get no token and others several: the last new token's row of each is
    computed, all other rows stay; rows outside the tensor are left out."""
    rng = np.random.default_rng(10)
    new = np.array([1, 0, 3, 1, 0, 40, 1])
    lens = np.array([50, 20, 33, 1, 0, 40, 700], np.int32)
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    for heads, kv in ((4, 2), (6, 1)):
        tables, kc, vc = _cache(rng, lens, kv, 16)
        T = int(cu[-1]) + 4
        q = rng.integers(-127, 128, (T, heads * 64)).astype(np.int8)
        out = torch.full((T, heads * 64), 55, dtype=torch.int8, device="cuda")

        def call(offsets):
            out.fill_(55)
            ctx().ibert_attention_decode_i8(dev(q), dev(kc), dev(vc), dev(tables), dev(lens), 700, heads, *SC, out=out, cu_seqlens=dev(offsets))
            return host(out), ctx().ibert_last_status()

        want = np.full((T, heads * 64), 55, np.int8)
        has = np.flatnonzero(new)
        want[cu[has + 1] - 1] = ref.attention_decode(q[cu[has + 1] - 1], kc, vc, tables[has], lens[has], 0, 0, SC, 255)
        got, status = call(cu)
        assert status == 0
        assert_same(got, want)
        bad = cu.copy()
        bad[7] = T + 1                                               # the last sequence's row does not exist
        want[cu[7] - 1] = 55
        got, status = call(bad)
        assert status == -8
        assert_same(got, want)


def test_many_calls_agree():
    rng = np.random.default_rng(8)
    tables, kc, vc = _cache(rng, [3000, 100], 1, 16)
    d = [dev(a) for a in (rng.integers(-127, 128, (2, 8 * 64)).astype(np.int8), kc, vc, tables, np.array([3000, 100], np.int32))]
    first, _ = ctx().ibert_attention_decode_i8(*d, 3000, 8, *SC)
    for _ in range(30):
        out, _ = ctx().ibert_attention_decode_i8(*d, 3000, 8, *SC)
        assert torch.equal(out, first)


def test_cache_past_4_gib():
    """Offsets into a cache of more than 2^32 bytes."""
    n_pages, P, kv = 40000, 256, 8                                   # 5.2e9 bytes each
    kc = torch.zeros(n_pages, kv, P, 64, dtype=torch.int8, device="cuda")
    vc = torch.zeros_like(kc)
    rng = np.random.default_rng(9)
    pages = np.array([n_pages - 1, 2, n_pages - 2], np.int32)
    small_k, small_v = (rng.integers(-127, 128, (3, kv, P, 64)).astype(np.int8) for _ in range(2))
    kc[dev(pages.astype(np.int64))], vc[dev(pages.astype(np.int64))] = dev(small_k), dev(small_v)
    q = rng.integers(-40, 41, (1, 16 * 64)).astype(np.int8)
    out, _ = ctx().ibert_attention_decode_i8(dev(q), kc, vc, dev(pages[None]), dev(np.array([700], np.int32)), 700, 16, *SC)
    ctx().check()
    assert_same(host(out), ref.attention_decode(q, small_k, small_v, np.array([[0, 1, 2]]), [700], 0, 0, SC, 255))

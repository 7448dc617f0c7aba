"""Variants of the generation kernels that their callers choose by size: several heads per group of lanes in the heads' pass,
and the two forms of the paged attention with whole and split groups of query heads."""
import numpy as np
import pytest

import generation_reference as ref
from gpu_util import assert_same, ctx, dev, host
from paper_2101_01321_b200 import binding

pytestmark = pytest.mark.gpu
SC = (0.05, 0.04, 0.03, 0.01)


# ----------------------------------------------------------------------------- heads' pass
@pytest.mark.parametrize("T,heads,kv,P", [(2500, 21, 7, 16), (1900, 21, 7, 64), (9001, 15, 5, 16), (1301, 34, 1, 256)])
@pytest.mark.parametrize("bits,norm", [(8, True), (8, False), (16, True), (16, False)])
@pytest.mark.parametrize("rot,interleaved,with_kv,cache", [(24, False, True, True), (64, False, False, True), (48, True, True, True),
                                                          (0, False, False, True), (56, True, True, False)])
def test_several_heads_one_after_the_other(T, heads, kv, P, bits, norm, rot, interleaved, with_kv, cache):
    """The head count per group of lanes is tokens * heads / (128 SMs), here 2 to 8, mostly with an uneven last part."""
    rng = np.random.default_rng(T + rot + bits)
    top = 127 if bits == 8 else 32767
    n = heads + 2 * kv
    x = np.clip(np.rint(rng.standard_normal((T, n * 64)) * (30 if bits == 8 else 5000)), -top, top).astype(np.int8 if bits == 8 else np.int16)
    S_in = 1 / 30 if bits == 8 else 1 / 5000
    gq, gk = (1 + 0.3 * rng.standard_normal((2, 64))) if norm else (None, None)
    rope = binding.ibert_rope_rows(binding.ibert_rope_frequencies(rot), 300) if rot else None
    pos = rng.integers(0, 300, T).astype(np.int32)
    args = dict(gamma_q=gq, gamma_k=gk, interleaved=interleaved, with_kv=with_kv)
    if rot:
        args.update(rope=dev(rope), positions=dev(pos))
    pages = -(-T // P) + 2
    kc, vc = (rng.integers(-127, 128, (pages, kv, P, 64)).astype(np.int8) for _ in range(2))
    slots = rng.permutation(pages * P)[:T].astype(np.int32)
    slots[rng.random(T) < 0.1] = -1
    dk, dv = dev(kc), dev(vc)
    if cache:
        args.update(slots=dev(slots), k_cache=dk, v_cache=dv)
    out, _ = ctx().ibert_qkv_rope_i8(dev(x), S_in, heads, kv, 0.05, 0.04, 0.03, **args)
    ctx().check()
    q, k, v = ref.qkv_rope(x, heads, kv, S_in, 0.05, 0.04, 0.03, gq, gk, rope, pos, interleaved)
    assert_same(host(out), (np.concatenate([q, k, v], 1) if with_kv else q).reshape(T, -1), "out")
    if cache:
        at = np.flatnonzero(slots >= 0)
        kc[slots[at] // P, :, slots[at] % P], vc[slots[at] // P, :, slots[at] % P] = k[at], v[at]
    assert_same(host(dk), kc, "k_cache")
    assert_same(host(dv), vc, "v_cache")


# ----------------------------------------------------------------------------- paged attention
GROUPS = pytest.mark.parametrize("heads,kv", [(4, 2), (3, 1), (8, 1), (9, 1)])     # scores kept; computed twice; a whole group; two pieces


def _cache(rng, lens, kv, P, spread=35):
    used = -(-np.asarray(lens) // P)
    n_pages = int(used.sum()) + 3
    ids, at = rng.permutation(n_pages).astype(np.int32), np.concatenate([[0], np.cumsum(used)])
    tables = np.full((len(lens), max(1, int(used.max()))), -1, np.int32)
    for b, u in enumerate(used):
        tables[b, :u] = ids[at[b]:at[b + 1]]
    return (tables,) + tuple(np.clip(np.rint(rng.standard_normal((n_pages, kv, P, 64)) * spread), -127, 127).astype(np.int8) for _ in range(2))


def _decode(q, cache, lens, heads, max_len, status=0, window=0, sinks=0, p_max=255, scales=SC, taken=None):
    tables, kc, vc = cache
    out, _ = ctx().ibert_attention_decode_i8(dev(q), dev(kc), dev(vc), dev(tables), dev(np.asarray(lens, np.int32)), max_len, heads, *scales,
                                             window=window, sinks=sinks, p_max=p_max)
    assert ctx().ibert_last_status() == status
    want = ref.attention_decode(q, kc, vc, tables, lens if taken is None else taken, window, sinks, scales, p_max)
    assert_same(host(out), want, "decode")


def _q(rng, B, heads):
    return np.clip(np.rint(rng.standard_normal((B, heads * 64)) * 35), -127, 127).astype(np.int8)


@GROUPS
@pytest.mark.parametrize("scales", [(1e-4, 1e-4, 1.0, 1.0), (0.3, 0.3, 1e-6, 1.0), (1.0, 1.0, 5.0, 0.001), (1e-5, 1e-5, 0.02, 0.02),
                                    (0.9, 0.9, 0.1, 0.1), (0.0123, 0.077, 0.5, 0.25), (0.02, 0.02, 0.1, 0.1), (0.003, 0.003, 0.1, 0.1),
                                    (0.04, 0.02, 0.1, 0.05), (0.35, 0.23, 0.1, 0.1)])
@pytest.mark.parametrize("p_max", [255, 127])
def test_every_form_of_the_exponential(heads, kv, scales, p_max):
    rng = np.random.default_rng(heads)
    lens = [3, 77, 500, 1111]
    _decode(_q(rng, 4, heads), _cache(rng, lens, kv, 16), lens, heads, 1111, p_max=p_max, scales=scales)


@GROUPS
@pytest.mark.parametrize("window", [1, 31, 33, 100, 1000])
@pytest.mark.parametrize("sinks", [0, 1, 4, 33, 70])
def test_windows(heads, kv, window, sinks):
    rng = np.random.default_rng(window * 100 + sinks)
    lens = [1, 2, sinks + 1, window, window + 1, window + sinks, window + sinks + 33, 500, 96, 1300, 0]
    _decode(_q(rng, len(lens), heads), _cache(rng, lens, kv, 16), lens, heads, 1300, window=window, sinks=sinks)


@GROUPS
@pytest.mark.parametrize("k,v,q", [(127, 127, 127), (-127, -127, 127), (0, 127, 127), (-128, -128, 127), (-128, -128, -128)])
def test_ends_of_the_range(heads, kv, k, v, q):
    tables, kc, vc = _cache(np.random.default_rng(5), [300], kv, 16)
    kc[:], vc[:] = k, v
    kc[tables[0, 3], 0, 5] = -kc[tables[0, 3], 0, 5].clip(-127)
    _decode(np.full((1, heads * 64), q, np.int8), (tables, kc, vc), [300], heads, 300, scales=(0.05, 0.04, 0.03, 0.03))


@GROUPS
def test_keys_on_bad_pages_are_left_out(heads, kv):
    rng = np.random.default_rng(7)
    lens = [100, 64, 40, 700]
    tables, kc, vc = _cache(rng, lens, kv, 16)
    tables[0, 2], tables[1, 0], tables[1, 3], tables[3, 5:40:2] = -1, kc.shape[0], 2 ** 31 - 1, -7
    q = _q(rng, 4, heads)
    _decode(q, (tables, kc, vc), lens, heads, 700, status=-8)
    _decode(q, (tables, kc, vc), lens, heads, 700, status=-8, window=90, sinks=40)
    tables[:] = -5
    _decode(q, (tables, kc, vc), lens, heads, 700, status=-8)
    cache = _cache(rng, [112, 64, 48, 16], kv, 16)
    for odd, taken in (([101, 64, 40, 0], [100, 64, 40, 0]), ([2 ** 31 - 1, -5, 40, -2 ** 31], [100, 0, 40, 0])):
        _decode(q, cache, odd, heads, 100, status=-8, taken=taken)


@GROUPS
@pytest.mark.parametrize("P", [16, 256])
def test_generous_bounds_change_nothing(heads, kv, P):
    """A bound on the lengths far above those that occur, as a captured step has it: other cluster widths, same results."""
    rng = np.random.default_rng(11)
    lens = [1, 300, 777, 0, 40]
    tables, kc, vc = _cache(rng, lens, kv, P)
    wide = np.full((5, 65536 // P), -1, np.int32)
    wide[:, :tables.shape[1]] = tables
    q = _q(rng, 5, heads)
    for max_len in (777, 1024, 8192, 65536):
        _decode(q, (wide, kc, vc), lens, heads, max_len)

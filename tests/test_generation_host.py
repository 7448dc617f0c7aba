"""Operators for generation, what needs no GPU: the rotation tables, and every call that is refused before a launch."""
import ctypes as C

import numpy as np
import pytest

ARG, SHAPE, SCALE, ALIGN = -1, -2, -3, -4


@pytest.fixture(scope="module")
def lib():
    from paper_2101_01321_b200 import build, binding
    build.build()
    return binding.lib()


# A context that is never looked into: every call below is refused before that
CTX = C.create_string_buffer(1 << 16)
MEM = C.create_string_buffer(1 << 13)
P16 = (C.addressof(MEM) + 255) // 256 * 256
P = [P16 + 256 * i for i in range(8)]          # arrays that start at addresses of their own


def _slots(lib, **kw):
    a = dict(ctx=CTX, lens=P[0], new=P[1], tables=P[2], B=4, max_pages=8, page=16, free=P[3], cap=64, n_free=P[4], max_tokens=16,
             lens_out=P[0], n_out=P[4], cu=P[5], slots=P[6], positions=P[7]) | kw
    return lib.ibert_kv_slots(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(ctx=None), ARG), (dict(B=-1), ARG), (dict(max_tokens=-1), ARG), (dict(cap=-1), ARG), (dict(max_pages=-1), ARG),
    (dict(page=0), SHAPE), (dict(page=8), SHAPE), (dict(page=24), SHAPE), (dict(page=512), SHAPE), (dict(B=8193), SHAPE),
    (dict(max_pages=1 << 27), SHAPE), (dict(max_pages=1 << 22, B=1024), SHAPE), (dict(max_tokens=1 << 31), SHAPE),
    (dict(cap=1 << 31), SHAPE)] + [
    (dict(lens_out=P[1]), ARG), (dict(slots=P[7]), ARG), (dict(cu=P[0]), ARG), (dict(positions=P[4]), ARG), (dict(free=P[2]), ARG)] + [
    ({n: None}, ARG) for n in ("lens", "new", "tables", "free", "n_free", "lens_out", "n_out", "cu", "slots", "positions")] + [
    ({n: P16 + 2}, ALIGN) for n in ("lens", "new", "tables", "free", "n_free", "lens_out", "n_out", "cu", "slots", "positions")])
def test_kv_slots_refuses(lib, kw, code):
    assert _slots(lib, **kw) == code


def _rope(lib, ctx=CTX, qkv=P16, T=4, positions=P16, with_kv=1, out=P[1], slots=None, k=None, v=None, **kw):
    from paper_2101_01321_b200.binding import RopeDesc
    gamma = np.ones(64)
    d = RopeDesc(4, 2, 8, 64, 0, 16, 8, 100, P16, None, None, 0.03, 0.03, 0.03, 0.03)
    for n, x in kw.items():
        setattr(d, n, gamma.ctypes.data if x == "ones" else x)
    return lib.ibert_qkv_rope_i8(ctx, C.byref(d), qkv, T, positions, with_kv, out, slots, k, v, None)


CACHE = dict(slots=P16, k=P[2], v=P[3])


@pytest.mark.parametrize("kw,code", [
    (dict(ctx=None), ARG), (dict(T=-1), ARG), (dict(with_kv=2), ARG), (dict(interleaved=2), ARG), (dict(qkv=None), ARG),
    (dict(out=None), ARG), (dict(positions=None), ARG), (dict(rope=None), ARG), (dict(max_pos=0), ARG), (dict(gamma_q="ones"), ARG),
    (dict(gamma_k="ones"), ARG), (dict(slots=P16), ARG), (dict(k=P[2], v=P[3]), ARG), (dict(slots=P16, k=P[2]), ARG), (dict(out=P16), ARG),
    (dict(CACHE, v=P[2]), ARG), (dict(CACHE, k=P[1]), ARG),
    (dict(heads=0), SHAPE), (dict(kv_heads=0), SHAPE), (dict(kv_heads=3), SHAPE), (dict(in_bits=32), SHAPE), (dict(rot_dim=4), SHAPE),
    (dict(rot_dim=72), SHAPE), (dict(rot_dim=-8), SHAPE), (dict(heads=4098), SHAPE), (dict(T=1 << 31), SHAPE),
    (dict(CACHE, page_size=48), SHAPE), (dict(CACHE, n_pages=-1), SHAPE), (dict(CACHE, n_pages=1 << 27), SHAPE),
    (dict(qkv=P16 + 4), ALIGN), (dict(out=P16 + 8), ALIGN), (dict(rope=P16 + 8), ALIGN), (dict(positions=P16 + 1), ALIGN),
    (dict(CACHE, k=P16 + 8), ALIGN), (dict(CACHE, v=P16 + 8), ALIGN), (dict(CACHE, slots=P16 + 2), ALIGN),
    (dict(S_in=0.0), SCALE), (dict(S_q=-1.0), SCALE), (dict(S_k=float("nan")), SCALE), (dict(S_v=float("inf")), SCALE),
    (dict(gamma_q="ones", gamma_k="ones", S_q=1e-9), SCALE)])
def test_qkv_rope_refuses(lib, kw, code):
    assert _rope(lib, **kw) == code


def test_no_tokens_are_no_work(lib):
    assert _rope(lib, T=0, qkv=None, out=None, positions=None) == 0
    assert _decode(lib, B=0, rows=0, q=None, out=None) == 0
    assert _decode(lib, cu=P16, rows=0, q=None, out=None) == 0


def _desc(kw):
    """The fields of ibert_attention_desc out of kw, and the rest."""
    from paper_2101_01321_b200.binding import AttentionDesc
    names = [n for n, _ in AttentionDesc._fields_]
    f = dict(heads=4, kv_heads=2, max_len=100, window=0, sinks=0, p_max=255, page_size=16, max_pages=8, n_pages=16, S_q=0.05, S_k=0.05,
             S_v=0.05, S_ctx=0.02) | {n: x for n, x in kw.items() if n in names}
    return C.byref(AttentionDesc(*(f[n] for n in names))), {n: x for n, x in kw.items() if n not in names}


def _decode(lib, **kw):
    desc, kw = _desc(kw)
    a = dict(ctx=CTX, desc=desc, q=P16, k=P[1], v=P[2], tables=P16, lens=P16, B=2, cu=None, rows=2, out=P[3], S_ret=None) | kw
    return lib.ibert_attention_decode_i8(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(ctx=None), ARG), (dict(B=-1), ARG), (dict(window=-1), ARG), (dict(sinks=-1), ARG), (dict(p_max=100), ARG),
    (dict(max_len=0), SHAPE), (dict(max_len=129), SHAPE), (dict(heads=0), SHAPE), (dict(kv_heads=0), SHAPE), (dict(heads=3), SHAPE),
    (dict(page_size=40), SHAPE), (dict(desc=None), ARG), (dict(n_pages=-1), SHAPE), (dict(n_pages=1 << 27), SHAPE), (dict(max_len=65537, max_pages=1 << 20), SHAPE),
    (dict(max_len=80000, max_pages=1 << 20, window=65536, sinks=1), SHAPE), (dict(B=1 << 23, rows=1 << 23), SHAPE),
    (dict(out=P16), ARG), (dict(out=P[1]), ARG), (dict(rows=3), SHAPE), (dict(cu=P16, rows=-1), SHAPE), (dict(cu=P16, rows=1 << 29), SHAPE), (dict(cu=P16 + 2), ALIGN), (dict(B=-1, rows=-1), ARG),
    (dict(max_len=(1 << 31) - 256, max_pages=1 << 27, window=5), SHAPE),
    (dict(S_q=0.0), SCALE), (dict(S_ctx=float("inf")), SCALE), (dict(S_q=2.0, S_k=2.0), SCALE), (dict(S_q=1.5, S_k=1.4), SCALE),
    (dict(q=P16 + 8), ALIGN), (dict(k=P16 + 8), ALIGN), (dict(v=P16 + 8), ALIGN), (dict(out=P16 + 8), ALIGN), (dict(tables=P16 + 2), ALIGN),
    (dict(lens=P16 + 2), ALIGN)] + [({n: None}, ARG) for n in ("q", "k", "v", "tables", "lens", "out")])
def test_attention_decode_refuses(lib, kw, code):
    assert _decode(lib, **kw) == code


def _window(lib, **kw):
    desc, kw = _desc(kw)
    a = dict(ctx=CTX, desc=desc, qkv=P16, cu=P16, B=2, T=50, out=P[1], S_ret=None) | kw
    return lib.ibert_attention_window_i8(*a.values())


@pytest.mark.parametrize("kw,code", [
    (dict(ctx=None), ARG), (dict(B=-1), ARG), (dict(T=-1), ARG), (dict(window=-1), ARG), (dict(sinks=-1), ARG), (dict(p_max=1), ARG),
    (dict(qkv=None), ARG), (dict(cu=None), ARG), (dict(out=None), ARG), (dict(out=P16), ARG), (dict(max_len=0), SHAPE), (dict(max_len=65537), SHAPE),
    (dict(max_len=70000, window=65000, sinks=537), SHAPE), (dict(max_len=(1 << 31) - 256, window=5), SHAPE), (dict(heads=0), SHAPE), (dict(heads=5), SHAPE), (dict(kv_heads=0), SHAPE),
    (dict(T=(1 << 31) - 256), SHAPE), (dict(S_k=0.0), SCALE), (dict(S_q=1.5, S_k=1.4), SCALE), (dict(S_v=float("nan")), SCALE),
    (dict(qkv=P16 + 8), ALIGN), (dict(out=P16 + 8), ALIGN), (dict(cu=P16 + 2), ALIGN)])
def test_attention_window_refuses(lib, kw, code):
    assert _window(lib, **kw) == code


def test_no_rows_are_no_work(lib):
    assert _window(lib, T=0, qkv=None, out=None) == 0
    assert _window(lib, B=0, T=5) == 0


@pytest.mark.parametrize("S", [0.2, 0.05, 7.3e-3, 1.1e-3, 4e-4, 2.5e-4, 1.77e-4, 1.2e-4, 9e-5, 5e-5, 3e-5, 1e-6, 1.25e-9])
def test_quotients_of_the_exponential_hold_for_every_distance(lib, S):
    assert lib.ibert_selftest_exp_division(S, None) == 0


# ----------------------------------------------------------------------------- rotation tables
@pytest.mark.parametrize("rot", [8, 16, 48, 64])
@pytest.mark.parametrize("pos0,n,factor", [(0, 50, 1.0), (131000, 9, 1.0), (7, 3, 1.37), (5, 0, 1.0)])
def test_rope_rows_are_the_rounded_cosines(lib, rot, pos0, n, factor):
    from paper_2101_01321_b200 import binding
    f = binding.ibert_rope_frequencies(rot)
    assert np.allclose(f, 10000.0 ** (-np.arange(0, rot, 2) / rot), rtol=1e-15)
    rows = binding.ibert_rope_rows(f, n, factor, pos0)
    a = (pos0 + np.arange(n))[:, None].astype(np.longdouble) * f.astype(np.longdouble)
    # half a step of rounding; the angle in double precision is off by a relative 2^-53: 131008 rad by 1.5e-11, i.e. 2.4e-7 steps
    for i, fn in ((0, np.cos), (1, np.sin)):
        assert np.abs(rows[:, i::2] - fn(a) * 16384 * factor).max(initial=0) <= 0.5 + 1e-6
    assert (rows.astype(np.int64)[:, 0::2] ** 2 + rows.astype(np.int64)[:, 1::2] ** 2).max(initial=0) < 2 ** 30


def test_rope_frequencies_of_longer_contexts(lib):
    from paper_2101_01321_b200 import binding
    base = binding.ibert_rope_frequencies(64)
    assert np.allclose(binding.ibert_rope_frequencies(64, stretch=4.0), base / 4.0, rtol=1e-15)
    f = binding.ibert_rope_frequencies(64, stretch=8.0, trained_len=4096, low_turns=1.0, high_turns=32.0)
    turns = 4096 * base / (2 * np.pi)
    assert np.array_equal(f[turns >= 32], base[turns >= 32]) and np.allclose(f[turns <= 1], base[turns <= 1] / 8, rtol=1e-15)
    mid = (turns > 1) & (turns < 32)
    keep = (turns[mid] - 1) / 31
    assert mid.sum() > 3 and np.allclose(f[mid], base[mid] * (keep + (1 - keep) / 8), rtol=1e-14)


@pytest.mark.parametrize("args,code", [
    ((12, 1e4, 1.0, 0.0, 1.0, 2.0), SHAPE), ((72, 1e4, 1.0, 0.0, 1.0, 2.0), SHAPE), ((0, 1e4, 1.0, 0.0, 1.0, 2.0), SHAPE),
    ((64, 1.0, 1.0, 0.0, 1.0, 2.0), ARG), ((64, 1e4, 0.5, 0.0, 1.0, 2.0), ARG), ((64, 1e4, 1.0, -1.0, 1.0, 2.0), ARG),
    ((64, 1e4, 2.0, 100.0, 2.0, 2.0), ARG), ((64, 1e4, 2.0, 100.0, -1.0, 2.0), ARG), ((64, float("nan"), 2.0, 100.0, 1.0, 2.0), ARG)])
def test_rope_frequencies_refuse(lib, args, code):
    assert lib.ibert_rope_frequencies(*args, P16) == code
    assert lib.ibert_rope_frequencies(64, 1e4, 1.0, 0.0, 1.0, 2.0, None) == ARG


def test_rope_rows_refuse(lib):
    f = np.ones(32)
    call = lambda f=f.ctypes.data, rot=64, pos0=0, n=1, factor=1.0, rows=P16: lib.ibert_rope_rows(f, rot, pos0, n, factor, rows)  # noqa: E731
    assert call() == 0
    assert call(f=None) == ARG and call(rows=None) == ARG and call(n=-1) == ARG and call(pos0=-1) == ARG
    assert call(rot=20) == SHAPE and call(rot=0) == SHAPE
    assert call(factor=0.0) == ARG and call(factor=2.0) == ARG and call(factor=float("nan")) == ARG
    f[3] = np.inf
    assert call() == ARG

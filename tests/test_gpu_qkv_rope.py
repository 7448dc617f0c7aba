"""Norm of the heads + rotary positions + int8 + cache on the GPU against the plain 64-bit form, and the plain form
against real arithmetic."""
import numpy as np
import pytest
import torch

import generation_reference as ref
from gpu_util import assert_same, ctx, dev, host
from paper_2101_01321_b200 import binding

pytestmark = pytest.mark.gpu
SC = dict(S_q=0.05, S_k=0.04, S_v=0.03)


def _x(rng, T, n, bits, S=None):
    top = 127 if bits == 8 else 32767
    x = rng.standard_normal((T, n, 64)) * (30 if bits == 8 else 5000) * np.exp(rng.standard_normal((T, n, 1)))
    return np.clip(np.rint(x), -top, top).astype(np.int8 if bits == 8 else np.int16).reshape(T, n * 64), (1 / 30 if bits == 8 else 1 / 5000)


def _run(x, S_in, heads, kv, norm, rope, positions, interleaved, with_kv, cache, P=16, seed=0, sc=SC):
    """The GPU's call and the plain form on the same inputs, compared whole."""
    rng = np.random.default_rng(seed + 1)
    T = x.shape[0]
    gq, gk = norm
    args = dict(gamma_q=gq, gamma_k=gk, interleaved=interleaved, with_kv=with_kv)
    if rope is not None:
        args.update(rope=dev(rope), positions=dev(positions))
    if cache:
        pages = -(-T // P) + 2
        kc, vc = (rng.integers(-127, 128, (pages, kv, P, 64)).astype(np.int8) for _ in range(2))
        slots = rng.permutation(pages * P)[:T].astype(np.int32)
        slots[rng.random(T) < 0.2] = -1
        dk, dv = dev(kc), dev(vc)
        args.update(slots=dev(slots), k_cache=dk, v_cache=dv)
    out, S = ctx().ibert_qkv_rope_i8(dev(x), S_in, heads, kv, sc["S_q"], sc["S_k"], sc["S_v"], **args)
    ctx().check()
    assert S == (sc["S_q"], sc["S_k"], sc["S_v"])
    q, k, v = ref.qkv_rope(x, heads, kv, S_in, sc["S_q"], sc["S_k"], sc["S_v"], gq, gk, rope, positions, interleaved)
    assert_same(host(out), (np.concatenate([q, k, v], 1) if with_kv else q).reshape(T, -1), "out")
    if cache:
        for t in np.flatnonzero(slots >= 0):
            kc[slots[t] // P, :, slots[t] % P], vc[slots[t] // P, :, slots[t] % P] = k[t], v[t]
        assert_same(host(dk), kc, "k_cache")
        assert_same(host(dv), vc, "v_cache")
    return q, k, v


def _gammas(rng):
    return 1 + 0.3 * rng.standard_normal(64), 1 + 0.3 * rng.standard_normal(64)


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("rot,interleaved", [(0, False), (8, False), (16, True), (24, False), (48, True), (56, False), (64, False), (64, True)])
def test_matches_the_plain_form(bits, norm, rot, interleaved):
    rng = np.random.default_rng(rot + bits)
    T, heads, kv = 45, 6, 2
    x, S_in = _x(rng, T, heads + 2 * kv, bits)
    rope = binding.ibert_rope_rows(binding.ibert_rope_frequencies(rot), 300) if rot else None
    for with_kv, cache in ((True, False), (False, True), (True, True), (False, False)):
        _run(x, S_in, heads, kv, _gammas(rng) if norm else (None, None), rope, rng.integers(0, 300, T).astype(np.int32), interleaved,
             with_kv, cache, P=32, seed=rot)


@pytest.mark.parametrize("T,heads,kv", [(1, 1, 1), (1, 12, 12), (2, 3, 1), (7, 16, 16), (33, 32, 4), (300, 12, 12), (1001, 5, 5)])
@pytest.mark.parametrize("bits", [8, 16])
def test_token_and_head_counts(T, heads, kv, bits):
    rng = np.random.default_rng(T)
    x, S_in = _x(rng, T, heads + 2 * kv, bits)
    rope = binding.ibert_rope_rows(binding.ibert_rope_frequencies(64), 2048)
    _run(x, S_in, heads, kv, _gammas(rng), rope, (np.arange(T) * 7 % 2048).astype(np.int32), False, True, True, P=16, seed=T)


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("fill", ["zero", "one", "top", "bottom", "lowest", "spike", "ones"])
def test_extreme_heads(bits, fill):
    """Heads of zeros, one small value, the ends of the range and the container's lowest value (outside the format)."""
    top = 127 if bits == 8 else 32767
    x = np.zeros((3, 3 * 64), np.int8 if bits == 8 else np.int16)
    rng = np.random.default_rng(4)
    if fill == "one":
        x[:, 5::64] = 1
    elif fill == "ones":
        x[:] = 1
    elif fill == "top":
        x[:] = top
    elif fill == "bottom":
        x[:] = -top
    elif fill == "lowest":
        x[:] = -top - 1
    elif fill == "spike":
        x[:, 7::64] = -top
        x[:, 9::64] = 1
    rope = binding.ibert_rope_rows(binding.ibert_rope_frequencies(64), 64)
    for norm in (_gammas(rng), (np.zeros(64), np.full(64, -50.0)), (np.full(64, 1e-6), np.r_[40.0, np.full(63, 1e-3)]), (None, None)):
        _run(x, 1.0 / top, 1, 1, norm, rope, np.array([0, 1, 63], np.int32), False, True, True)


@pytest.mark.parametrize("S_q", [1e-4, 0.01, 3.0, 1000.0])
def test_scales(S_q):
    rng = np.random.default_rng(8)
    x, S_in = _x(rng, 9, 4, 16)
    rope = binding.ibert_rope_rows(binding.ibert_rope_frequencies(64), 64, 1.9)
    sc = dict(S_q=S_q, S_k=S_q / 3, S_v=S_q)
    for norm in (_gammas(rng), (None, None)):
        _run(x, S_in, 2, 1, norm, rope, np.arange(9, dtype=np.int32), True, True, False, sc=sc)


def test_multipliers_far_above_one():
    """Without a norm, scales of the result so fine that almost everything is clamped (shifts below 17)."""
    rng = np.random.default_rng(12)
    for bits in (8, 16):
        x, S_in = _x(rng, 9, 4, bits)
        x[0] = 0
        x[1, ::2] = 1
        _run(x, S_in, 2, 1, (None, None), None, None, False, True, False, sc=dict(S_q=1e-7, S_k=3e-8, S_v=1e-6))


def test_tensors_past_2_gib():
    T, heads, kv = 700001, 40, 5
    n = (heads + 2 * kv) * 64
    qkv = torch.randint(-100, 101, (T, n), dtype=torch.int8, device="cuda")
    rng = np.random.default_rng(13)
    gq, gk = _gammas(rng)
    rope = binding.ibert_rope_rows(binding.ibert_rope_frequencies(64), 100)
    pos = (np.arange(T) % 100).astype(np.int32)
    out, _ = ctx().ibert_qkv_rope_i8(qkv, 0.01, heads, kv, *SC.values(), gq, gk, rope=dev(rope), positions=dev(pos))
    ctx().check()
    for rows in (slice(0, 3), slice(699040, 699060), slice(T - 5, T)):
        q, k, v = ref.qkv_rope(host(qkv[rows]), heads, kv, 0.01, *SC.values(), gq, gk, rope, pos[rows], False)
        assert_same(host(out[rows]), np.concatenate([q, k, v], 1).reshape(-1, n))


def test_long_positions_and_stretched_frequencies():
    rng = np.random.default_rng(2)
    f = binding.ibert_rope_frequencies(64, 500000.0, 8.0, 8192.0, 1.0, 4.0)
    rope = binding.ibert_rope_rows(f, 131072)
    x, S_in = _x(rng, 64, 4, 16)
    _run(x, S_in, 2, 1, _gammas(rng), rope, rng.integers(100000, 131072, 64).astype(np.int32), False, True, False)


def test_out_of_range_positions_and_slots_are_reported_and_harmless():
    rng = np.random.default_rng(6)
    x, S_in = _x(rng, 6, 3, 8)
    rope = binding.ibert_rope_rows(binding.ibert_rope_frequencies(64), 50)
    kc = torch.zeros(2, 1, 16, 64, dtype=torch.int8, device="cuda")
    vc = torch.zeros_like(kc)

    def call(positions, slots):
        out, _ = ctx().ibert_qkv_rope_i8(dev(x), S_in, 1, 1, 0.05, 0.05, 0.05, rope=dev(rope), positions=dev(np.array(positions, np.int32)),
                                         slots=dev(np.array(slots, np.int32)), k_cache=kc, v_cache=vc)
        return host(out), ctx().ibert_last_status()

    good, st = call([0, 1, 2, 0, 4, 49], [-1, 3, 31, -1, 7, 0])
    assert st == 0
    before = host(kc)
    got, st = call([50, 1, 2, -1, 4, 49], [-1, 3, 31, -1, 7, 0])
    assert st == -8
    assert_same(got, good, "positions outside are taken as 0")
    got, st = call([0, 1, 2, 0, 4, 49], [32, 3, -2, 1 << 30, 7, 0])
    assert st == -8
    assert_same(got, good)
    assert_same(host(kc), before, "slots outside store nothing")


def test_the_integers_follow_the_real_operator():
    """Against norm and rotation in double precision: half a step of the last rounding, 2^-7 steps and a bit of u's (twice,
    through the rotation, times sqrt 2), the table's 2^-15 of 127 steps, gamma's 2^-16 and rho's 2^-29 of them, and the
    root's own rounding (relative 2^-12 of 127 steps and less at the norms drawn here)."""
    rng = np.random.default_rng(0)
    T, heads, kv = 200, 2, 1
    f = binding.ibert_rope_frequencies(64)
    rope = binding.ibert_rope_rows(f, 512)
    pos = rng.integers(0, 512, T).astype(np.int32)
    gq, gk = _gammas(rng)
    for bits in (8, 16):
        x, S_in = _x(rng, T, heads + 2 * kv, bits)
        q, k, _ = _run(x, S_in, heads, kv, (gq, gk), rope, pos, False, True, False)
        r = x.reshape(T, heads + 2 * kv, 64).astype(np.float64)
        for got, part, gamma, S in ((q, r[:, :heads], gq, SC["S_q"]), (k, r[:, heads:heads + kv], gk, SC["S_k"])):
            y = part / np.sqrt((part ** 2).mean(-1, keepdims=True)) * gamma
            a = pos[:, None, None] * f
            c, s = np.cos(a), np.sin(a)
            y = np.concatenate([y[..., :32] * c - y[..., 32:] * s, y[..., :32] * s + y[..., 32:] * c], -1) / S
            inside = np.abs(y) < 127
            assert np.abs(got - y)[inside].max() < 0.5 + 2 ** -7 * 1.5 * 2 ** 0.5 + 180 * (2 ** -14 + 2 ** -12)

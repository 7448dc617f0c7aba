"""Plain 64-bit integer forms of the operators for generation (slots, heads with rotary positions, windowed and paged
attention), written from their definitions in ``include/ibert.h``; numpy on the host."""
import math

import numpy as np

import oracle

D = 64


# ----------------------------------------------------------------------------- slots
def kv_slots(lens, new, tables, stack, n_free, P, max_tokens):
    """(lens_out, n_free_out, cu_seqlens, slots, positions, tables, stack, whether something was out of range)"""
    tables, stack, bad = tables.copy(), stack.copy(), False
    B, max_pages = tables.shape
    most, cap = max_pages * P, stack.size
    top = min(max(int(n_free), 0), cap)
    bad |= top != n_free
    held = []
    for n in lens:
        held.append(min(max(int(n), 0), most))
        bad |= held[-1] != n
    pages = lambda n: -(-n // P)  # noqa: E731
    for b in range(B):
        if new[b] < 0:
            for j in range(pages(held[b])):
                if top < cap:
                    stack[top] = tables[b, j]
                    top += 1
                else:
                    bad = True
    slots, positions = np.full(max_tokens, -1, np.int64), np.zeros(max_tokens, np.int64)
    cu, out = [0], []
    for b in range(B):
        want = max(int(new[b]), 0)
        n = min(want, max_tokens - cu[-1])
        bad |= n < want
        stored, missing = 0, False
        for i in range(n):
            p, t = held[b] + i, cu[-1] + i
            if p >= most:
                bad = True
                continue
            if p % P == 0:
                missing = top == 0
                if not missing:
                    top -= 1
                tables[b, p // P] = -1 if missing else stack[top]
            positions[t] = p
            page = int(tables[b, p // P])
            if page >= 0 and page * P + p % P < 2 ** 31:
                slots[t] = page * P + p % P
            else:
                bad = True
            stored += not missing
        cu.append(cu[-1] + n)
        out.append(0 if new[b] < 0 else held[b] + stored)
    return (np.array(out, np.int64), top, np.array(cu, np.int64), slots, positions, tables, stack, bad)


# ----------------------------------------------------------------------------- norm, rotation, int8
def _requant(v, b, c, qmax):
    return np.clip((v * b + ((1 << c) >> 1)) >> c, -qmax, qmax)


def head_norm_multipliers(gamma, S):
    a = np.asarray(gamma, np.float64) * (128.0 / S)
    top = np.abs(a).max()
    g = 16
    while top * 2.0 ** g > 32767:
        g -= 1
    return (np.sign(a) * np.floor(np.abs(a) * 2.0 ** g + 0.5)).astype(np.int64), g


def head_values(x, bits, gamma, S_in, S):
    """u of heads x [..., 64]: whole numbers at scale S / 128."""
    x = x.astype(np.int64)
    if gamma is None:
        b, c = oracle.dyadic(128.0 * S_in / S)
        return _requant(x, b, c, 32767)
    b, g = head_norm_multipliers(gamma, S)
    s0 = 16 if bits == 8 else 10
    ss = (x * x).sum(-1)
    r = np.array([max(1, math.isqrt(int(v) << s0)) for v in ss.reshape(-1)], np.int64).reshape(ss.shape + (1,))
    l = np.array([int(v).bit_length() for v in r.reshape(-1)], np.int64).reshape(r.shape)  # noqa: E741
    rho, sh = (np.int64(1) << (l + 29)) // r, l + 26 - s0 // 2 + g
    return np.clip((x * b * rho + (np.int64(1) << (sh - 1))) >> sh, -32767, 32767)


def rotate(u, rows, interleaved):
    """int8 of u [T, h, 64] rotated by rows [T, rot] of the table (None: not at all)."""
    y = u << 14
    rot = 0 if rows is None else rows.shape[1]
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        c, s = rows[:, 2 * i, None].astype(np.int64), rows[:, 2 * i + 1, None].astype(np.int64)
        y[..., a], y[..., b] = u[..., a] * c - u[..., b] * s, u[..., a] * s + u[..., b] * c
    return np.clip((y + (1 << 20)) >> 21, -127, 127).astype(np.int8)


def qkv_rope(x, heads, kv_heads, S_in, S_q, S_k, S_v, gamma_q, gamma_k, rope, positions, interleaved):
    """q [T, heads, 64], k, v [T, kv_heads, 64] as int8."""
    bits = 8 * x.itemsize
    x = x.reshape(-1, heads + 2 * kv_heads, D)
    rows = None if rope is None else rope[positions]
    q = rotate(head_values(x[:, :heads], bits, gamma_q, S_in, S_q), rows, interleaved)
    k = rotate(head_values(x[:, heads:heads + kv_heads], bits, gamma_k, S_in, S_k), rows, interleaved)
    b, c = oracle.dyadic(S_in / S_v)
    return q, k, _requant(x[:, heads + kv_heads:].astype(np.int64), b, c, 127).astype(np.int8)


# ----------------------------------------------------------------------------- attention
def iexp(d, S):
    """i-exp (Algorithm 3) of distances d >= 0 at scale S, and its largest value."""
    s_in = 0
    while math.floor(1.353 / math.ldexp(S, s_in)) > 32767:
        s_in += 1
    Sp = math.ldexp(S, s_in)
    q_ln2, q_b, q_c = math.floor(0.6931471805599453 / Sp), math.floor(1.353 / Sp), math.floor(0.344 / ((0.3585 * Sp) * Sp))
    s_out = max(0, (q_b * q_b + q_c).bit_length() - 21)
    d = d >> s_in
    z = d // q_ln2
    return ((q_b - (d - z * q_ln2)) ** 2 + q_c) >> np.minimum(z + s_out, 31), (q_b * q_b + q_c) >> s_out


def weighted(s, v, S_q, S_k, S_v, S_ctx, p_max):
    """Result of one query: scores s [n] of its visible keys, values v [n, 64]."""
    if s.size == 0:
        return np.zeros(D, np.int64)
    e, top = iexp(s.max() - s, S_q * S_k / 8.0)
    w = (e * ((p_max << 24) // top) + (1 << 23)) >> 24
    O, W = (w.astype(np.float64) @ v.astype(np.float64)).astype(np.int64), int(w.sum())    # (exact: below 2^53)
    assert w.max() == p_max and np.abs(O).max() < 2 ** 31
    b, c = oracle.dyadic(S_v / S_ctx)
    n = W.bit_length()
    R, sh = (b << (n - 1)) // W, c + n - 1
    return np.clip((O * R + (1 << (sh - 1))) >> sh, -127, 127)


def visible(n, window, sinks):
    """Keys that the last of n tokens sees."""
    j = np.arange(n)
    return j if not window else j[(j >= n - window) | (j < sinks)]


def attention_decode(q, k_cache, v_cache, tables, lens, window, sinks, scales, p_max):
    """q [B, heads * 64]; pages outside the pool are left out."""
    n_pages, kv, P, _ = k_cache.shape
    B = tables.shape[0]
    q = q.reshape(B, kv, -1, D).astype(np.int64)
    out = np.zeros(q.shape, np.int64)
    for b in range(B):
        j = visible(int(lens[b]), window, sinks)
        page = tables[b, j // P]
        j, page = j[(page >= 0) & (page < n_pages)], page[(page >= 0) & (page < n_pages)]
        for h in range(kv):
            k, v = k_cache[page, h, j % P].astype(np.int64), v_cache[page, h, j % P].astype(np.int64)
            for i in range(q.shape[2]):
                out[b, h, i] = weighted(k @ q[b, h, i], v, *scales, p_max)
    return out.reshape(B, -1).astype(np.int8)


def attention_window(qkv, cu, heads, kv_heads, window, sinks, scales, p_max):
    """Causal attention of packed sequences; rows of other tokens are 0."""
    x = qkv.reshape(qkv.shape[0], heads + 2 * kv_heads, D).astype(np.int64)
    out = np.zeros((qkv.shape[0], heads, D), np.int64)
    for b in range(len(cu) - 1):
        for i in range(int(cu[b + 1] - cu[b])):
            j = cu[b] + visible(i + 1, window, sinks)
            for h in range(heads):
                kh = heads + h // (heads // kv_heads)
                out[cu[b] + i, h] = weighted(x[j, kh] @ x[cu[b] + i, h], x[j, kh + kv_heads], *scales, p_max)
    return out.reshape(qkv.shape[0], -1).astype(np.int8)

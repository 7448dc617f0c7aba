"""Integer-only generation over a paged int8 key-value cache, as measurable cases.

Four operators that a program which generates text calls in turn, every one on integer tensors with
their scales and with results that are whole numbers fixed by the definition (int8 activations are
returned as the whole numbers they hold, at the scale that the call was given):

  slots    block tables, slot maps, positions and row offsets of a step, from the requests' lengths
  rope     Q | K | V of new tokens: norm of every head, rotary positions, int8; K and V into the cache's pages
  window   causal attention of packed prompts, with a sliding window and first tokens that stay visible
  decode   attention of one new token per sequence over the paged cache

Heads are those of this repository's configurations (12 and 16 heads of 64) or a generic grouping of
them; inputs are seeded random integers of the spread that quantised activations have.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

D = 64                       # head size
S_IN = 4.5 / 127.0           # scale of a unit-variance int8 activation


def listed() -> list[dict]:
    return [
        # the bookkeeping of one generation step: most requests get one token, a few end, a few prompts start
        {"name": "slots_step_b256", "op": "slots", "B": 256, "P": 16, "most_new": 1, "max_len": 4096},
        # the bookkeeping of a large batch of prompts
        {"name": "slots_prompts_b512", "op": "slots", "B": 512, "P": 64, "most_new": 512, "max_len": 8192},
        # one generation step of 32 sequences: the linear layer's Q16 values, normed, rotated, cached; Q alone is kept
        {"name": "rope_step_t32", "op": "rope", "T": 32, "heads": 12, "kv_heads": 12, "bits": 16, "norm": True, "rot": 64,
         "interleaved": False, "P": 16, "cache": True, "with_kv": False},
        # an odd number of prompt tokens of grouped heads without norm, a quarter of the head rotated, no cache
        {"name": "rope_part_t4099", "op": "rope", "T": 4099, "heads": 16, "kv_heads": 4, "bits": 8, "norm": False, "rot": 16,
         "interleaved": True, "P": 16, "cache": False, "with_kv": True},
        # the prompts of a large batch: Q, K, V for the attention and K, V into the cache
        {"name": "rope_prompts_t32768", "op": "rope", "T": 32768, "heads": 16, "kv_heads": 16, "bits": 16, "norm": True, "rot": 64,
         "interleaved": False, "P": 64, "cache": True, "with_kv": True},
        # a few short prompts
        {"name": "window_short_b4", "op": "window", "B": 4, "longest": 97, "heads": 12, "kv_heads": 12, "window": 0, "sinks": 0, "p_max": 255},
        # prompts of very different lengths, plain causal attention with grouped heads
        {"name": "window_causal_b5", "op": "window", "B": 5, "longest": 1531, "heads": 16, "kv_heads": 4, "window": 0, "sinks": 0, "p_max": 255},
        # one long document with a sliding window and sinks
        {"name": "window_long_l8192", "op": "window", "B": 1, "longest": 8192, "heads": 16, "kv_heads": 16, "window": 2048, "sinks": 4, "p_max": 255},
        # one sequence at a time: interactive use, where latency counts
        {"name": "decode_b1_l1000", "op": "decode", "B": 1, "longest": 1000, "heads": 12, "kv_heads": 12, "P": 16, "window": 0, "sinks": 0, "p_max": 255},
        # a batch of sequences of different lengths
        {"name": "decode_b64_l2048", "op": "decode", "B": 64, "longest": 2048, "heads": 16, "kv_heads": 16, "P": 64, "window": 0, "sinks": 0, "p_max": 255},
        # few very long sequences of grouped heads
        {"name": "decode_b16_l32768", "op": "decode", "B": 16, "longest": 32768, "heads": 32, "kv_heads": 4, "P": 128, "window": 0, "sinks": 0, "p_max": 255},
        # a large batch with a sliding window: most of the cache stays unread
        {"name": "decode_window_b128", "op": "decode", "B": 128, "longest": 5000, "heads": 16, "kv_heads": 4, "P": 32, "window": 1024, "sinks": 4, "p_max": 127},
    ]


def _log_int(rng, lo: int, hi: int) -> int:
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng) -> dict:
    op = rng.choice(["slots", "rope", "rope", "window", "window", "decode", "decode", "decode"])
    P = rng.choice([16, 32, 64, 128])
    kv = rng.choice([1, 2, 4, 8, 12, 16])
    heads = kv * rng.choice([g for g in (1, 2, 3, 4, 8) if kv * g <= 32])
    if op == "slots":
        new = rng.choice([1, 1, _log_int(rng, 8, 512)])
        return {"op": op, "B": _log_int(rng, 1, 4096 if new == 1 else 512), "P": P, "most_new": new, "max_len": _log_int(rng, 512, 16384)}
    if op == "rope":
        cache = rng.random() < 0.7
        return {"op": op, "T": _log_int(rng, 1, 32768 * 32 // (heads + 2 * kv) // 2), "heads": heads, "kv_heads": kv, "bits": rng.choice([8, 16]),
                "norm": rng.random() < 0.6, "rot": rng.choice([0, 16, 32, 48, 64, 64]), "interleaved": rng.random() < 0.5, "P": P,
                "cache": cache, "with_kv": not cache or rng.random() < 0.5}
    window = rng.choice([0, 0, _log_int(rng, 16, 4096)])
    sinks = rng.choice([0, 1, 4, 37]) if window else 0
    p_max = rng.choice([255, 255, 127])
    if op == "window":
        longest = _log_int(rng, 1, 2900)
        return {"op": op, "B": _log_int(rng, 1, max(1, 8192 // longest)), "longest": longest, "heads": min(heads, 16) if min(heads, 16) % kv == 0 else kv,
                "kv_heads": kv, "window": window, "sinks": sinks, "p_max": p_max}
    longest = _log_int(rng, 1, 32768)
    return {"op": op, "B": _log_int(rng, 1, max(1, min(256, (1 << 21) // (longest * kv)))), "longest": longest, "heads": heads, "kv_heads": kv, "P": P,
            "window": window, "sinks": sinks, "p_max": p_max}


# --------------------------------------------------------------------------- inputs
def _int8(g, *shape, spread: float = 28.0) -> torch.Tensor:
    return (torch.randn(*shape, generator=g, device="cuda") * spread).round_().clamp_(-127, 127).to(torch.int8)


def _lengths(case: dict) -> np.ndarray:
    """Lengths of a case's batch, in no particular order: between an eighth of the longest and the longest, which occurs."""
    n = np.random.default_rng([case["B"], case["longest"]]).integers(max(1, case["longest"] // 8), case["longest"] + 1, case["B"])
    n[0] = case["longest"]
    return n


def _step(case: dict):
    """What the requests of a scheduler's step hold and get (-1: ended), in no particular order."""
    rng = np.random.default_rng([case["B"], case["max_len"], case["most_new"]])
    B, most = case["B"], case["most_new"]
    low = 0 if most > 1 else 1
    lens = rng.integers(low, max(low + 1, case["max_len"] - most), B)
    new = rng.integers(0, most + 1, B) if most > 1 else np.ones(B, dtype=np.int64)
    new[rng.random(B) < 0.05] = -1                                         # requests that ended
    if most == 1:
        some = rng.random(B) < 0.02                                        # requests that start
        lens[some], new[some] = 0, rng.integers(1, 65, B)[some]
    new[0] = max(new[0], 1)
    return lens, new


def _pages(rng, lens: np.ndarray, P: int, columns: int):
    """Block table of sequences whose pages lie scattered over a pool, and the size of the pool."""
    need = -(-lens // P)
    total = int(need.sum()) + 3
    order = rng.permutation(total).astype(np.int32)
    table = np.full((lens.size, columns), -1, dtype=np.int32)
    first = np.concatenate([[0], np.cumsum(need)])
    for b in range(lens.size):
        table[b, :need[b]] = order[first[b]:first[b + 1]]
    return table, total


def _rope_rows(rot: int, n: int) -> np.ndarray:
    """cos and sin of every position in units of 2^-14, pair by pair."""
    inv = 10000.0 ** (-np.arange(0, rot, 2, dtype=np.float64) / rot)
    a = np.arange(n, dtype=np.float64)[:, None] * inv[None, :]
    return np.floor(np.stack([np.cos(a), np.sin(a)], axis=-1) * 16384.0 + 0.5).astype(np.int16).reshape(n, rot)


def prepare(case: dict, seed: int) -> dict:
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    rng = np.random.default_rng(int(seed))
    st = dict(case)
    put = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    if case["op"] == "slots":
        B, P = case["B"], case["P"]
        order = rng.permutation(B)
        lens, new = (a[order] for a in _step(case))
        columns = -(-case["max_len"] // P)
        table, total = _pages(rng, lens, P, columns)
        free = rng.permutation(int(np.maximum(new, 0).sum()) // P + B + 8).astype(np.int32) + total
        st.update(lens=put(lens.astype(np.int32)), new=put(new.astype(np.int32)), table=put(table),
                  free=put(np.concatenate([free, np.full(total, -1, dtype=np.int32)])),
                  n_free=put(np.array([free.size], dtype=np.int32)), max_tokens=int(np.maximum(new, 0).sum()) + 5)
        T = st["max_tokens"]
        st.update(outs=dict(lens_out=torch.empty_like(st["lens"]), n_free_out=torch.empty_like(st["n_free"]),
                            cu_seqlens=torch.empty(B + 1, dtype=torch.int32, device="cuda"), slots=torch.empty(T, dtype=torch.int32, device="cuda"),
                            positions=torch.empty(T, dtype=torch.int32, device="cuda")))
    elif case["op"] == "rope":
        T, hq, hk, P = case["T"], case["heads"], case["kv_heads"], case["P"]
        n = hq + 2 * hk
        x = torch.randn(T, n * D, generator=g, device="cuda")
        x *= torch.exp(torch.randn(1, n, 1, generator=g, device="cuda") * 0.5).expand(1, n, D).reshape(1, n * D)
        top, spread = (127, 28.0) if case["bits"] == 8 else (32767, 6000.0)
        st["x"] = (x * spread).round_().clamp_(-top, top).to(torch.int8 if case["bits"] == 8 else torch.int16)
        st["S_x"] = 1.0 / spread
        st["gamma_q"], st["gamma_k"] = (1.0 + 0.2 * rng.standard_normal(D), 1.0 + 0.2 * rng.standard_normal(D)) if case["norm"] else (None, None)
        st["table"] = put(_rope_rows(case["rot"], 8192)) if case["rot"] else None
        st["positions"] = put(rng.integers(0, 8192, T).astype(np.int32))
        pages = -(-T // P) + 2
        if case["cache"]:
            slots = rng.permutation(pages * P)[:T].astype(np.int32) if T < 1024 else (
                rng.permutation(pages)[:, None] * P + np.arange(P)[None, :]).reshape(-1)[:T].astype(np.int32)
            st.update(slots=put(slots), k_cache=_int8(g, pages, hk, P, D), v_cache=_int8(g, pages, hk, P, D))
        else:
            st.update(slots=None, k_cache=None, v_cache=None)
        st["out"] = torch.empty(T, (n if case["with_kv"] else hq) * D, dtype=torch.int8, device="cuda")
    elif case["op"] == "window":
        lens = rng.permutation(_lengths(case))
        st["cu"] = put(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32))
        st["T"] = int(lens.sum())
        st["qkv"] = _int8(g, st["T"], (case["heads"] + 2 * case["kv_heads"]) * D)
        st["out"] = torch.empty(st["T"], case["heads"] * D, dtype=torch.int8, device="cuda")
    else:
        lens = rng.permutation(_lengths(case))
        columns = -(-case["longest"] // case["P"])
        table, total = _pages(rng, lens, case["P"], columns)
        st["lens"], st["table"] = put(lens.astype(np.int32)), put(table)
        st["q"] = _int8(g, case["B"], case["heads"] * D)
        st["k_cache"] = _int8(g, total, case["kv_heads"], case["P"], D)
        st["v_cache"] = _int8(g, total, case["kv_heads"], case["P"], D)
        st["out"] = torch.empty(case["B"], case["heads"] * D, dtype=torch.int8, device="cuda")
    if "T" in st or case["op"] in ("rope", "decode"):
        st.update(S_q=1.5 * S_IN, S_k=S_IN, S_v=S_IN, S_ctx=S_IN / 2.0)
    return st


_ctx = None


def _context():
    """The framework's handle that a program keeps."""
    global _ctx
    if _ctx is None:
        from paper_2101_01321_b200 import binding
        _ctx = binding.Context(torch.cuda.current_device())
    return _ctx


# --------------------------------------------------------------------------- the passes
def run(st: dict):
    return _own(st) if own else _PLAIN[st["op"]](st)


def _own(st: dict):
    ctx = _context()
    if st["op"] == "slots":
        o = st["outs"]
        ctx.ibert_kv_slots(st["lens"], st["new"], st["table"], st["free"], st["n_free"], st["P"], **o)
        return [o["lens_out"], o["n_free_out"], o["cu_seqlens"], o["slots"], o["positions"], st["table"], st["free"]]
    if st["op"] == "rope":
        ctx.ibert_qkv_rope_i8(st["x"], st["S_x"], st["heads"], st["kv_heads"], st["S_q"], st["S_k"], st["S_v"], gamma_q=st["gamma_q"],
                              gamma_k=st["gamma_k"], rope=st["table"], positions=st["positions"], interleaved=st["interleaved"],
                              slots=st["slots"], k_cache=st["k_cache"], v_cache=st["v_cache"], with_kv=st["with_kv"], out=st["out"])
        return [st["out"]] + ([st["k_cache"], st["v_cache"]] if st["cache"] else [])
    scales = (st["S_q"], st["S_k"], st["S_v"], st["S_ctx"])
    if st["op"] == "window":
        ctx.ibert_attention_window_i8(st["qkv"], st["cu"], st["longest"], st["heads"], st["kv_heads"], *scales, window=st["window"],
                                      sinks=st["sinks"], p_max=st["p_max"], out=st["out"])
    else:
        ctx.ibert_attention_decode_i8(st["q"], st["k_cache"], st["v_cache"], st["table"], st["lens"], st["longest"], st["heads"], *scales,
                                      window=st["window"], sinks=st["sinks"], p_max=st["p_max"], out=st["out"])
    return st["out"]


# --------------------------------------------------------------------------- plain forms: elementary torch operations
def _dyadic(m: float) -> tuple[int, int]:
    c = min(31, 31 - math.frexp(m)[1])
    b = math.floor(math.ldexp(m, c) + 0.5)
    return (1 << 30, c - 1) if b == 1 << 31 else (b, c)


def _exp_constants(S: float, p_max: int):
    """Constants of i-exp for scores at scale S: pre-shift, q_ln2, q_b, q_c, post-shift, weight multiplier."""
    s_in = 0
    while math.floor(1.353 / math.ldexp(S, s_in)) > 32767:
        s_in += 1
    Sp = math.ldexp(S, s_in)
    q_b, q_c = math.floor(1.353 / Sp), math.floor(0.344 / ((0.3585 * Sp) * Sp))
    top = q_b * q_b + q_c
    s_out = max(0, top.bit_length() - 21)
    return s_in, math.floor(0.6931471805599453 / Sp), q_b, q_c, s_out, (p_max << 24) // (top >> s_out)


def _plain_attend(s: torch.Tensor, seen: torch.Tensor, v: torch.Tensor, st: dict) -> torch.Tensor:
    """Weights of whole-number scores s [..., L] where `seen`, and the weighted mean of v [..., L, 64], as int8.

    (Scores and weights are whole numbers below 2^24 and 2^8, so the products in floating point are exact.)"""
    s_in, q_ln2, q_b, q_c, s_out, b_w = _exp_constants(st["S_q"] * st["S_k"] / 8.0, st["p_max"])
    s = s.to(torch.int32)
    top = torch.where(seen, s, torch.full_like(s, -(1 << 30))).amax(-1, keepdim=True)
    d = torch.where(seen, top - s, torch.zeros_like(s)) >> s_in
    z = d // q_ln2
    t = q_b - (d - z * q_ln2)
    e = (t * t + q_c) >> (z + s_out).clamp_(max=31)
    w = torch.where(seen, (e.long() * b_w + (1 << 23)) >> 24, 0).double()
    total, mass = torch.matmul(w, v).long(), w.sum(-1, keepdim=True)
    bits = torch.frexp(mass).exponent.long().clamp(min=1)
    mass = mass.long()
    b, c = _dyadic(st["S_v"] / st["S_ctx"])
    share = (b << (bits - 1)) // mass.clamp(min=1)
    out = (total * share + (1 << (c + bits - 2).clamp(min=0))) >> (c + bits - 1)
    return torch.where(mass > 0, out, 0).clamp_(-127, 127).to(torch.int8)


def _plain_window(st: dict):
    T, hq, hk = st["T"], st["heads"], st["kv_heads"]
    x = st["qkv"].float().view(T, hq + 2 * hk, D).transpose(0, 1)
    q, k, v = x[:hq].reshape(hk, hq // hk, T, D), x[hq:hq + hk], x[hq + hk:].double()
    at = torch.arange(T, device="cuda")
    seq = torch.searchsorted(st["cu"][1:].long(), at, right=True)
    first = st["cu"].long()[seq]
    seen = (seq[:, None] == seq[None, :]) & (at[:, None] >= at[None, :])
    if st["window"]:
        seen &= (at[:, None] - at[None, :] < st["window"]) | ((at - first)[None, :] < st["sinks"])
    out = _plain_attend(torch.matmul(q, k[:, None].transpose(-1, -2)), seen, v[:, None], st)
    return out.reshape(hq, T, D).transpose(0, 1).reshape(T, hq * D)


def _plain_decode(st: dict):
    B, hq, P = st["B"], st["heads"], st["P"]
    hk = st["kv_heads"]
    table = st["table"].long().clamp(min=0)
    k = st["k_cache"][table].permute(0, 2, 1, 3, 4).reshape(B, hk, -1, D)
    v = st["v_cache"][table].permute(0, 2, 1, 3, 4).reshape(B, hk, -1, D)
    j = torch.arange(k.shape[2], device="cuda")[None, :]
    n = st["lens"].long()[:, None]
    seen = j < n
    if st["window"]:
        seen &= (j >= n - st["window"]) | (j < st["sinks"])
    q = st["q"].float().view(B, hk, hq // hk, D)
    return _plain_attend(torch.matmul(q, k.float().transpose(-1, -2)), seen[:, None, None, :], v.double(), st).reshape(B, hq * D)


def _gamma_constants(gamma, S_out: float):
    a = np.asarray(gamma, dtype=np.float64) * (128.0 / S_out)
    m = float(np.abs(a).max())
    g = 16 if m == 0 else min(16, math.floor(math.log2(32767.0 / m)))
    while np.floor(np.abs(a) * 2.0 ** g + 0.5).max() > 32767:
        g -= 1
    return np.sign(a) * np.floor(np.abs(a) * 2.0 ** g + 0.5), g


def _plain_head(x: torch.Tensor, gamma, S_x: float, S_out: float, bits: int) -> torch.Tensor:
    """Heads [T, h, 64] normed (gamma) or rescaled to whole numbers at scale S_out / 128."""
    x = x.long()
    if gamma is None:
        b, c = _dyadic(128.0 * S_x / S_out)
        return ((x * b + ((1 << c) >> 1)) >> c).clamp_(-32767, 32767)
    b, g = _gamma_constants(gamma, S_out)
    s0 = 16 if bits == 8 else 10
    root = torch.sqrt(((x * x).sum(-1, keepdim=True) << s0).double()).floor().long().clamp(min=1)
    n = torch.frexp(root.double()).exponent.long()
    rho, sh = (torch.ones_like(root) << (n + 29)) // root, n + 26 - s0 // 2 + g
    t = x * torch.from_numpy(b.astype(np.int64)).cuda()
    return ((t * rho + (1 << (sh - 1))) >> sh).clamp_(-32767, 32767)


def _plain_rotate(u: torch.Tensor, table, positions: torch.Tensor, interleaved: bool) -> torch.Tensor:
    y = u << 14
    if table is not None:
        rot = table.shape[1]
        cs = table[positions.long()].long().view(-1, 1, rot // 2, 2)
        c, s = cs[..., 0], cs[..., 1]
        a, b = (u[..., 0:rot:2], u[..., 1:rot:2]) if interleaved else (u[..., :rot // 2], u[..., rot // 2:rot])
        a, b = a * c - b * s, a * s + b * c
        y = torch.cat([torch.stack([a, b], -1).flatten(-2) if interleaved else torch.cat([a, b], -1), y[..., rot:]], -1)
    return ((y + (1 << 20)) >> 21).clamp_(-127, 127).to(torch.int8)


def _plain_rope(st: dict):
    T, hq, hk = st["T"], st["heads"], st["kv_heads"]
    x = st["x"].view(T, hq + 2 * hk, D)
    q = _plain_rotate(_plain_head(x[:, :hq], st["gamma_q"], st["S_x"], st["S_q"], st["bits"]), st["table"], st["positions"], st["interleaved"])
    k = _plain_rotate(_plain_head(x[:, hq:hq + hk], st["gamma_k"], st["S_x"], st["S_k"], st["bits"]), st["table"], st["positions"], st["interleaved"])
    b, c = _dyadic(st["S_x"] / st["S_v"])
    v = ((x[:, hq + hk:].long() * b + ((1 << c) >> 1)) >> c).clamp_(-127, 127).to(torch.int8)
    out = (torch.cat([q, k, v], 1) if st["with_kv"] else q).reshape(T, -1)
    if not st["cache"]:
        return [out]
    page, row = st["slots"].long() // st["P"], st["slots"].long() % st["P"]
    st["k_cache"][page, :, row] = k
    st["v_cache"][page, :, row] = v
    return [out, st["k_cache"], st["v_cache"]]


def _plain_slots(st: dict):
    P, T, table, free = st["P"], st["max_tokens"], st["table"], st["free"]
    lens, new = st["lens"].long(), st["new"].long()
    B = lens.numel()
    ended = new < 0
    had = (lens + P - 1) // P
    given = torch.where(ended, had, 0)                                      # pages that ended requests give back
    n0 = st["n_free"].long()
    column = torch.arange(table.shape[1], device="cuda")[None, :]
    back = column < given[:, None]
    to = torch.where(back, (n0 + given.cumsum(0) - given)[:, None] + column, free.numel())
    free.copy_(torch.cat([free, free[:1]]).scatter_(0, to.flatten(), table.flatten())[:-1])
    n1 = n0 + given.sum()
    new = new.clamp(min=0)
    after = torch.where(ended, 0, lens + new)
    need = torch.where(ended, 0, (after + P - 1) // P - had)
    fresh = (column >= had[:, None]) & (column < (had + need)[:, None])
    k = (need.cumsum(0) - need)[:, None] + column - had[:, None]            # position in the order of taking
    table.copy_(torch.where(fresh, free[(n1 - 1 - k).clamp(min=0, max=free.numel() - 1)], table))
    cu = torch.cat([new.new_zeros(1), new.cumsum(0)])
    t = torch.arange(T, device="cuda")
    b = torch.searchsorted(cu[1:], t, right=True).clamp(max=B - 1)
    real = t < cu[-1]
    pos = torch.where(real, lens[b] + t - cu[b], 0)
    slots = torch.where(real, table[b, (pos // P).clamp(max=table.shape[1] - 1)].long() * P + pos % P, -1)
    i32 = torch.int32
    return [after.to(i32), (n1 - need.sum()).to(i32), cu.to(i32), slots.to(i32), pos.to(i32), table, free]


_PLAIN = {"slots": _plain_slots, "rope": _plain_rope, "window": _plain_window, "decode": _plain_decode}


# --------------------------------------------------------------------------- cost
def work(case: dict) -> dict:
    if case["op"] == "slots":
        lens, new = _step(case)
        P, tokens, ended = case["P"], int(np.maximum(new, 0).sum()), new < 0
        taken = (-(-(lens + new) // P) - -(-lens // P))[~ended].sum()
        given = (-(-lens // P))[ended].sum()
        return {"bytes": 16.0 * case["B"] + 8.0 * tokens + 8.0 * float(taken + given), "flops": 0}
    if case["op"] == "rope":
        n, T = case["heads"] + 2 * case["kv_heads"], case["T"]
        kept = (n if case["with_kv"] else case["heads"]) + (2 * case["kv_heads"] if case["cache"] else 0)
        return {"bytes": T * D * (n * case["bits"] / 8.0 + kept) + T * (8.0 + 2.0 * case["rot"]), "flops": 10.0 * T * n * D}
    lens = _lengths(case).astype(np.float64)
    if case["op"] == "window":
        w = case["window"] + case["sinks"] if case["window"] else case["longest"]
        pairs = float(np.where(lens <= w, lens * (lens + 1) / 2, w * (w + 1) / 2 + (lens - w) * w).sum())
        return {"bytes": float(lens.sum()) * D * (2 * case["heads"] + 2 * case["kv_heads"]), "flops": 4.0 * D * pairs * case["heads"]}
    keys = float((np.minimum(lens, case["window"] + case["sinks"]) if case["window"] else lens).sum())
    return {"bytes": 2.0 * D * keys * case["kv_heads"] + 2.0 * D * case["B"] * case["heads"], "flops": 4.0 * D * keys * case["heads"]}


# --------------------------------------------------------------------------- the definition in 64 bits, on the host
def _exact_iexp(d: np.ndarray, S: float, p_max: int) -> np.ndarray:
    """Weights of distances d >= 0 from the row's maximum (float64 holding whole numbers)."""
    shift = 0
    while math.floor(1.353 / (S * 2.0 ** shift)) > 32767:
        shift += 1
    Sp = S * 2.0 ** shift
    ln2, qb, qc = (math.floor(0.6931471805599453 / Sp), math.floor(1.353 / Sp), math.floor(0.344 / ((0.3585 * Sp) * Sp)))
    post = 0
    while (qb * qb + qc) >> post >= 1 << 21:
        post += 1
    d = np.floor(d / 2.0 ** shift)
    z = np.floor(d / ln2)
    poly = (qb - (d - z * ln2)) ** 2 + qc
    e = np.floor(poly / 2.0 ** np.minimum(z + post, 31))
    unit = (p_max << 24) // ((qb * qb + qc) >> post)
    return np.floor((e * unit + 2.0 ** 23) / 2.0 ** 24)


def _exact_rows(q: np.ndarray, k: np.ndarray, v: np.ndarray, seen, S: dict, p_max: int) -> np.ndarray:
    """Rows q [n, 64] against keys [L, 64]: float64 products of whole numbers are exact below 2^53."""
    s = q @ k.T
    s = np.where(seen, s, -np.inf)
    top = s.max(axis=1, keepdims=True)
    ok = np.isfinite(top)
    w = np.where(seen & ok, _exact_iexp(np.where(np.isfinite(s), np.where(ok, top, 0) - s, 0.0), S["S_q"] * S["S_k"] / 8.0, p_max), 0.0)
    O, W = (w @ v).astype(np.int64), np.maximum(w.sum(axis=1, keepdims=True), 1.0).astype(np.int64)
    b, c = _dyadic(S["S_v"] / S["S_ctx"])
    bits = np.floor(np.log2(W + 0.5)).astype(np.int64) + 1
    r = (b * (np.int64(1) << (bits - 1))) // W
    return np.where(ok, np.clip((O * r + (np.int64(1) << np.maximum(c + bits - 2, 0))) >> (c + bits - 1), -127, 127), 0)


def exact(case: dict, seed: int):
    st = prepare(case, seed)
    host = lambda t: t.cpu().numpy()  # noqa: E731
    if case["op"] == "slots":
        P, table, free = case["P"], host(st["table"]).copy(), host(st["free"]).copy()
        lens, new, top = host(st["lens"]).tolist(), host(st["new"]).tolist(), int(st["n_free"].item())
        slots, positions = np.full(st["max_tokens"], -1, dtype=np.int64), np.zeros(st["max_tokens"], dtype=np.int64)
        for b in range(len(lens)):
            if new[b] < 0:
                for j in range(-(-lens[b] // P)):
                    free[top], top = table[b, j], top + 1
        cu, after = [0], []
        for b in range(len(lens)):
            for p in range(lens[b], lens[b] + max(new[b], 0)):
                if p % P == 0:
                    top -= 1
                    table[b, p // P] = free[top]
                slots[cu[-1] + p - lens[b]], positions[cu[-1] + p - lens[b]] = table[b, p // P] * P + p % P, p
            cu.append(cu[-1] + max(new[b], 0))
            after.append(0 if new[b] < 0 else lens[b] + new[b])
        i64 = np.int64
        return [np.array(after, i64), np.array([top], i64), np.array(cu, i64), slots, positions, table.astype(i64), free.astype(i64)]
    if case["op"] == "rope":
        T, hq, hk, bits = case["T"], case["heads"], case["kv_heads"], case["bits"]
        if T * (hq + 2 * hk) > 400000:
            return None
        x = host(st["x"]).astype(np.int64).reshape(T, hq + 2 * hk, D)

        def head(v, gamma, S_out):
            if gamma is None:
                b, c = _dyadic(128.0 * st["S_x"] / S_out)
                return np.clip((v * b + ((1 << c) >> 1)) >> c, -32767, 32767)
            b, g = _gamma_constants(gamma, S_out)
            s0 = 16 if bits == 8 else 10
            root = np.array([max(1, math.isqrt(int(n) << s0)) for n in (v * v).sum(-1).reshape(-1)], dtype=np.int64).reshape(v.shape[:2] + (1,))
            n = np.array([int(r).bit_length() for r in root.reshape(-1)], dtype=np.int64).reshape(root.shape)
            sh = n + 26 - s0 // 2 + g
            return np.clip((v * b.astype(np.int64) * ((np.int64(1) << (n + 29)) // root) + (np.int64(1) << (sh - 1))) >> sh, -32767, 32767)

        def rotate(u):
            y = u << 14
            if st["table"] is not None:
                cs = host(st["table"]).astype(np.int64)[host(st["positions"])]
                for i in range(case["rot"] // 2):
                    a, b = (2 * i, 2 * i + 1) if case["interleaved"] else (i, i + case["rot"] // 2)
                    c, s = cs[:, 2 * i, None], cs[:, 2 * i + 1, None]
                    y[..., a], y[..., b] = u[..., a] * c - u[..., b] * s, u[..., a] * s + u[..., b] * c
            return np.clip((y + (1 << 20)) >> 21, -127, 127)

        b, c = _dyadic(st["S_x"] / st["S_v"])
        q, k = rotate(head(x[:, :hq], st["gamma_q"], st["S_q"])), rotate(head(x[:, hq:hq + hk], st["gamma_k"], st["S_k"]))
        v = np.clip((x[:, hq + hk:] * b + ((1 << c) >> 1)) >> c, -127, 127)
        out = [(np.concatenate([q, k, v], 1) if case["with_kv"] else q).reshape(T, -1)]
        if case["cache"]:
            kc, vc, at = host(st["k_cache"]).astype(np.int64), host(st["v_cache"]).astype(np.int64), host(st["slots"])
            for t in range(T):
                kc[at[t] // case["P"], :, at[t] % case["P"]], vc[at[t] // case["P"], :, at[t] % case["P"]] = k[t], v[t]
            out += [kc, vc]
        return out
    heads, kv, p_max = case["heads"], case["kv_heads"], case["p_max"]
    if work(case)["flops"] > 7e10:
        return None
    out = []
    if case["op"] == "window":
        x, cu = host(st["qkv"]).astype(np.float64), host(st["cu"])
        res = np.zeros((st["T"], heads * D), dtype=np.int64)
        for b in range(case["B"]):
            for h in range(heads):
                kh = heads + h // (heads // kv)
                for i0 in range(0, cu[b + 1] - cu[b], 512):
                    i = np.arange(i0, min(i0 + 512, cu[b + 1] - cu[b]))
                    j = np.arange(0, i[-1] + 1)
                    seen = j[None, :] <= i[:, None]
                    if case["window"]:
                        j = j[(j < case["sinks"]) | (j > i0 - case["window"])]
                        seen = (j[None, :] <= i[:, None]) & ((j[None, :] > i[:, None] - case["window"]) | (j[None, :] < case["sinks"]))
                    rows = x[cu[b]:cu[b + 1]]
                    res[cu[b] + i, h * D:(h + 1) * D] = _exact_rows(rows[i, h * D:(h + 1) * D], rows[j, kh * D:(kh + 1) * D],
                                                                     rows[j, (kh + kv) * D:(kh + kv + 1) * D], seen, st, p_max)
        return res
    table, lens, kc, vc, q = host(st["table"]), host(st["lens"]), host(st["k_cache"]), host(st["v_cache"]), host(st["q"]).astype(np.float64)
    for b in range(case["B"]):
        j = np.arange(lens[b])
        if case["window"]:
            j = j[(j >= lens[b] - case["window"]) | (j < case["sinks"])]
        pg, at = table[b, j // case["P"]], j % case["P"]
        row = [_exact_rows(q[b].reshape(kv, -1, D)[h], kc[pg, h, at].astype(np.float64), vc[pg, h, at].astype(np.float64), np.ones((1, j.size), bool), st, p_max)
               for h in range(kv)]
        out.append(np.concatenate(row).reshape(-1))
    return np.stack(out)

"""The operators for generation as they are used together: prompts in, then token after token over the paged cache; on
streams, in a captured graph, and against real arithmetic."""
import numpy as np
import pytest
import torch

import generation_reference as ref
from gpu_util import assert_same, ctx, dev, host
from paper_2101_01321_b200 import binding

pytestmark = pytest.mark.gpu

HEADS, KV, HIDDEN, P = 6, 2, 256, 16
COLS = (HEADS + 2 * KV) * 64
SC = dict(S_q=0.04, S_k=0.04, S_v=0.04)
S_CTX, S_X, S_QKV = 0.01, 0.03, 2e-4


class _Layer:
    """Q | K | V projection, heads, cache and attention of one layer; everything it keeps between steps lies on the GPU."""

    def __init__(self, c, B, max_len, window, sinks, seed=0):
        rng = np.random.default_rng(seed)
        self.c, self.B, self.max_len, self.window, self.sinks = c, B, max_len, window, sinks
        self.w = dev(rng.integers(-127, 128, (COLS, HIDDEN)).astype(np.int8))
        self.S_w = np.full(COLS, 0.02 / 127)
        self.gammas = 1 + 0.1 * rng.standard_normal(64), 1 + 0.1 * rng.standard_normal(64)
        self.rope = dev(binding.ibert_rope_rows(binding.ibert_rope_frequencies(64), max_len))
        columns = -(-max_len // P)
        pool = B * columns
        self.tables = torch.full((B, columns), -1, dtype=torch.int32, device="cuda")
        self.stack = dev(rng.permutation(pool).astype(np.int32))
        self.n_free = torch.tensor([pool], dtype=torch.int32, device="cuda")
        self.lens = torch.zeros(B, dtype=torch.int32, device="cuda")
        self.k = torch.zeros(pool, KV, P, 64, dtype=torch.int8, device="cuda")
        self.v = torch.zeros_like(self.k)

    def heads(self, x, new, rows, with_kv):
        _, _, cu, slots, pos = self.c.ibert_kv_slots(self.lens, new, self.tables, self.stack, self.n_free, P, rows, lens_out=self.lens,
                                                     n_free_out=self.n_free)
        qkv, _ = self.c.ibert_linear_i8(x, S_X, self.w, self.S_w, None, 3, S_QKV)
        out, _ = self.c.ibert_qkv_rope_i8(qkv, S_QKV, HEADS, KV, *SC.values(), *self.gammas, rope=self.rope, positions=pos, slots=slots,
                                          k_cache=self.k, v_cache=self.v, with_kv=with_kv)
        return out, cu

    def prompts(self, x, new):
        qkv, cu = self.heads(x, new, x.shape[0], True)
        return self.c.ibert_attention_window_i8(qkv, cu, self.max_len, HEADS, KV, *SC.values(), S_CTX, self.window, self.sinks)[0]

    def step(self, x, new):
        q, _ = self.heads(x, new, x.shape[0], False)
        return self.c.ibert_attention_decode_i8(q, self.k, self.v, self.tables, self.lens, self.max_len, HEADS, *SC.values(), S_CTX,
                                                self.window, self.sinks)[0]


def _inputs(rng, rows):
    return np.clip(np.rint(rng.standard_normal((rows, HIDDEN)) * 35), -127, 127).astype(np.int8)


@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 4)])
def test_tokens_one_by_one_equal_the_whole_prompt(window, sinks):
    """Prompts, then single tokens: every step's context is the row that the whole sequence as one prompt gives."""
    rng = np.random.default_rng(1)
    prompt, steps = np.array([33, 1, 100, 16]), 20
    full = [_inputs(rng, n + steps) for n in prompt]
    a = _Layer(ctx(), 4, 160, window, sinks)
    whole = host(a.prompts(dev(np.concatenate(full)), dev((prompt + steps).astype(np.int32))))
    ctx().check()
    at = np.concatenate([[0], np.cumsum(prompt + steps)])
    b = _Layer(ctx(), 4, 160, window, sinks)
    got = host(b.prompts(dev(np.concatenate([f[:n] for f, n in zip(full, prompt)])), dev(prompt.astype(np.int32))))
    cu = np.concatenate([[0], np.cumsum(prompt)])
    for i, n in enumerate(prompt):
        assert_same(got[cu[i]:cu[i + 1]], whole[at[i]:at[i] + n], f"prompt {i}")
    one = torch.ones(4, dtype=torch.int32, device="cuda")
    for s in range(steps):
        got = host(b.step(dev(np.stack([f[n + s] for f, n in zip(full, prompt)])), one))
        assert_same(got, np.stack([whole[at[i] + n + s] for i, n in enumerate(prompt)]), f"step {s}")
    ctx().check()
    assert host(b.lens).tolist() == (prompt + steps).tolist()


def test_requests_end_and_others_take_their_pages():
    """A request that ends gives its pages to the next one, whose contexts are those of a fresh cache."""
    rng = np.random.default_rng(2)
    a = _Layer(ctx(), 2, 96, 0, 0)
    a.prompts(dev(_inputs(rng, 90 + 60)), dev(np.array([90, 60], np.int32)))
    a.heads(dev(_inputs(rng, 1)), dev(np.array([-1, 0], np.int32)), 1, False)
    assert host(a.lens).tolist() == [0, 60]
    x = _inputs(rng, 70)
    got = host(a.prompts(dev(x), dev(np.array([70, 0], np.int32))))
    b = _Layer(ctx(), 2, 96, 0, 0)
    assert_same(got, host(b.prompts(dev(x), dev(np.array([70, 0], np.int32)))))
    y = _inputs(rng, 2)
    one = torch.ones(2, dtype=torch.int32, device="cuda")
    assert_same(host(a.step(dev(y), one))[0], host(b.step(dev(y), one))[0])
    ctx().check()


def test_a_captured_step_replays():
    """One generation step in a CUDA graph: lengths, tables and stack live on the GPU, so replaying it goes on."""
    rng = np.random.default_rng(3)
    s = torch.cuda.Stream()
    c = binding.Context(0, stream=s)
    with torch.cuda.stream(s):
        a, b = (_Layer(c, 3, 200, 50, 2) for _ in range(2))
        first = dev(_inputs(rng, 3 * 30))
        new, one = dev(np.full(3, 30, np.int32)), torch.ones(3, dtype=torch.int32, device="cuda")
        a.prompts(first, new)
        b.prompts(first, new)
        xs = [dev(_inputs(rng, 3)) for _ in range(25)]
        hold = xs[0].clone()
        b.step(hold, torch.zeros_like(one))                       # constants are uploaded before the capture
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        out = b.step(hold, one)
    for x in xs:
        with torch.cuda.stream(s):
            want = a.step(x, one)
            hold.copy_(x)
            g.replay()
        torch.cuda.synchronize()
        assert_same(host(out), host(want))
    c.check()
    assert torch.equal(a.lens, b.lens) and torch.equal(a.tables, b.tables) and torch.equal(a.k, b.k)


def test_two_streams_at_once():
    rng = np.random.default_rng(4)
    streams = [torch.cuda.Stream() for _ in range(2)]
    cs = [binding.Context(0, stream=s) for s in streams]
    xs = [[dev(_inputs(rng, 4)) for _ in range(30)] for _ in range(2)]
    first = [dev(_inputs(rng, 4 * 60)) for _ in range(2)]
    new, one = dev(np.full(4, 60, np.int32)), torch.ones(4, dtype=torch.int32, device="cuda")
    alone = []
    for i in range(2):
        layer = _Layer(ctx(), 4, 128, 0, 0, seed=i)
        layer.prompts(first[i], new)
        alone.append([host(layer.step(x, one)) for x in xs[i]])
    torch.cuda.synchronize()
    layers, got = [], [[], []]
    for i in range(2):
        with torch.cuda.stream(streams[i]):
            layers.append(_Layer(cs[i], 4, 128, 0, 0, seed=i))
            layers[i].prompts(first[i], new)
    for t in range(30):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(layers[i].step(xs[i][t], one))
    torch.cuda.synchronize()
    for i in range(2):
        cs[i].check()
        for t in range(30):
            assert_same(host(got[i][t]), alone[i][t])


def test_contexts_follow_real_attention():
    """Against softmax attention in double precision.  A weight is off by half a step of rounding (1/510) and by what i-exp is
    off: 0.0019 of the polynomial (the paper's bound) and its whole-number constants, below 0.001 at this scale -- together
    d < 0.005 for each of n keys.  With E the sum of the real weights the weighted mean moves by at most
    2 n d / E of the values' largest magnitude, and the result's own rounding adds half a step (and a bit)."""
    rng = np.random.default_rng(5)
    n, scales = 200, (0.05, 0.04, 0.03, 0.02)
    qkv = np.clip(np.rint(rng.standard_normal((n, 3 * 64)) * 28), -127, 127).astype(np.int8)
    out, _ = ctx().ibert_attention_window_i8(dev(qkv), dev(np.array([0, n], np.int32)), n, 1, 1, *scales)
    ctx().check()
    q, k, v = (qkv[:, 64 * i:64 * i + 64].astype(np.float64) * s for i, s in enumerate(scales[:3]))
    s = np.where(np.tri(n, dtype=bool), q @ k.T / 8, -np.inf)
    e = np.exp(s - s.max(1, keepdims=True))
    E = e.sum(1)
    got = host(out).astype(np.float64) * scales[3]
    limit = 2 * np.arange(1, n + 1) * 0.005 / E * np.abs(v).max() + 0.501 * scales[3]
    assert (np.abs(got - e @ v / E[:, None]).max(1) <= limit).all()

"""Paged attention whose CTAs form clusters: CTAs without keys of their own, which reach the exchange of the maxima while
others of their cluster may not have started, among many that are busy."""
import numpy as np
import pytest
import torch

import generation_reference as ref
from gpu_util import assert_same, ctx, dev, host

pytestmark = pytest.mark.gpu
SC = (0.05, 0.04, 0.03, 0.01)


@pytest.mark.parametrize("heads,kv", [(2, 2), (2, 1), (8, 1), (9, 1)])
@pytest.mark.parametrize("B,top", [(3, 9000), (40, 2000)])
def test_short_sequences_on_wide_clusters(heads, kv, B, top):
    """max_len asks for clusters of several CTAs; most sequences have keys for one of them, or none."""
    rng = np.random.default_rng(B + heads)
    lens = rng.integers(0, 70, B)
    lens[:2] = 0, top
    P = 16
    used = -(-lens // P)
    n_pages = int(used.sum()) + 1
    order = rng.permutation(n_pages).astype(np.int32)
    tables = np.full((B, -(-top // P)), -1, np.int32)
    at = np.concatenate([[0], np.cumsum(used)])
    for b in range(B):
        tables[b, :used[b]] = order[at[b]:at[b + 1]]
    kc, vc = (rng.integers(-127, 128, (n_pages, kv, P, 64)).astype(np.int8) for _ in range(2))
    q = rng.integers(-50, 51, (B, heads * 64)).astype(np.int8)
    want = ref.attention_decode(q, kc, vc, tables, lens, 0, 0, SC, 255)
    args = [dev(a) for a in (q, kc, vc, tables, lens.astype(np.int32))]
    outs = [ctx().ibert_attention_decode_i8(*args, top, heads, *SC)[0] for _ in range(20)]
    ctx().check()
    for out in outs:
        assert_same(host(out), want)
    assert torch.equal(args[4].cpu(), torch.from_numpy(lens.astype(np.int32)))

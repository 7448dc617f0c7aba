"""A step in which no request gets a token: every generation call takes tensors without rows."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2101_01321_b200 import binding


@pytest.fixture(scope="module")
def lib():
    from paper_2101_01321_b200 import build
    build.build()
    return binding.lib()


def test_no_tokens_need_no_slots(lib):
    """No tokens, a cache, and slots of an array without entries (which has no address); with tokens that is refused."""
    ctx, mem = C.create_string_buffer(1 << 16), C.create_string_buffer(1 << 12)     # (neither is looked into)
    at = [(C.addressof(mem) + 255) // 256 * 256 + 256 * i for i in range(4)]
    d = binding.RopeDesc(4, 2, 8, 64, 0, 16, 8, 100, at[0], None, None, 0.03, 0.03, 0.03, 0.03)
    assert lib.ibert_qkv_rope_i8(ctx, C.byref(d), None, 0, None, 0, None, None, at[2], at[3], None) == 0
    assert lib.ibert_qkv_rope_i8(ctx, C.byref(d), None, 0, None, 0, None, at[1], at[2], at[3], None) == 0
    for T, qkv, slots, k, v in ((1, at[0], None, at[2], at[3]), (0, None, None, at[2], None), (0, None, at[1], None, None)):
        assert lib.ibert_qkv_rope_i8(ctx, C.byref(d), qkv, T, at[0], 0, at[1], slots, k, v, None) == -1


@pytest.mark.gpu
def test_a_step_without_tokens():
    from gpu_util import ctx, dev, host
    i32, i8 = torch.int32, torch.int8
    lens = dev(np.array([5, 20], np.int32))
    tables, stack = dev(np.array([[0, -1], [1, 2]], np.int32)), dev(np.array([3, 4], np.int32))
    lens_out, n, cu, slots, pos = ctx().ibert_kv_slots(lens, torch.zeros(2, dtype=i32, device="cuda"), tables, stack,
                                                       torch.tensor([2], dtype=i32, device="cuda"), 16, 0)
    k, v = (torch.full((5, 2, 16, 64), 3, dtype=i8, device="cuda") for _ in range(2))
    rope = dev(binding.ibert_rope_rows(binding.ibert_rope_frequencies(64), 32))
    qkv = torch.empty(0, 8 * 64, dtype=torch.int16, device="cuda")
    for with_kv in (False, True):
        q, _ = ctx().ibert_qkv_rope_i8(qkv, 0.01, 4, 2, 0.1, 0.1, 0.1, rope=rope, positions=pos, slots=slots, k_cache=k, v_cache=v,
                                       with_kv=with_kv)
        assert q.shape == (0, (8 if with_kv else 4) * 64)
    out, _ = ctx().ibert_attention_window_i8(q, cu, 32, 4, 2, 0.1, 0.1, 0.1, 0.1)
    assert out.shape == (0, 256)
    out, _ = ctx().ibert_attention_decode_i8(q[:, :256], k, v, tables, lens_out, 32, 4, 0.1, 0.1, 0.1, 0.1, cu_seqlens=cu)
    assert out.shape == (0, 256)
    ctx().check()
    assert host(lens_out).tolist() == [5, 20] and host(n).tolist() == [2] and host(cu).tolist() == [0, 0, 0]
    assert (k == 3).all() and (v == 3).all()

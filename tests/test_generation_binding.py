"""What the binding hands to the library for the generation calls; the library is a stand-in, so no GPU is needed."""
import ctypes as C
import threading

import numpy as np
import torch

from paper_2101_01321_b200 import binding


def _context(monkeypatch, fake):
    monkeypatch.setattr(binding, "lib", lambda: fake)
    monkeypatch.setattr(binding, "_dev", lambda t, dtype: None if t is None else t.data_ptr())
    c = binding.Context(0)
    c.h = None                                     # (nothing to destroy)
    return c


class _Fake:
    def ibert_create(self, handle, device, stream):
        return 0


def test_head_norms_of_calls_at_once(monkeypatch):
    """Two threads, one context, each with its own factors: the library reads a call's factors while the other call is made."""
    inside, other_done, seen = threading.Event(), threading.Event(), {}

    class Fake(_Fake):
        def ibert_qkv_rope_i8(self, h, desc, qkv, T, *rest):
            if T == 1:
                inside.set()
                assert other_done.wait(30)
            d = binding.RopeDesc.from_buffer_copy(desc)
            seen[T] = [np.ctypeslib.as_array((C.c_double * 64).from_address(p)).copy() for p in (d.gamma_q, d.gamma_k)]
            return 0

    c = _context(monkeypatch, Fake())
    factors = {T: (np.arange(64) * T + 0.5, np.arange(64) - 7.0 * T) for T in (1, 2)}

    def call(T):
        c.ibert_qkv_rope_i8(torch.zeros(T, 3 * 64, dtype=torch.int8), 0.1, 1, 1, 0.1, 0.1, 0.1, *factors[T])

    first = threading.Thread(target=call, args=(1,))
    first.start()
    assert inside.wait(30)
    call(2)
    other_done.set()
    first.join(30)
    for T in (1, 2):
        assert np.array_equal(seen[T], factors[T]), T


def test_head_norms_in_any_form(monkeypatch):
    seen = []

    class Fake(_Fake):
        def ibert_qkv_rope_i8(self, h, desc, *rest):
            d = binding.RopeDesc.from_buffer_copy(desc)
            seen.append([p and np.ctypeslib.as_array((C.c_double * 64).from_address(p)).copy() for p in (d.gamma_q, d.gamma_k)])
            return 0

    c = _context(monkeypatch, Fake())
    x = torch.zeros(2, 3 * 64, dtype=torch.int8)
    g = np.linspace(-2, 2, 64)
    for q, k in ((g, g[::-1]), (g.astype(np.float32), list(g)), (torch.from_numpy(g), tuple(g)), (np.stack([g, g], 1)[:, 0], g)):
        c.ibert_qkv_rope_i8(x, 0.1, 1, 1, 0.1, 0.1, 0.1, q, k)
        assert np.array_equal(seen[-1], [np.asarray(q, np.float64), np.asarray(k, np.float64)])
    c.ibert_qkv_rope_i8(x, 0.1, 1, 1, 0.1, 0.1, 0.1)
    assert seen[-1] == [None, None]

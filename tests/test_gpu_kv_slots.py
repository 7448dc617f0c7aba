"""Block tables and slot maps on the GPU against the plain form: whole steps, in place, and everything that runs out."""
import threading

import numpy as np
import pytest
import torch

import generation_reference as ref
from paper_2101_01321_b200 import binding
from gpu_util import assert_same, ctx, dev, host

pytestmark = pytest.mark.gpu


def _state(rng, B, P, max_pages, longest, new_of, ended=0.2, spare=50):
    """Requests with scattered pages, and a stack with `spare` pages more than the step takes."""
    lens = rng.integers(0, min(longest, max_pages * P) + 1, B)
    new = np.minimum(new_of(rng, B), max_pages * P - lens)
    new[rng.random(B) < ended] = -rng.integers(1, 5)
    used = -(-lens // P)
    need = int((-(-(lens + np.maximum(new, 0)) // P) - used).sum())
    ids = rng.permutation(int(used.sum()) + need + spare).astype(np.int32)
    tables = np.full((B, max_pages), -7, np.int32)
    at = 0
    for b in range(B):
        tables[b, :used[b]] = ids[at:at + used[b]]
        at += used[b]
    stack = np.full(ids.size, -9, np.int32)
    free = ids[at:]
    stack[:free.size] = free
    return lens.astype(np.int32), new.astype(np.int32), tables, stack, np.array([free.size], np.int32)


def _check(lens, new, tables, stack, n_free, P, max_tokens, in_place=False, out_of_range=None):
    want = ref.kv_slots(lens, new, tables, stack, n_free[0], P, max_tokens)
    d = [dev(a) for a in (lens, new, tables, stack, n_free)]
    got = ctx().ibert_kv_slots(*d, P, max_tokens, **(dict(lens_out=d[0], n_free_out=d[4]) if in_place else {}))
    status = ctx().ibert_last_status()
    names = ("lens_out", "n_free_out", "cu_seqlens", "slots", "positions", "block_tables", "free_pages")
    for name, g, w in zip(names, [*got, d[2], d[3]], [want[0], np.array([want[1]]), *want[2:7]]):
        assert_same(host(g), w, name)
    assert status == (-8 if want[7] else 0)
    if out_of_range is not None:
        assert want[7] == out_of_range
    if not in_place:
        assert_same(host(d[0]), lens, "lens are left alone")
        assert_same(host(d[4]), n_free, "n_free is left alone")
    return want


ONE = lambda rng, B: np.ones(B, np.int64)  # noqa: E731
MANY = lambda rng, B: rng.integers(0, 300, B)  # noqa: E731


@pytest.mark.parametrize("P", [16, 32, 128, 256])
@pytest.mark.parametrize("B,max_pages,longest,new_of", [(1, 3, 40, ONE), (2, 40, 500, MANY), (31, 40, 600, ONE), (255, 20, 300, MANY),
                                                        (1024, 9, 140, ONE), (1025, 9, 140, ONE), (3000, 30, 200, MANY)])
@pytest.mark.parametrize("in_place", [False, True])
def test_step_matches_the_plain_form(P, B, max_pages, longest, new_of, in_place):
    rng = np.random.default_rng(B + P)
    st = _state(rng, B, P, max_pages, longest, new_of)
    _check(*st, P, int(np.maximum(st[1], 0).sum()) + 3, in_place, out_of_range=False)


def test_no_requests_no_tokens_no_pages():
    z = np.zeros(0, np.int32)
    _check(z, z, np.zeros((0, 5), np.int32), np.arange(4, dtype=np.int32), np.array([4], np.int32), 16, 3, out_of_range=False)
    _check(np.zeros(3, np.int32), np.zeros(3, np.int32), np.zeros((3, 5), np.int32), np.arange(4, dtype=np.int32), np.array([2], np.int32),
           16, 0, out_of_range=False)
    _check(np.zeros(3, np.int32), np.array([1, 0, 2], np.int32), np.zeros((3, 0), np.int32), np.zeros(0, np.int32), np.array([0], np.int32),
           16, 5, out_of_range=True)


def test_largest_batch():
    rng = np.random.default_rng(5)
    st = _state(rng, 8192, 16, 6, 90, ONE)
    _check(*st, 16, 8192, True, out_of_range=False)


@pytest.mark.parametrize("have", [0, 1, 5, 17, 40])
def test_stack_runs_out(have):
    rng = np.random.default_rng(have)
    lens, new, tables, stack, n_free = _state(rng, 24, 16, 30, 200, MANY, ended=0.0)
    want = _check(lens, new, tables, stack, np.array([have], np.int32), 16, int(new.sum()), out_of_range=True)
    assert want[1] == 0 and (want[3] == -1).any()


def test_pages_given_back_are_taken_in_the_same_step():
    lens = np.array([40, 5, 33, 0], np.int32)
    new = np.array([-1, 60, -1, 20], np.int32)
    tables = np.arange(20, dtype=np.int32).reshape(4, 5)
    want = _check(lens, new, tables, np.full(12, 99, np.int32), np.array([1], np.int32), 16, 80, out_of_range=False)   # 1 + 6 pages, 4 + 2 taken
    assert set(want[3][want[3] >= 0] // 16) - {5} <= {0, 1, 2, 10, 11, 12, 99}


def test_what_is_out_of_range_is_cut_and_reported():
    rng = np.random.default_rng(3)
    lens, new, tables, stack, n_free = _state(rng, 20, 16, 12, 100, MANY)
    _check(lens, new, tables, stack, n_free, 16, int(np.maximum(new, 0).sum()) - 1, out_of_range=True)     # too many tokens
    _check(lens, new, tables, stack, n_free, 16, 7, out_of_range=True)
    more = new.copy()
    more[3] = 16 * 12 - lens[3] + 1                                                                        # table full
    _check(lens, more, tables, stack, n_free, 16, int(np.maximum(more, 0).sum()), out_of_range=True)
    bad = lens.copy()
    bad[2], bad[5] = -3, 16 * 12 + 1
    _check(bad, np.where(np.arange(20) == 5, -1, new).astype(np.int32), tables, stack, n_free, 16, 5000, out_of_range=True)
    _check(lens, new, tables, stack, np.array([-2], np.int32), 16, 5000, out_of_range=True)
    _check(lens, new, tables, stack, np.array([stack.size + 1], np.int32), 16, 5000, out_of_range=True)
    huge = np.full(20, 2 ** 31 - 1, np.int32)
    _check(lens, huge, tables, stack, n_free, 16, 50, out_of_range=True)


def test_tables_wider_than_the_cache_and_views_off_16_bytes():
    rng = np.random.default_rng(9)
    lens, new, tables, stack, n_free = _state(rng, 7, 16, 100, 60, ONE)
    hold = torch.zeros(lens.size + 1, dtype=torch.int32, device="cuda")
    hold[1:] = dev(lens)
    got = ctx().ibert_kv_slots(hold[1:], dev(new), dev(tables), dev(stack), dev(n_free), 16, 9)
    ctx().check()
    want = ref.kv_slots(lens, new, tables, stack, n_free[0], 16, 9)
    assert_same(host(got[0]), want[0])
    assert_same(host(got[3]), want[3])


def test_many_steps_of_one_pool():
    """Requests come, grow and end; at every time no page is held twice and none is lost."""
    rng = np.random.default_rng(1)
    B, P, max_pages, pool = 12, 16, 8, 70
    tables = torch.full((B, max_pages), -1, dtype=torch.int32, device="cuda")
    stack, n_free = torch.arange(pool, dtype=torch.int32, device="cuda"), torch.tensor([pool], dtype=torch.int32, device="cuda")
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    for step in range(40):
        now = host(lens)
        new = np.where(rng.random(B) < 0.1, -1, np.minimum(rng.integers(0, 9, B), max_pages * P - now)).astype(np.int32)
        ctx().ibert_kv_slots(lens, dev(new), tables, stack, n_free, P, 200, lens_out=lens, n_free_out=n_free)
        t, n, s = host(tables), host(lens), host(stack)[:int(n_free)]
        if ctx().ibert_last_status():
            assert int(n_free) == 0
        held = np.concatenate([t[b, :-(-n[b] // P)] for b in range(B)])
        held = held[held >= 0]
        assert np.unique(np.concatenate([held, s])).size == held.size + s.size <= pool


def test_two_host_threads_with_batches_of_different_sizes():
    """Every launch finds the shared memory that it asks for, whatever another thread launches in between.  (The step is not in
    place, so it gives the same again and again.)"""
    rng = np.random.default_rng(12)
    work, errors = [], []
    for B in (8192, 3000):
        st = _state(rng, B, 16, 6, 90, ONE)
        d, sizes = [dev(a) for a in st], dict(lens_out=B, n_free_out=1, cu_seqlens=B + 1, slots=B, positions=B)
        out = {name: torch.empty(n, dtype=torch.int32, device="cuda") for name, n in sizes.items()}
        work.append((binding.Context(0, stream=torch.cuda.Stream()), d, out, ref.kv_slots(*st[:4], st[4][0], 16, B)))
    torch.cuda.synchronize()
    start = threading.Barrier(len(work))

    def run(c, d, out):
        try:
            start.wait(30)
            for _ in range(1500):
                c.ibert_kv_slots(*d, 16, **out)
        except Exception as e:  # noqa: BLE001 -- for the test's own thread
            errors.append(e)

    threads = [threading.Thread(target=run, args=w[:3]) for w in work]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors
    for c, d, out, want in work:
        c.check()
        for g, w in zip([*out.values(), d[2], d[3]], [want[0], np.array([want[1]]), *want[2:7]]):
            assert_same(host(g), w)

"""Refusals, failures and page tables of chunks under a mask, on the CPU (tests/chunk_host.py)."""
import ctypes
import math
import random

import pytest

import chunk_host as chunk
import pool_host as host
from chunk_host import KEPT, KEYS, LSE, ROWS, VALUES, WEIGHTS, Pool
from paper_2604_20289_amd.xcache import (XC_ERR_HIP, XC_ERR_INVALID_ARG, XC_ERR_OOM, XC_ERR_STATE, XC_ERR_UNSUPPORTED,
                                         XC_F32, XC_OK)

pytestmark = pytest.mark.skipif(host.shutil.which("g++") is None, reason="no host compiler")


def lib():
    return chunk.lib()


def test_masks_and_rows_are_checked():
    pool = Pool(n_pages=400)
    a, b = pool.new(100), pool.new(50)
    for mask in ((-1, 0, 0), (0, -1, 0), (0, 0, -1)):
        assert pool.set([a], [1], *mask) == XC_ERR_INVALID_ARG
    for seqs, new in (([a, a], [1, 1]), ([a, 63], [1, 1]), ([-1], [1]), ([a], [101]), ([a], [-1])):
        assert pool.set(seqs, new) == XC_ERR_INVALID_ARG
    assert lib().xc_chunk_set(None, 0, None, None, None) == XC_ERR_INVALID_ARG
    assert lib().xc_chunk_set(pool.b, 1, None, None, None) == XC_ERR_INVALID_ARG
    assert pool.attention() == XC_ERR_STATE and pool.weights() == XC_ERR_STATE
    # the largest numbers that a mask's fields can hold, no mask, no rows
    big = 2 ** 31 - 1
    for mask in ((big, big, big), (1, big, big), (big, 1, big), (0, 0, big)):
        assert pool.set([a, b], [100, 1], *mask) == XC_OK and pool.attention() == XC_OK and pool.weights() == XC_OK
    assert lib().xc_chunk_set(pool.b, 1, host.ints(a), host.ints(7), None) == XC_OK and pool.attention() == XC_OK
    launches = chunk.info()["launches"]
    for seqs, new in (([], []), ([a, b], [0, 0])):
        assert pool.set(seqs, new) == XC_OK
        assert pool.attention(None, None, None) == XC_OK and pool.weights(None, None, None) == XC_OK
    assert chunk.info()["launches"] == launches
    pool.close()


def test_which_batch_serves_which_attention():
    pool = Pool(n_pages=400)
    a = pool.new(100)
    branch = lambda: lib().xc_branch_attention(pool.b, 0, ROWS, 64, 0.0, ROWS + (1 << 38), 64)  # noqa: E731
    assert lib().xc_batch_set(pool.b, 1, host.ints(a), host.ints(3)) == XC_OK
    assert branch() == XC_OK and pool.attention() == XC_ERR_STATE and pool.weights() == XC_ERR_STATE
    assert pool.set([a], [3]) == XC_OK
    assert branch() == XC_ERR_STATE and pool.attention() == XC_OK and pool.weights() == XC_OK
    assert lib().xc_batch_set(pool.b, 1, host.ints(a), host.ints(3)) == XC_OK and branch() == XC_OK
    assert pool.attention() == XC_ERR_STATE
    # a table that changed
    assert pool.set([a], [3]) == XC_OK and lib().xc_seq_extend(pool.p, 1, host.ints(a), host.ints(1)) == XC_OK
    assert pool.attention() == XC_ERR_STATE and pool.weights() == XC_ERR_STATE
    pool.close()


def test_arguments_of_attention_and_weights_are_checked():
    pool = Pool(n_pages=400, q_heads=4, kv_heads=2, n_blocks=2)
    a, b = pool.new(100), pool.new(150)
    assert pool.set([a, b], [10, 20]) == XC_OK
    w, far = 4 * 64, 1 << 38
    launches = chunk.info()["launches"]
    for kw in (dict(q=None), dict(out=None), dict(block=-1), dict(block=2), dict(ld=w - 8), dict(out_ld=w - 8), dict(ld=w + 4),
               dict(out_ld=w + 1), dict(q=ROWS + 8), dict(out=ROWS + far + 2), dict(lse=LSE + 2), dict(scale=-1.0),
               dict(scale=math.nan), dict(scale=math.inf), dict(scale=1e-45), dict(out=ROWS), dict(out=ROWS + 2 * w),
               dict(out=KEYS), dict(out=VALUES + 32), dict(lse=ROWS), dict(lse=ROWS + far), dict(lse=KEYS + 64),
               dict(ld=(1 << 36) + 8)):
        assert pool.attention(**kw) == XC_ERR_INVALID_ARG, kw
    for kw in (dict(q=None), dict(lse=None), dict(w=None), dict(block=2), dict(q_ld=w - 8), dict(q_ld=w + 4), dict(q=ROWS + 8),
               dict(lse=LSE + 1), dict(w=WEIGHTS + 2), dict(ld=149), dict(ld=-1), dict(ld=(1 << 36) + 1), dict(decay=-0.5),
               dict(decay=math.nan), dict(decay=math.inf), dict(scale=-1.0), dict(w=ROWS), dict(w=LSE), dict(w=KEYS),
               dict(w=ROWS + 30 * w * 2 - 4)):
        assert pool.weights(**kw) == XC_ERR_INVALID_ARG, kw
    assert pool.weights(q_ld=1 << 27) == XC_ERR_UNSUPPORTED
    assert chunk.info()["launches"] == launches
    # beside each other, no log-sum-exp, the narrowest weights
    assert pool.attention(out=ROWS + 2 * w, ld=2 * w, out_ld=2 * w, lse=None) == XC_OK
    assert pool.weights(ld=150, decay=0.0) == XC_OK and pool.weights(w=ROWS + 30 * w * 2) == XC_OK
    pool.close()


def test_arguments_of_evictions_are_checked():
    pool = Pool(n_pages=400)
    a, b = pool.new(100), pool.new(50)
    before, launches = pool.tables(), chunk.info()["launches"]
    for args, kw in ((([a, a], [1, 1]), {}), (([63], [1]), {}), (([a], [-1]), {}), (([a], [10]), dict(sinks=-1)),
                     (([a], [10]), dict(recent=-1)), (([a], [10]), dict(sinks=6, recent=5)),
                     (([a], [10]), dict(sinks=2 ** 31 - 1, recent=2 ** 31 - 1)), (([a], [10]), dict(w=None)),
                     (([a], [10]), dict(ld=99)), (([b, a], [10, 10]), dict(kept_ld=9)), (([a], [10]), dict(w=WEIGHTS + 2)),
                     (([a], [10]), dict(kept=KEPT + 1)), (([a], [10]), dict(w=KEYS)), (([a], [10]), dict(kept=VALUES)),
                     (([a], [10]), dict(kept=WEIGHTS)), (([a], [10]), dict(ld=-1)), (([a], [10]), dict(kept_ld=-1)),
                     (([a], [100]), dict(kept_ld=99))):
        assert pool.evict(*args, **kw) == XC_ERR_INVALID_ARG, (args, kw)
    assert lib().xc_chunk_evict(None, 0, None, None, 0, 0, None, 0, None, 0) == XC_ERR_INVALID_ARG
    assert lib().xc_chunk_evict(pool.b, 1, None, None, 0, 0, None, 0, None, 0) == XC_ERR_INVALID_ARG
    assert pool.tables() == before and chunk.info()["launches"] == launches
    # nothing shrinks: nothing is launched, unless the numbers are asked for
    assert pool.evict([a, b], [100, 50], w=None, kept=None, kept_ld=0) == XC_OK and chunk.info()["launches"] == launches
    assert pool.evict([a, b], [1000, 2 ** 31 - 1], sinks=2000, w=None) == XC_OK and chunk.info()["launches"] == launches + 1
    assert pool.tables() == before
    assert pool.evict([], []) == XC_OK
    pool.close()


def test_changes_are_refused_while_the_stream_is_captured():
    pool = Pool(n_pages=400)
    a = pool.new(100)
    assert pool.set([a], [3]) == XC_OK
    before = pool.tables()
    lib().fake_set(0, 1)
    assert pool.set([a], [4]) == XC_ERR_STATE and pool.evict([a], [10]) == XC_ERR_STATE
    assert pool.attention() == XC_OK and pool.weights() == XC_OK
    lib().fake_set(0, 0)
    assert pool.tables() == before and pool.attention() == XC_OK
    # ... of another stream: allocations are let through
    lib().fake_elsewhere(1)
    assert pool.set([a], [100]) == XC_OK and pool.evict([a], [10]) == XC_OK
    lib().fake_elsewhere(0)
    assert chunk.info()["broken_captures"] == 0
    pool.close()


@pytest.mark.parametrize("where", ["host", "device"])
@pytest.mark.parametrize("dtype", [None, XC_F32])
def test_memory_that_ends_in_the_middle_of_a_call(where, dtype):
    """Every allocation of a batch under a mask and of an eviction in turn: whole, or nothing has changed."""
    statuses = {"set": [], "evict": []}
    for n in range(400):
        pool = Pool(n_pages=3000, **({} if dtype is None else dict(dtype=dtype)))
        kids = pool.fork(pool.new(5000), 6)
        assert lib().xc_seq_extend(pool.p, 6, host.ints(*kids), host.ints(1, 2, 3, 4, 5, 600)) == XC_OK
        faults = (n, -1, -1) if where == "device" else (-1, n, -1)
        lib().fake_faults(*faults)
        status = pool.set(kids, [1, 2, 3, 4, 5, 600], 1, 900, 8)
        ahead = chunk.info()["fault_ahead"]
        lib().fake_faults(-1, -1, -1)
        statuses["set"].append(status)
        if status != XC_OK:
            assert status == XC_ERR_OOM and pool.attention() == XC_ERR_STATE and pool.weights() == XC_ERR_STATE
            assert lib().xc_chunk_attention(pool.b, 0, None, 64, 0.0, None, 64, None) == XC_ERR_STATE
            assert pool.set(kids, [1, 2, 3, 4, 5, 600]) == XC_OK
        assert pool.attention() == XC_OK and pool.weights() == XC_OK
        before = pool.tables()
        lib().fake_faults(*faults)
        status = pool.evict(kids, [1000, 5, 5, 70, 9000, 400], 3, 2)
        ahead += chunk.info()["fault_ahead"]
        lib().fake_faults(-1, -1, -1)
        statuses["evict"].append(status)
        if status != XC_OK:
            assert status == XC_ERR_OOM
            assert pool.tables() == before and pool.attention() == XC_OK
            assert pool.evict(kids, [1000, 5, 5, 70, 9000, 400], 3, 2) == XC_OK
        pool.close()
        if ahead == 2:
            break
    for which, got in statuses.items():
        assert got[-1] == XC_OK and XC_ERR_OOM in got and set(got) <= {XC_OK, XC_ERR_OOM}, (which, got)
    assert ahead == 2


@pytest.mark.parametrize("shape", [dict(q_heads=4, kv_heads=4, head_dim=128), dict(head_dim=32, dtype=XC_F32)], ids=["few", "f32"])
def test_refused_sizes_leave_the_rows_and_their_memory(shape):
    """More workgroups than a launch has: refused before the buffers of the rows set before are given up for larger ones."""
    pool = Pool(n_pages=1 << 22, page_tokens=256, max_seqs=4, **shape)
    a, b = pool.new(100), pool.new((1 << 29) + 100000)
    assert pool.set([a], [1]) == XC_OK and chunk.info()["live_bytes"] > 0
    before = chunk.info()["live_bytes"]
    assert pool.set([b], [1]) == XC_ERR_UNSUPPORTED
    assert chunk.info()["live_bytes"] == before
    assert pool.attention() == XC_OK and pool.weights() == XC_OK
    pool.close()


def test_pages_that_run_out_and_launches_that_fail():
    pool = Pool(n_pages=20)
    a = pool.new(160)
    b = pool.fork(a, 1)[0]
    assert pool.evict([b], [159]) == XC_OK  # ten pages are free
    c = pool.fork(a, 1)[0]
    before = pool.tables()
    assert pool.evict([c], [1]) == XC_ERR_OOM and pool.tables() == before
    assert pool.evict([c], [16], sinks=16) == XC_OK  # a page of first tokens stays shared
    assert pool.evict([a], [3]) == XC_ERR_OOM and lib().xc_seq_free(pool.p, 1, host.ints(b)) == XC_OK
    lib().fake_faults(-1, -1, 0)
    assert pool.evict([a], [3]) == XC_ERR_HIP
    lib().fake_faults(-1, -1, -1)
    assert pool.evict([a], [2]) == XC_ERR_HIP and pool.set([a], [1]) == XC_ERR_HIP and pool.attention() == XC_ERR_HIP
    pool.close()


def test_the_pools_device_serves_every_call():
    pool = Pool(n_pages=400)  # on device 0
    a = pool.new(100)
    lib().fake_set(5, 0)
    for call in (lambda: pool.set([a], [9]), pool.attention, pool.weights, lambda: pool.evict([a], [10])):
        assert call() == XC_OK and chunk.info()["device"] == 5 and chunk.info()["launched_on"] == 0
    lib().fake_set(0, 0)
    pool.close()


def test_tables_of_random_evictions():
    """Growth, forks, trims, frees and evictions in any order, against lists of pages: which page is kept, which is new, which
    is given up, by the rules of include/xcache.h."""
    rng = random.Random(5)
    for page in (16, 64):
        pool = Pool(n_pages=300, page_tokens=page, max_seqs=12)
        refs = [0] * 300
        seqs = {}
        pool.evictions = 0

        def take():
            p = refs.index(0)
            refs[p] = 1
            return p

        for step in range(1500):
            what = rng.random()
            if what < 0.15 and len(seqs) < 12:
                src = rng.choice(list(seqs)) if seqs and rng.random() < 0.7 else None
                if src is None:
                    seqs[pool.new()] = [0, 0, []]
                else:
                    s = pool.fork(src, 1)[0]
                    seqs[s] = [seqs[src][0], seqs[src][1], list(seqs[src][2])]
                    for p in seqs[s][2]:
                        refs[p] += 1
            elif what < 0.25 and seqs:
                s = rng.choice(list(seqs))
                assert lib().xc_seq_free(pool.p, 1, host.ints(s)) == XC_OK
                for p in seqs.pop(s)[2]:
                    refs[p] -= 1
            elif what < 0.5 and seqs:
                s, n = rng.choice(list(seqs)), rng.randint(1, 5 * page)
                first, have, pages = seqs[s]
                copy = (first + have) % page and refs[pages[-1]] > 1
                need = -(-(first + have + n) // page) - len(pages) + bool(copy)
                ok = need <= refs.count(0)
                assert lib().xc_seq_extend(pool.p, 1, host.ints(s), host.ints(n)) == (XC_OK if ok else XC_ERR_OOM)
                if ok:
                    if copy:
                        refs[pages[-1]] -= 1
                        pages[-1] = take()
                    while len(pages) * page < first + have + n:
                        pages.append(take())
                    seqs[s][1] += n
            elif what < 0.6 and seqs:
                s = rng.choice(list(seqs))
                first, have, pages = seqs[s]
                front = rng.randint(0, have // 3)
                assert lib().xc_seq_trim(pool.p, s, front, 0) == XC_OK
                if front:
                    gone = (first + front) // page if have - front else len(pages)
                    for p in pages[:gone]:
                        refs[p] -= 1
                    seqs[s] = [(first + front) % page if have - front else 0, have - front, pages[gone:]]
            elif seqs:
                some = rng.sample(list(seqs), rng.randint(1, min(4, len(seqs))))
                sinks = rng.choice([0, 0, rng.randint(0, 3 * page)])
                keep = [max(rng.randint(0, seqs[s][1] + 5), sinks) for s in some]
                held, plans, gone = list(refs), [], []
                for s, k in zip(some, keep):
                    first, have, pages = seqs[s]
                    if k >= have:
                        plans.append(None)
                        continue
                    n = -(-(first + k) // page) if k else 0
                    plans.append([p if held[p] == 1 or (j + 1) * page <= first + sinks else None for j, p in enumerate(pages[:n])])
                ok = sum(t.count(None) for t in plans if t is not None) <= refs.count(0)
                assert pool.evict(some, keep, sinks) == (XC_OK if ok else XC_ERR_OOM)
                if ok:
                    pool.evictions += any(t is not None for t in plans)
                    for s, k, t in zip(some, keep, plans):
                        if t is None:
                            continue
                        first, have, pages = seqs[s]
                        t = [take() if p is None else p for p in t]
                        gone += [p for j, p in enumerate(pages) if j >= len(t) or t[j] != p]
                        seqs[s] = [first if k else 0, k, t]
                    for p in gone:
                        refs[p] -= 1
            for s in range(12):
                want = seqs.get(s)
                got = pool.table(s)
                assert (got is None) == (want is None) and (got is None or list(got) == want), (step, s)
            live = ctypes.c_int32()
            assert lib().xc_pool_info(pool.p, ctypes.byref(live), None, None) == XC_OK
            assert live.value == sum(r > 0 for r in refs)
        assert pool.evictions > 200
        pool.close()

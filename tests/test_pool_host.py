"""Failures and memory of the branching cache's host side, forced on the CPU (tests/pool_host.py)."""
import pytest

import pool_host as host
from paper_2604_20289_amd.xcache import (XC_ERR_HIP, XC_ERR_INVALID_ARG, XC_ERR_OOM, XC_ERR_STATE, XC_ERR_UNSUPPORTED,
                                         XC_OK)

pytestmark = pytest.mark.skipif(host.shutil.which("g++") is None, reason="no host compiler")


def _grown(pool, n=6, history=5000):
    parent = pool.new(history)
    kids = pool.fork(parent, n)
    assert host.lib().xc_seq_extend(pool.p, n, host.ints(*kids), host.ints(*range(1, n + 1))) == XC_OK
    return kids


@pytest.mark.parametrize("where", ["host", "device"])
def test_a_batch_that_runs_out_of_memory_has_no_rows(where):
    """Every allocation of xc_batch_set in turn: either the call is whole (for pieces there is another way), or the batch is
    without rows."""
    statuses = []
    for n in range(200):
        pool = host.HostPool(n_pages=2000)
        kids, b = _grown(pool), pool.batch()
        assert host.set_batch(b, kids[:1], [1]) == XC_OK and host.attention(b) == XC_OK
        host.lib().fake_faults(*((n, -1) if where == "device" else (-1, n)), -1)
        status = host.set_batch(b, kids, [1] * len(kids))
        through = host.info()["fault_ahead"]
        host.lib().fake_faults(-1, -1, -1)
        statuses.append(status)
        if status == XC_ERR_OOM:
            launches = host.info()["launches"]
            assert host.attention(b) == XC_ERR_STATE
            assert host.lib().xc_branch_attention(b, 0, None, 64, 0.0, None, 64) == XC_ERR_STATE
            assert host.info()["launches"] == launches
            assert host.set_batch(b, kids, [1] * len(kids)) == XC_OK
        assert host.attention(b) == XC_OK
        assert host.lib().xc_batch_destroy(b) == XC_OK
        assert host.info()["freed_unknown"] == 0 and host.info()["freed_in_use"] == 0 and host.info()["blocks"] == 0
        pool.close()
        if through:
            break
    if where == "device":  # pieces, tables, staging memory
        assert statuses == [XC_OK, XC_ERR_OOM, XC_ERR_OOM, XC_OK]
    else:
        assert statuses[-1] == XC_OK and set(statuses[:-1]) == {XC_ERR_OOM} and len(statuses) > 20


def test_refused_rows_leave_the_earlier_ones():
    pool = host.HostPool(n_pages=70000, page_tokens=256)
    s, b = pool.new((1 << 24) + 1), pool.batch()
    assert host.set_batch(b, [s], [2]) == XC_OK
    for new, status in (((1 << 24) + 1, XC_ERR_UNSUPPORTED), ((1 << 24) + 2, XC_ERR_INVALID_ARG), (-1, XC_ERR_INVALID_ARG)):
        assert host.set_batch(b, [s], [new]) == status
        assert host.attention(b) == XC_OK
    host.lib().xc_batch_destroy(b)
    pool.close()


def test_a_failed_launch_sticks():
    pool = host.HostPool(n_pages=2000)
    kids, b = _grown(pool), pool.batch()
    host.lib().fake_faults(-1, -1, 0)
    assert host.set_batch(b, kids, [1] * len(kids)) == XC_ERR_HIP
    assert host.attention(b) == XC_ERR_HIP and host.set_batch(b, kids, [1] * len(kids)) == XC_ERR_HIP
    assert host.lib().xc_batch_destroy(b) == XC_OK
    pool.close()


def test_tables_are_unchanged_where_the_host_runs_out_of_memory():
    """Every allocation of a fork, a growth, a free and a compaction in turn."""
    pool = host.HostPool(n_pages=400, max_seqs=40)
    kids = _grown(pool, history=37)
    lib, n = host.lib(), len(kids)

    def tables():
        out = []
        for s in range(40):
            first, tokens, count, pages = host.ints(0), host.ints(0), (host.ctypes.c_size_t * 1)(), host.ints(*[0] * 400)
            if lib.xc_seq_pages(pool.p, s, first, tokens, pages, 400, count) == XC_OK:
                out.append((s, first[0], tokens[0], list(pages[:count[0]])))
        live = [host.ctypes.c_int32() for _ in range(3)]
        assert lib.xc_pool_info(pool.p, *map(host.ctypes.byref, live)) == XC_OK
        return out, [x.value for x in live]

    assert lib.xc_seq_free(pool.p, 1, host.ints(kids[0])) == XC_OK  # leaves a hole to compact into
    kids, n = kids[1:], n - 1
    for call in (lambda: lib.xc_seq_fork(pool.p, kids[0], 3, host.ints(0, 0, 0)),
                 lambda: lib.xc_seq_extend(pool.p, n, host.ints(*kids), host.ints(*[20] * n)),
                 lambda: lib.xc_seq_free(pool.p, 2, host.ints(kids[0], kids[2])),
                 lambda: lib.xc_pool_compact(pool.p, None)):
        before = tables()
        for i in range(100):
            lib.fake_faults(-1, i, -1)
            status = call()
            lib.fake_faults(-1, -1, -1)
            if status == XC_OK:
                break
            assert status == XC_ERR_OOM and tables() == before
        assert status == XC_OK and 0 < i < 100
    pool.close()


def test_buffers_that_became_too_small_are_released():
    """A batch that grows step by step holds what it needs and a reserve, and nothing goes while work reads it."""
    pool = host.HostPool(n_pages=30000, q_heads=8, kv_heads=8, head_dim=128, max_seqs=400)
    parent, b = pool.new(9000), pool.batch()
    kids = pool.fork(parent, 300)
    assert host.lib().xc_seq_extend(pool.p, 300, host.ints(*kids), host.ints(*[20] * 300)) == XC_OK
    fresh = {}
    for n in range(2, 300, 20):  # what a batch of its own takes
        one, before = pool.batch(), host.info()["live_bytes"]
        assert host.set_batch(one, kids[:n], [1] * n) == XC_OK
        fresh[n] = host.info()["live_bytes"] - before
        host.lib().xc_batch_destroy(one)
    assert host.info()["live_bytes"] == 0
    most = 0
    for n in range(2, 300, 20):
        assert host.set_batch(b, kids[:n], [1] * n) == XC_OK and host.attention(b, 8 * 128) == XC_OK
        assert host.info()["n_slots"] > 0
        most = max(most, fresh[n])
        assert host.info()["live_bytes"] <= 1.25 * most
    assert host.info()["freed_in_use"] == 0 and host.info()["freed_unknown"] == 0
    host.lib().xc_batch_destroy(b)
    assert host.info()["live_bytes"] == 0 and host.info()["freed_in_use"] == 0
    pool.close()


def test_without_memory_for_pieces_the_rows_go_without():
    pool = host.HostPool(n_pages=30000, q_heads=8, kv_heads=8, head_dim=128, max_seqs=400)
    parent, b = pool.new(9000), pool.batch()
    kids = pool.fork(parent, 300)
    assert host.lib().xc_seq_extend(pool.p, 300, host.ints(*kids), host.ints(*[20] * 300)) == XC_OK
    assert host.set_batch(b, kids, [1] * 300) == XC_OK and host.attention(b, 8 * 128) == XC_OK
    assert host.info()["n_slots"] > 0
    pieces = 300 * 8 * (4 * 128 + 8)
    host.lib().xc_batch_destroy(b)
    b = pool.batch()
    tables = 4 * 300 * (-(-9020 // 16)) * 3  # table entries, and room for what else a row and a unit need
    host.lib().fake_memory(tables + 2 * pieces - 1)
    assert host.set_batch(b, kids, [1] * 300) == XC_OK and host.attention(b, 8 * 128) == XC_OK
    assert host.info()["n_slots"] == 0
    host.lib().xc_batch_destroy(b)
    pool.close()


def test_columns_of_one_buffer_are_no_overlap():
    """Rows of one stride that lie beside each other are taken, in either order; any byte in common is refused."""
    pool = host.HostPool(q_heads=4, kv_heads=2, head_dim=64)  # q and out rows of 256 elements, qkv rows of 512
    s, b = pool.new(9), pool.batch()
    assert host.set_batch(b, [s], [7]) == XC_OK
    lib, at = host.lib(), host.ROWS

    def attention(q, out, q_ld, out_ld):
        return lib.xc_branch_attention(b, 0, at + 2 * q, q_ld, 0.0, at + 2 * out, out_ld)

    def norms(qkv, ld, q, q_ld):
        return lib.xc_qk_norm_rope(b, 0, at + 2 * qkv, ld, 16, 16, None, 1, 2.0, at + 2 * q, q_ld)

    for q, out in ((0, 256), (256, 0), (0, 512 - 256), (8, 264), (0, 512 + 256), (512 + 256, 0), (0, 7 * 512)):
        assert attention(q, out, 512, 512) == XC_OK, (q, out)
    for q, out in ((0, 0), (0, 248), (248, 0), (0, 264), (264, 0), (0, 512), (512, 0), (0, 512 + 248), (0, 6 * 512 + 248)):
        assert attention(q, out, 512, 512) == XC_ERR_INVALID_ARG, (q, out)
    # of other strides: none of one's bytes between the first and the last of the other's
    assert attention(0, 256, 512, 520) == XC_ERR_INVALID_ARG
    assert attention(0, 6 * 512 + 256, 512, 520) == XC_OK and attention(6 * 520 + 256, 0, 512, 520) == XC_OK
    for qkv, q in ((0, 512), (256, 0), (256, 768), (0, 768 + 512)):
        assert norms(qkv, 768, q, 768) == XC_OK, (qkv, q)
    for qkv, q in ((0, 504), (0, 520), (0, 768), (264, 0), (248, 0), (0, 0)):
        assert norms(qkv, 768, q, 768) == XC_ERR_INVALID_ARG, (qkv, q)
    # the page buffers, whole
    pages = host.KEYS - at
    assert norms(0, 512, pages // 2, 256) == XC_ERR_INVALID_ARG and attention(0, pages // 2 + 64, 256, 256) == XC_ERR_INVALID_ARG
    lib.xc_batch_destroy(b)
    pool.close()


def test_another_streams_capture_is_left_alone():
    """While some other stream is captured, in the mode that forbids allocations to everybody, a batch grows, is set anew and
    goes; the thread's mode is what it was."""
    pool = host.HostPool(n_pages=2000)
    kids, b, other = _grown(pool), pool.batch(), pool.batch()
    mode = host.info()["mode"]
    assert host.set_batch(b, kids[:1], [1]) == XC_OK and host.set_batch(other, kids[:1], [1]) == XC_OK
    host.lib().fake_elsewhere(1)
    assert host.set_batch(b, kids, [1] * len(kids)) == XC_OK and host.attention(b) == XC_OK
    assert host.info()["n_slots"] > 0
    assert host.lib().xc_batch_destroy(other) == XC_OK and host.lib().xc_batch_destroy(b) == XC_OK
    assert host.info()["live_bytes"] == 0 and host.info()["freed_unknown"] == 0
    assert host.info()["broken_captures"] == 0 and host.info()["mode"] == mode
    host.lib().fake_elsewhere(0)
    pool.close()

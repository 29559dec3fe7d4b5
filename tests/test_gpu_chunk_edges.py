"""Where chunks under a mask can go wrong on the GPU: heads and rows that divide nothing, strides, offsets past 32 bits, graphs
of several batches, work in flight, many evictions at once, and all of the operators in a run together."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import branch_reference as ref  # noqa: E402
import chunk_reference as chunk  # noqa: E402
from paper_2604_20289_amd import xcache  # noqa: E402
from paper_2604_20289_amd.xcache import Batch, Pool, XCacheError  # noqa: E402
from test_gpu_branches import BF16, F32, grow, make, pages_for, stream, write  # noqa: E402
from test_gpu_chunks import check, evict_check, p_eps  # noqa: E402


# ---------------------------------------------------------------- heads, rows

FEW = [(1, 1, 64), (2, 1, 128), (3, 1, 64), (4, 1, 128), (5, 1, 128), (7, 1, 64), (12, 1, 64), (6, 3, 64), (2, 10, 128), (1, 21, 128),
       (1, 21, 64)]


@pytest.mark.parametrize("kv,group,d", FEW)
@pytest.mark.parametrize("branches", [[(0, 1)], [(0, 1), (5, 2)], [(0, 1), (300, 1), (0, 1)], [(130, 3)]], ids=str)
def test_few_rows_of_any_number_of_heads(branches, kv, group, d):
    """Sequences whose query rows fit into one workgroup, three at most (times 21 heads); histories shared and not."""
    for history, drop in ((777, 5), (33, 0), (0, 0)):
        pool = make(BF16, pages=pages_for(history, branches, 16), kv=kv, heads=kv * group, page=16, d=d, seqs=len(branches) + 1)
        _, seqs = grow(pool, history, drop, branches)
        batch, new = Batch(pool), [n for _, n in branches]
        for mask in ((1, 0, 0), (0, 0, 0), (2, 100, 5), (1, 1, 0)):
            batch.set_chunk(seqs, new, *mask)
            check(pool, batch, seqs, new, mask)


@pytest.mark.parametrize("kv,group,d,dtype,rows", [
    (2, 1, 64, BF16, 65), (2, 1, 128, BF16, 257), (1, 3, 64, BF16, 43), (3, 5, 128, BF16, 77), (1, 65, 64, BF16, 9),
    (1, 100, 128, BF16, 33), (2, 128, 64, BF16, 3), (1, 64, 128, BF16, 65), (1, 2, 64, BF16, 513), (12, 1, 128, BF16, 130),
    (1, 3, 32, F32, 31), (2, 5, 64, F32, 40), (1, 29, 128, F32, 5), (3, 1, 32, F32, 97), (1, 32, 64, F32, 33)])
def test_many_rows_of_any_number_of_heads(kv, group, d, dtype, rows):
    """Query rows that end inside a stage, and stages that begin inside a token's heads."""
    branches = [(40, rows), (0, 1), (3, 0), (7, rows // 2)]
    pool = make(dtype, pages=pages_for(400, branches, 32), kv=kv, heads=kv * group, page=32, d=d, seqs=5)
    _, seqs = grow(pool, 400, 9, branches)
    batch, new = Batch(pool), [n for _, n in branches]
    for mask in ((1, 0, 0), (0, 0, 0), (6, 150, 9), (2, 1, 0)):
        batch.set_chunk(seqs, new, *mask)
        check(pool, batch, seqs, new, mask)


@pytest.mark.parametrize("kv,d", [(12, 128), (5, 128), (3, 128), (1, 128), (4, 64), (2, 64), (1, 64)])
def test_few_sequences_of_several_rows(kv, d):
    """One to three sequences whose rows fill a workgroup: their keys' sums are dealt to as many lanes as there are."""
    for branches in ([(0, 8)], [(3, 31)], [(0, 64)], [(0, 16), (9, 40)], [(0, 10), (0, 3), (20, 25)]):
        pool = make(BF16, pages=pages_for(300, branches, 16), kv=kv, page=16, d=d, seqs=len(branches) + 1)
        _, seqs = grow(pool, 300, 7, branches)
        batch, new = Batch(pool), [n for _, n in branches]
        for mask in ((1, 0, 0), (8, 50, 3)):
            batch.set_chunk(seqs, new, *mask)
            check(pool, batch, seqs, new, mask)


@pytest.mark.parametrize("n,d", [(65, 128), (70, 64), (129, 64), (300, 128), (700, 64)])
def test_many_single_tokens(n, d):
    """Sequences of one row over a history that they share, each with tokens of its own."""
    branches = [(i % 23, 1) for i in range(n)]
    pool = make(BF16, pages=pages_for(500, branches, 16), kv=2, page=16, d=d, seqs=n + 1)
    _, seqs = grow(pool, 500, 3, branches)
    batch = Batch(pool)
    for mask in ((1, 0, 0), (1, 64, 4)):
        batch.set_chunk(seqs, [1] * n, *mask)
        check(pool, batch, seqs, [1] * n, mask)


@pytest.mark.parametrize("dtype,kv,d,n", [(BF16, 2, 128, 9), (BF16, 1, 64, 40), (F32, 2, 64, 5), (BF16, 2, 64, 300)])
@pytest.mark.parametrize("what,bad", [("key", math.nan), ("value", math.nan), ("value", math.inf)])
def test_numbers_that_are_not_finite_in_a_shared_history(what, bad, dtype, kv, d, n):
    """Single tokens over one history: bad numbers among its first tokens, between them and the windows, where some windows begin
    and others do not, and where all of them see."""
    branches = [(i % 30, 1) for i in range(n)]
    pool = make(dtype, pages=pages_for(2000, branches, 16), kv=kv, page=16, d=d, seqs=n + 1)
    parent, seqs = grow(pool, 2000, 5, branches)
    g = torch.Generator().manual_seed(6)
    q = torch.randn(n, kv, d, generator=g).to(dtype).cuda()
    batch, tokens, (window, sinks) = Batch(pool), 1995, (700, 40)
    edge = tokens + 20 - window  # in the windows of branches of fewer than 20 tokens
    history = torch.randn(2, tokens, kv, d, generator=g)
    head, dim = kv - 1, d // 3
    for at in ([10], [200], [edge], [tokens - 100], [39, 40, 800, edge, tokens - 3]):
        pair = history.clone()
        pair["kv".index(what[0]), at, head, dim] = bad
        write(pool, parent, *pair)
        for i, s in enumerate(seqs):
            own = torch.randn(2, branches[i][0] + 1, kv, d, generator=g)
            write(pool, s, *torch.cat((pair, own), 1))
        batch.set_chunk(seqs, [1] * n, 1, window, sinks)
        out, lse = torch.empty_like(q), torch.empty(n, kv, device="cuda")
        w = torch.zeros(n, tokens + 40, device="cuda")
        batch.chunk_attention(0, q, out, lse=lse)
        batch.chunk_weights(0, q, lse, w, decay=0.0)
        for i, s in enumerate(seqs):
            k, v = (ref.gather(b, 0, pool.pages(s)) for b in (pool.keys, pool.values))
            see = chunk.sees(len(k), 1, 1, window, sinks)
            hit = bool(see[0, at].any())
            k0, v0 = (torch.where(torch.isfinite(x), x, torch.zeros_like(x)) for x in (k, v))
            args = q[i:i + 1].double().cpu()
            want, tol, want_lse, lse_tol = chunk.attention(args, k0, v0, d ** -0.5, see, dtype, p_eps(dtype))
            got, got_lse = out[i:i + 1].double().cpu(), lse[i:i + 1].double().cpu()
            fine, sums_fine = torch.ones(want.shape, dtype=torch.bool), torch.ones(want_lse.shape, dtype=torch.bool)
            if hit and what == "key":
                fine[0, head], sums_fine[0, head] = False, False
            elif hit:
                fine[0, head, dim] = False
                assert not torch.isfinite(got[0, head, dim])
            assert ((got - want).abs() <= tol)[fine].all() and ((got_lse - want_lse).abs() <= lse_tol)[sums_fine].all()
            if not hit or what == "value":
                total, tol = chunk.weights(args, k0, d ** -0.5, see, got_lse)
                assert ((w[i, :len(k)].double().cpu() - total).abs() <= tol + 1e-30).all()


# ---------------------------------------------------------------- memory

@pytest.mark.parametrize("dtype,rows", [(BF16, (7, 9)), (BF16, (70, 90)), (F32, (7, 90))])
def test_strided_rows_and_untouched_surroundings(dtype, rows):
    pool = make(dtype, pages=80, kv=2, heads=4, page=16, d=64)
    _, seqs = grow(pool, 50, 0, [(0, rows[0]), (3, rows[1])])
    batch, n = Batch(pool), sum(rows)
    batch.set_chunk(seqs, rows, 1, 60, 2)
    q = torch.randn(n + 2, 704).to(dtype).cuda()[1:n + 1, 8:264]
    frame = torch.full((n + 4, 400), 5.0, dtype=dtype, device="cuda")
    dense, lse, again = (torch.empty(n, 256, dtype=dtype, device="cuda"), *torch.empty(2, n, 4, device="cuda"))
    batch.chunk_attention(0, q, frame[2:n + 2, 16:272], lse=lse)
    batch.chunk_attention(0, q.contiguous(), dense)
    assert torch.equal(frame[2:n + 2, 16:272], dense)
    batch.chunk_attention(0, q.contiguous(), dense, lse=again)
    assert torch.equal(lse, again)
    frame[2:n + 2, 16:272] = 5.0
    assert (frame == 5.0).all()
    most = max(map(pool.tokens, seqs))
    table = torch.full((4, most + 9), 5.0, device="cuda")
    part = torch.zeros(2, most, device="cuda")
    batch.chunk_weights(0, q, lse, table[1:3, 4:4 + most], decay=0.0)
    batch.chunk_weights(0, q.contiguous(), lse, part, decay=0.0)
    for i, s in enumerate(seqs):
        t = pool.tokens(s)
        assert torch.equal(table[1 + i, 4:4 + t], part[i, :t]) and part[i, :t].sum() > 0
        table[1 + i, 4:4 + t] = 5.0
    assert (table == 5.0).all()
    # an eviction: its rows alone too
    table[1:3, 4:4 + most] = torch.rand(2, most)
    kept = torch.full((4, 60), -7, dtype=torch.int32, device="cuda")
    batch.evict(seqs, [30, 40], table[1:3, 4:4 + most], kept[1:3, 10:50], sinks=2, recent=3)
    assert (table[[0, 3]] == 5.0).all() and (table[:, :4] == 5.0).all() and (table[:, 4 + most:] == 5.0).all()
    assert (kept[[0, 3]] == -7).all() and (kept[:, :10] == -7).all() and (kept[:, 50:] == -7).all()
    assert (kept[1, 40:50] == -7).all() and (kept[1, 10:40] >= 0).all() and (kept[2, 10:50] >= 0).all()


def test_offsets_past_32_bits():
    """Pages whose elements lie past 2^32, rows of queries and outputs and of weights whose bytes do."""
    kv, page, d = 8, 256, 128
    n_pages = (1 << 32) // (kv * page * d) + 40  # 2^32 elements, 8 GiB, and a little
    k = torch.zeros(1, n_pages, kv, page, d, dtype=BF16, device="cuda")
    v = torch.zeros_like(k)
    pool = Pool(k, v, q_heads=kv, max_seqs=6, stream=stream())
    low = pool.new()
    pool.extend([low], [(n_pages - 40) * page])  # holds every low page
    parent, seqs = grow(pool, 1000, 3, [(30, 5), (0, 300)])
    assert min(pool.pages(parent)[2]) >= n_pages - 40
    g = torch.Generator(device="cuda").manual_seed(0)
    for buf in (k, v):
        buf[0, n_pages - 40:] = torch.randn(40, kv, page, d, device="cuda", generator=g).to(BF16)
    batch = Batch(pool)
    for mask in ((1, 0, 0), (7, 300, 4)):
        batch.set_chunk(seqs, [5, 300], *mask)
        check(pool, batch, seqs, [5, 300], mask, only=[0, 7])
        batch.set_chunk(seqs, [5, 0], *mask)  # few rows
        check(pool, batch, seqs, [5, 0], mask, only=[0, 7])
    # rows 16 MiB apart, weights 4 GiB
    batch.set_chunk(seqs, [5, 300], 1)
    far = torch.empty(306 << 23, dtype=BF16, device="cuda").view(306, 1 << 23)
    q = torch.randn(305, kv * d, device="cuda", generator=g).to(BF16)
    out, lse, lse2 = torch.empty_like(q), *torch.empty(2, 305, kv, device="cuda")
    far[:305, :kv * d] = q
    batch.chunk_attention(0, q, out, lse=lse)
    batch.chunk_attention(0, far[:305, :kv * d], far[:305, kv * d:2 * kv * d], lse=lse2)
    assert torch.equal(far[:305, kv * d:2 * kv * d], out) and torch.equal(lse, lse2)
    w, wide = torch.zeros(2, 1400, device="cuda"), torch.zeros((1 << 30) + 2000, device="cuda").as_strided((2, 1400), (1 << 30, 1))
    batch.chunk_weights(0, q, lse, w, decay=0.0)
    batch.chunk_weights(0, far[:305, :kv * d], lse, wide, decay=0.0)
    assert torch.equal(w, wide) and w.sum() > 0
    del far
    # evictions of far pages, into far pages and low ones; and of a sequence of more than 2^32 elements
    evict_check(pool, batch, seqs, [500, 700], 4, 100, wide)
    keep = 3000
    weights = torch.rand(1, pool.tokens(low), device="cuda", generator=g)
    best = weights[0, :-10].topk(keep - 10).indices.sort().values
    k[0, :n_pages - 40, :, :, 0] = torch.randn(n_pages - 40, kv, page, device="cuda", generator=g).to(BF16)
    at = torch.cat((best, torch.arange(pool.tokens(low) - 10, pool.tokens(low), device="cuda")))
    first, _, pages = pool.pages(low)
    table = torch.from_numpy(pages.copy()).cuda().long()
    want = k[0][table[at // page], :, at % page].clone()
    kept = torch.empty(1, keep, dtype=torch.int32, device="cuda")
    batch.evict([low], [keep], weights, kept, recent=10)
    assert torch.equal(kept[0].long(), at)
    table = torch.from_numpy(pool.pages(low)[2].copy()).cuda().long()
    at = torch.arange(keep, device="cuda")
    assert torch.equal(k[0][table[at // page], :, at % page], want)


@pytest.mark.parametrize("dtype,blocks,kv,page,n", [(BF16, 3, 2, 16, 100), (F32, 2, 1, 64, 20), (BF16, 1, 12, 256, 5)])
def test_many_evictions_at_once(dtype, blocks, kv, page, n):
    """Sequences that share pages with each other and are all listed: none reads what another has already written."""
    g = torch.Generator().manual_seed(4)
    branches = [(int(torch.randint(0, 150, (1,), generator=g)), 1) for _ in range(n)]
    pool = make(dtype, blocks=blocks, pages=pages_for(700, branches, page) + (n + 1) * (-(-851 // page)), kv=kv, page=page, d=64, seqs=n + 1)
    parent, seqs = grow(pool, 700, 11, branches)
    w = torch.rand(n + 1, 900, generator=g).cuda()
    keep = [int(x) for x in torch.randint(40, 880, (n + 1,), generator=g)]
    evict_check(pool, Batch(pool), [parent] + seqs, keep, 20, 15, w)


@pytest.mark.parametrize("dtype,d,kv,n", [(BF16, 128, 6, 90), (F32, 128, 6, 90), (F32, 64, 8, 65), (BF16, 64, 6, 86), (F32, 32, 3, 180),
                                          (BF16, 128, 12, 9), (F32, 128, 12, 9), (BF16, 128, 1, 3), (F32, 128, 1, 3)])
def test_evictions_of_rows_in_one_piece_and_in_several(dtype, d, kv, n):
    """As many workgroups as rows move in whole, in parts of 128 bytes and of 64."""
    g = torch.Generator().manual_seed(8)
    branches = [(i % 90, 30) for i in range(n)]
    pool = make(dtype, pages=n * 16 + 8, kv=kv, page=16, d=d, seqs=n + 1)
    _, seqs = grow(pool, 80, 3, branches)
    keep = [int(x) for x in torch.randint(10, 150, (n,), generator=g)]
    evict_check(pool, Batch(pool), seqs, keep, 5, 4, torch.rand(n, 210, generator=g).cuda())


@pytest.mark.parametrize("pages", [1, 2, 63, 64, 65, 415, 416, 417, 900])
@pytest.mark.parametrize("shared", [False, True])
def test_evictions_of_tables_of_every_size(shared, pages):
    """One sequence's tables: of which so many fit into a kernel's arguments."""
    pool = make(BF16, pages=2 * pages + 2, kv=1, page=16, d=64, seqs=3)
    batch, s, g = Batch(pool), pool.new(), torch.Generator().manual_seed(pages)
    pool.extend([s], [16 * pages])
    if shared:
        other, = pool.fork(s, 1)
        before = ref.gather(pool.keys, 0, pool.pages(other))
    evict_check(pool, batch, [s], [16 * pages - 3], 2, 5, torch.rand(1, 16 * pages, generator=g).cuda())
    if shared:
        assert torch.equal(ref.gather(pool.keys, 0, pool.pages(other)), before)


@pytest.mark.parametrize("n", [1000, 1024, 1025, 5000, 24576, 24577, 60000])
@pytest.mark.parametrize("sinks,recent", [(0, 0), (7, 300)])
def test_evictions_among_few_different_weights(sinks, recent, n):
    """Ties that begin and end in other waves' tokens, of every value that is none like the others."""
    pool = make(BF16, pages=-(-(n + 3) // 64) + 1, kv=1, page=64, d=64, seqs=2)
    batch, s, g = Batch(pool), pool.new(), torch.Generator().manual_seed(n)
    pool.extend([s], [n + 3])
    pool.trim(s, front=3)
    values = torch.tensor([math.nan, 0.0, -0.0, 0.25, 1.0, math.inf, -math.inf, 1e-40, -2.0])
    for keep in (n - 1, n * 5 // 7, n // 2, n // 9 + 310):
        if keep >= pool.tokens(s):
            continue
        w = values[torch.randint(0, len(values), (1, pool.tokens(s)), generator=g)]
        evict_check(pool, batch, [s], [keep], sinks, recent, w.cuda())


# ---------------------------------------------------------------- streams and graphs

def test_graphs_of_two_batches_follow_their_inputs():
    """Attention and weights of each batch in a graph of its own, replayed with new inputs, eager work of both between; the
    stream is not the current one when they run eagerly."""
    st = torch.cuda.Stream()
    made = make(BF16, pages=400, kv=4, page=16, d=128, seqs=20)
    pool = Pool(made.keys, made.values, q_heads=4, max_seqs=20, stream=st.cuda_stream)
    _, seqs = grow(pool, 1500, 0, [(i, 40) for i in range(8)])
    torch.cuda.synchronize()
    graphs = []
    for part, new, mask in ((seqs[:4], [1] * 4, (1, 900, 4)), (seqs[4:], [30, 40, 1, 0], (1, 0, 0)), (seqs[2:5], [40] * 3, (8, 200, 0))):
        with torch.cuda.stream(st):
            b, n = Batch(pool), sum(new)
            b.set_chunk(part, new, *mask)
            q, out = torch.randn(n, 4, 128, device="cuda").to(BF16), torch.zeros(n, 4, 128, dtype=BF16, device="cuda")
            lse, w = torch.zeros(n, 4, device="cuda"), torch.zeros(len(part), 1600, device="cuda")

            def call(b=b, q=q, out=out, lse=lse, w=w):
                b.chunk_attention(0, q, out, lse=lse)
                b.chunk_weights(0, q, lse, w, decay=0.5)

            call()
            st.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=st):
                call()
            graphs.append((q, out, lse, w, call, g))
    for turn in range(4):
        for q, out, lse, w, call, g in graphs:
            with torch.cuda.stream(st):
                q.copy_(torch.randn(q.shape, device="cuda"))
                before = w.clone()
                g.replay()
                st.synchronize()
                got = [x.clone() for x in (out, lse, w)]
                out.zero_(), lse.zero_(), w.copy_(before)
            st.synchronize()
            call()  # on the pool's stream, whatever the current one is
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, (out, lse, w))) and not torch.equal(before, w)


def test_rows_set_anew_under_work_in_flight():
    """A batch set again and evictions while the work before them is still running; each result against its own once more."""
    pool = make(BF16, pages=2400, kv=8, page=16, d=128, seqs=40)
    _, seqs = grow(pool, 20000, 0, [(i % 4, 2) for i in range(32)])
    batch, single = Batch(pool), Batch(pool)
    q = torch.randn(64, 8, 128, device="cuda").to(BF16)
    done = []
    for n in (1, 2, 5, 12, 30, 32, 3):
        batch.set_chunk(seqs[:n], [2] * n, 1, 9000, 3)
        out, lse, w = torch.empty(2 * n, 8, 128, dtype=BF16, device="cuda"), torch.empty(2 * n, 8, device="cuda"), \
            torch.zeros(n, 20006, device="cuda")
        for _ in range(2):
            batch.chunk_attention(0, q[:2 * n], out, lse=lse)
            batch.chunk_weights(0, q[:2 * n], lse, w, decay=0.0)
        done.append((n, out, lse, w))
    for n, *got in done:
        single.set_chunk(seqs[:n], [2] * n, 1, 9000, 3)
        torch.cuda.synchronize()
        again = [torch.zeros_like(x) for x in got]
        single.chunk_attention(0, q[:2 * n], again[0], lse=again[1])
        single.chunk_weights(0, q[:2 * n], again[1], again[2], decay=0.0)
        assert all(torch.equal(a, b) for a, b in zip(got, again))
    # evictions one after the other, without a wait
    s = seqs[0]
    tokens = ref.gather(pool.keys, 0, pool.pages(s))
    w = torch.rand(1, 20002, device="cuda")
    at, old = list(range(20002)), w[0].tolist()
    torch.cuda.synchronize()
    for keep in (2000, 1500, 700, 20):
        batch.evict([s], [keep], w, sinks=2, recent=5)
        left = chunk.kept([old[x] for x in at], keep, 2, 5)
        at = [at[x] for x in left]
    assert torch.equal(ref.gather(pool.keys, 0, pool.pages(s)), tokens[at])
    assert w[0, :20].tolist() == [old[x] for x in at] and (w[0, 20:] == 0).all()


# ---------------------------------------------------------------- a run of them together

@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_bounded_cache_over_many_chunks(dtype):
    """Branches that grow chunk by chunk: keys and values written, attention under a mask, its weights summed over blocks, the
    light tokens evicted, and now and then a fork.  Beside it a list of (key, value, weight) per branch."""
    blocks, kv, group, page, d, bound, sinks, recent = 2, 2, 2, 16, 64, 150, 4, 20
    heads = kv * group
    pool = make(dtype, blocks=blocks, pages=300, kv=kv, heads=heads, page=page, d=d, seqs=8, fill="nan")
    width = (heads + 2 * kv) * d
    g = torch.Generator().manual_seed(3)
    one = torch.ones(d, device="cuda")
    batch, live = Batch(pool), [pool.new(), pool.new()]
    store = torch.zeros(8, bound + 100, device="cuda")  # a row of weights per sequence number
    total = {s: [] for s in live}  # the weight of every token, in 64 bits
    for turn in range(9):
        new = [int(x) for x in torch.randint(1, 70 if turn % 3 else 3, (len(live),), generator=g)]
        if turn == 5:
            new[0] = 0
        mask = [(1, 0, 0), (8, 60, 4), (0, 0, 0)][turn % 3]
        pool.extend(live, new)
        batch.set_chunk(live, new, *mask)
        rows = sum(new)
        w = torch.zeros(len(live), bound + 100, device="cuda")
        for i, (s, n) in enumerate(zip(live, new)):
            old = pool.tokens(s) - n
            w[i, :old] = store[s, :old]
            total[s] += [0.0] * n
        spread = [torch.zeros(len(total[s])) for s in live]
        for b in range(blocks):
            qkv = torch.randn(rows, width, generator=g).to(dtype).cuda()
            pos = torch.arange(rows).int()[:, None].cuda()
            q, out = (torch.empty(rows, heads, d, dtype=dtype, device="cuda") for _ in range(2))
            lse = torch.empty(rows, heads, device="cuda")
            batch.qk_norm_rope(b, qkv, one, one, pos, 100.0, q)
            batch.chunk_attention(b, q, out, lse=lse)
            batch.chunk_weights(b, q, lse, w, decay=0.75 if b == 0 else 1.0)
            row = 0
            for i, (s, n) in enumerate(zip(live, new)):
                if not n:
                    continue  # its weights stay as they are
                part, see = slice(row, row + n), chunk.sees(pool.tokens(s), n, *mask)
                k, v = ref.gather(pool.keys, b, pool.pages(s)), ref.gather(pool.values, b, pool.pages(s))
                qs = q[part].double().cpu()
                want, tol, want_lse, lse_tol = chunk.attention(qs, k, v, d ** -0.5, see, dtype, p_eps(dtype))
                assert ((out[part].double().cpu() - want).abs() <= tol).all()
                assert ((lse[part].double().cpu() - want_lse).abs() <= lse_tol).all()
                sums, tol = chunk.weights(qs, k, d ** -0.5, see, lse[part].double().cpu())
                f = 0.75 if b == 0 else 1.0
                total[s] = [x * f + y for x, y in zip(total[s], sums.tolist())]
                spread[i] = spread[i] * f + tol + 2.0 ** -22 * torch.tensor(total[s])
                row += n
        for i, s in enumerate(live):
            t = pool.tokens(s)
            got = w[i, :t].double().cpu()
            assert ((got - torch.tensor(total[s]).double()).abs() <= spread[i] + 1e-30).all()
            total[s] = got.tolist()  # (its own from here on: what an eviction orders)
        evict_check(pool, batch, live, [bound] * len(live), sinks, recent, w)
        for i, s in enumerate(live):
            total[s] = [total[s][x] for x in chunk.kept(total[s], bound, sinks, recent)]
            store[s] = w[i]
            assert pool.tokens(s) == len(total[s]) <= bound
        if turn in (2, 5):
            kid, = pool.fork(live[-1], 1)
            store[kid], total[kid] = store[live[-1]], list(total[live[-1]])
            live.append(kid)
        if turn == 6:
            pool.free([live.pop(0)])
            pool.compact()
    pool.free(live)
    assert pool.info()["live_pages"] == 0


def test_a_rollouts_window_is_evicted_and_extended():
    """The window of a rollout's own cache, imported, thinned out and attended to by a chunk of branches."""
    import synth
    from paper_2604_20289_amd.xcache import XCache
    w = synth.workload(0)
    w = synth.with_model(w, rope=1, kv_window=2, n_heads=2, head_dim=64, hidden=128, mlp_hidden=128, dtype="bf16", n_blocks=2)
    m = w.model
    h = XCache(m, w.gate, synth.make_weights(m), torch.cuda.current_stream().cuda_stream)
    (e,), (a,) = synth.latent_stream(m, w.stream, 0, 1), synth.action_stream(m, w.stream, 0, 1)
    y = torch.empty(m.tokens, m.hidden, device="cuda")
    h.forward_chunk(0, synth.timesteps(m)[0], a, torch.from_numpy(e).cuda(), y)
    h.kv_update(0.0, a, y)
    pool = make(BF16, blocks=2, pages=4 * (-(-m.tokens // 16)) + 20, kv=2, page=16, d=64)
    batch, s = Batch(pool), pool.new()
    pool.import_window(s, h)
    kids = pool.fork(s, 3)
    weights = torch.rand(3, m.tokens, device="cuda")
    evict_check(pool, batch, kids, [m.tokens // 2, m.tokens, m.tokens // 3], 3, m.tokens // 4, weights)
    pool.extend(kids, [9, 1, 40])
    for b in range(2):
        batch.set_chunk(kids, [9, 1, 40], 4)
        check(pool, batch, kids, [9, 1, 40], (4, 0, 0), block=b)
    h.close()


# ---------------------------------------------------------------- refusals

def test_changed_tables_and_other_attentions_are_refused():
    pool = make(BF16, pages=60, kv=2, page=16, d=64)
    _, (a, b) = grow(pool, 100, 0, [(0, 3), (2, 5)])
    batch = Batch(pool)
    q, out = torch.randn(8, 2, 64).to(BF16).cuda(), torch.zeros(8, 2, 64, dtype=BF16, device="cuda")
    lse, w = torch.zeros(8, 2, device="cuda"), torch.ones(2, 120, device="cuda")

    def refused(call, status):
        with pytest.raises(XCacheError) as e:
            call()
        assert e.value.status == status

    attention, weights = (lambda: batch.chunk_attention(0, q, out, lse=lse)), (lambda: batch.chunk_weights(0, q, lse, w))
    batch.set([a, b], [3, 5])
    refused(attention, xcache.XC_ERR_STATE)
    batch.set_chunk([a, b], [3, 5])
    refused(lambda: batch.attention(0, q, out), xcache.XC_ERR_STATE)
    refused(lambda: batch.set_chunk([a, b], [3, 5], group=-1), xcache.XC_ERR_INVALID_ARG)
    refused(lambda: batch.chunk_weights(0, q, lse, w, decay=math.nan), xcache.XC_ERR_INVALID_ARG)
    refused(lambda: batch.evict([a], [5], torch.ones(1, 120, device="cuda"), sinks=3, recent=3), xcache.XC_ERR_INVALID_ARG)
    assert (out == 0).all() and (lse == 0).all() and (w == 1).all()
    attention(), weights()
    batch.evict([b], [50], w[1:])
    refused(attention, xcache.XC_ERR_STATE)
    refused(weights, xcache.XC_ERR_STATE)
    st = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        held = Pool(pool.keys, pool.values, q_heads=2, max_seqs=4, stream=st.cuda_stream)
        s = held.new()
        held.extend([s], [40])
        own, one = Batch(held), torch.ones(1, 40, device="cuda")
        own.set_chunk([s], [8])
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            refused(lambda: own.set_chunk([s], [1]), xcache.XC_ERR_STATE)
            refused(lambda: own.evict([s], [5], one), xcache.XC_ERR_STATE)
            own.chunk_attention(0, q, out, lse=lse)
        assert held.tokens(s) == 40
        for turn in range(3):
            q.copy_(torch.randn(8, 2, 64))
            graph.replay()
            st.synchronize()
            got = out.clone()
            own.chunk_attention(0, q, out, lse=lse)
            st.synchronize()
            assert torch.equal(got, out)

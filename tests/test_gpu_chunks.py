"""Chunks under a mask on the GPU: attention with its log-sum-exp, the weights of cached keys and evictions, each against
a plain 64-bit implementation, and a run of them together."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import branch_reference as ref  # noqa: E402
import chunk_reference as chunk  # noqa: E402
from paper_2604_20289_amd import xcache  # noqa: E402
from paper_2604_20289_amd.xcache import Batch, XCacheError  # noqa: E402
from test_gpu_branches import BF16, F32, grow, make, pages_for, write  # noqa: E402


def p_eps(dtype):
    return ref.EPS_OF[BF16] if dtype == BF16 else 2.0 ** -24


def check(pool, batch, seqs, new, mask, block=0, scale=0.0, seed=0, gain=1.5, q=None, only=None):
    """Attention, log-sum-exps and weights of a batch that is set, against 64 bits.  Returns what the kernels gave."""
    c = pool.config
    heads, d, dtype, rows = c.q_heads, c.head_dim, pool.keys.dtype, sum(new)
    if q is None:
        q = (torch.randn(rows, heads, d, generator=torch.Generator().manual_seed(seed)) * gain).to(dtype).cuda()
    out = torch.full((rows, heads, d), 7.0, dtype=dtype, device="cuda")
    lse = torch.full((rows, heads), 7.0, device="cuda")
    batch.chunk_attention(block, q, out, lse=lse, scale=scale)
    most = max(pool.tokens(s) for s in seqs)
    w = torch.full((len(seqs), most + 3), math.nan, device="cuda")
    batch.chunk_weights(block, q, lse, w, decay=0.0, scale=scale)
    first = w.clone()
    batch.chunk_weights(block, q, lse, w, decay=0.5, scale=scale)
    got, got_lse, worst, row = out.double().cpu(), lse.double().cpu(), [0.0, 0.0, 0.0], 0
    pick = list(range(heads)) if only is None else only
    for i, (s, n) in enumerate(zip(seqs, new)):
        tokens = pool.tokens(s)
        assert torch.isnan(w[i, tokens if n else 0:]).all()  # left as it was
        if not n:
            continue
        table = pool.pages(s)
        k, v = ref.gather(pool.keys, block, table), ref.gather(pool.values, block, table)
        part, see = slice(row, row + n), chunk.sees(tokens, n, *mask)
        qs = q[part].double().cpu()
        kv = [h * c.kv_heads // heads for h in pick]
        want, tol, want_lse, lse_tol = chunk.attention(qs[:, pick], k[:, kv], v[:, kv], scale or d ** -0.5, see, dtype,
                                                       p_eps(dtype))
        for j, (a, b, t) in enumerate(((got[part][:, pick], want, tol), (got_lse[part][:, pick], want_lse, lse_tol))):
            assert torch.isfinite(a).all(), (s, n)
            worst[j] = max(worst[j], ((a - b).abs() / t).max().item())
            assert ((a - b).abs() <= t).all(), (i, s, n, tokens, j, worst)
        total, tol = chunk.weights(qs, k, scale or d ** -0.5, see, got_lse[part])
        a, b = first[i, :tokens].double().cpu(), w[i, :tokens].double().cpu()
        worst[2] = max(worst[2], ((a - total).abs() / (tol + 1e-30)).max().item())
        assert ((a - total).abs() <= tol + 1e-30).all(), (i, s, n, tokens, worst)
        assert ((b - (a * 0.5 + total)).abs() <= tol + 2.0 ** -23 * (a + total) + 1e-30).all()
        assert (a[~see.any(0)] == 0).all()
        row += n
    return out, lse, w, worst


MASKS = [(0, 0, 0), (1, 0, 0), (7, 0, 0), (1, 100, 0), (16, 130, 5), (1, 1, 0), (3, 2, 1), (64, 1000, 70)]

CASES = [
    # dtype, key heads, group, d, page, history, dropped, (own earlier, new) per branch
    (BF16, 1, 1, 128, 16, 0, 0, [(0, 1)]),
    (BF16, 2, 1, 64, 16, 1, 0, [(0, 1), (0, 1)]),
    (BF16, 2, 1, 128, 64, 63, 0, [(0, 1), (1, 1)]),
    (BF16, 2, 1, 64, 64, 64, 0, [(0, 2), (0, 65)]),
    (BF16, 3, 1, 128, 16, 100, 15, [(3, 2), (0, 5), (40, 1)]),
    (BF16, 1, 5, 64, 32, 333, 17, [(0, 60), (9, 1), (0, 0), (100, 31)]),
    (BF16, 2, 4, 128, 256, 700, 255, [(0, 257), (300, 3)]),
    (BF16, 2, 1, 128, 128, 0, 0, [(0, 600), (0, 300)]),
    (BF16, 4, 1, 64, 64, 900, 9, [(i * 7, 1) for i in range(9)]),
    (BF16, 1, 64, 64, 16, 130, 3, [(0, 4), (1, 5)]),
    (BF16, 1, 1, 128, 16, 3000, 7, [(0, 400)]),
    (F32, 1, 1, 32, 16, 0, 0, [(0, 1)]),
    (F32, 4, 1, 32, 16, 64, 0, [(0, 64)] * 3),
    (F32, 1, 3, 64, 32, 100, 15, [(3, 2), (0, 50), (40, 1)]),
    (F32, 2, 2, 128, 256, 700, 255, [(0, 130), (300, 3)]),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{str(c[0])[6:]}-{c[1]}x{c[2]}-d{c[3]}-p{c[4]}-h{c[5]}-{len(c[7])}")
def test_chunks_under_every_mask(case):
    """NaN everywhere outside the sequences' tokens: what is not theirs is not read."""
    dtype, kv, group, d, page, prefix, drop, branches = case
    pool = make(dtype, blocks=2, pages=pages_for(prefix, branches, page), kv=kv, heads=kv * group, page=page, d=d,
                seqs=len(branches) + 1, fill="nan")
    parent, seqs = grow(pool, prefix, drop, branches)
    g = torch.Generator().manual_seed(1)
    history = torch.randn(2, prefix - drop, kv, d, generator=g)
    for s, (a, b) in zip(seqs, branches):
        own = torch.randn(2, a + b, kv, d, generator=g)
        write(pool, s, *(torch.cat((history, own), 1).to(dtype)), block=1)
    batch, new = Batch(pool), [b for _, b in branches]
    for mask in MASKS:
        batch.set_chunk(seqs, new, *mask)
        out, lse, w, worst = check(pool, batch, seqs, new, mask, block=1)
        again = check(pool, batch, seqs, new, mask, block=1)
        assert all(torch.equal(x.nan_to_num(), y.nan_to_num()) for x, y in zip((out, lse, w), again))  # the same bits
        print(f"[chunks] {case} {mask} worst error / bound {worst}", flush=True)


# ---------------------------------------------------------------- eviction

def evict_check(pool, batch, seqs, keep, sinks, recent, w, block_seed=0):
    """An eviction against the lists of tokens that it should leave."""
    before = {s: [ref.gather(b, i, pool.pages(s)) for b in (pool.keys, pool.values) for i in range(pool.config.n_blocks)]
              for s in seqs}
    tokens = [pool.tokens(s) for s in seqs]
    old = w.cpu().clone()
    kept = torch.full((len(seqs), max(tokens) + 2), -7, dtype=torch.int32, device="cuda")
    batch.evict(seqs, keep, w, kept, sinks=sinks, recent=recent)
    for i, (s, k, n) in enumerate(zip(seqs, keep, tokens)):
        want = chunk.kept(old[i, :n].tolist(), k, sinks, recent)
        assert kept[i, :len(want)].tolist() == want
        assert (kept[i, len(want):] == -7).all()
        assert pool.tokens(s) == len(want)
        after = [ref.gather(b, j, pool.pages(s)) for b in (pool.keys, pool.values) for j in range(pool.config.n_blocks)]
        for a, b in zip(after, before[s]):
            assert torch.equal(a, b[want])
        expect = old[i].clone()
        if k < n:
            expect[:n] = 0
            expect[:len(want)] = old[i][want]
        assert torch.equal(w[i].cpu().nan_to_num(nan=-1.0), expect.nan_to_num(nan=-1.0))
    return kept


@pytest.mark.parametrize("dtype,kv,d,page", [(BF16, 3, 128, 64), (BF16, 2, 64, 16), (F32, 1, 32, 16), (F32, 2, 128, 256)])
def test_evictions_keep_the_heaviest(dtype, kv, d, page):
    """One sequence after the other shrinks, grows and shrinks again, its first token inside a page; ties, NaN, infinities and
    zeros of both signs among the weights."""
    pool = make(dtype, blocks=2, pages=400 * 16 // page + 8, kv=kv, page=page, d=d, seqs=4)
    batch, s = Batch(pool), pool.new()
    pool.extend([s], [1700])
    pool.trim(s, front=5)
    g = torch.Generator().manual_seed(2)
    for keep, sinks, recent, grown in ((1500, 4, 300, 900), (1499, 0, 0, 10), (800, 130, 0, 3000), (64, 1, 63, 1),
                                       (65, 0, 65, 700), (33, 33, 0, 200), (100, 0, 7, 5), (1, 0, 0, 40), (0, 0, 0, 60),
                                       (60, 3, 3, 9)):
        n = pool.tokens(s)
        w = torch.randn(1, n + 4, generator=g).exp()
        w[0, torch.rand(n + 4, generator=g) < 0.3] = 0.25  # alike
        for value in (math.nan, math.inf, -math.inf, -0.0, 0.0, -1.5):
            w[0, torch.randint(0, n, (max(1, n // 50),), generator=g)] = value
        evict_check(pool, batch, [s], [keep], sinks, recent, w.cuda())
        pool.extend([s], [grown])
    info = pool.info()
    first, tokens, pages = pool.pages(s)
    assert info["live_pages"] == len(pages) == -(-(first + tokens) // page)


def test_evictions_of_branches_leave_the_others():
    """Pages that others hold are replaced, those of first tokens alone stay shared; a fork that is not listed, and one that
    keeps everything, are as they were."""
    page = 16
    pool = make(BF16, blocks=3, pages=400, kv=2, page=page, d=64, seqs=8)
    parent, seqs = grow(pool, 203, 7, [(40, 10), (3, 60), (0, 1), (100, 0)])
    batch = Batch(pool)
    untouched = [ref.gather(b, i, pool.pages(x)) for x in (parent, seqs[3]) for b in (pool.keys, pool.values) for i in range(3)]
    w = torch.rand(4, 300, device="cuda")
    live = pool.info()["live_pages"]
    evict_check(pool, batch, seqs, [100, 77, 60, 1000], 40, 20, w)
    shared = (7 + 40) // page  # pages of first tokens
    tables = [pool.pages(x)[2].tolist() for x in [parent] + seqs]
    for t in tables[1:4]:
        assert t[:shared] == tables[0][:shared] and not set(t[shared:]) & set(tables[0])
    assert untouched and all(torch.equal(a, b) for a, b in zip(
        untouched, [ref.gather(b, i, pool.pages(x)) for x in (parent, seqs[3]) for b in (pool.keys, pool.values) for i in range(3)]))
    assert pool.info()["live_pages"] == len(set(sum(tables, []))) <= live + 20


def test_an_eviction_that_finds_no_page_changes_nothing():
    pool = make(BF16, blocks=1, pages=8, kv=1, page=16, d=64, seqs=4)
    a = pool.new()
    pool.extend([a], [100])
    b = pool.fork(a, 1)[0]
    batch, w = Batch(pool), torch.rand(1, 100, device="cuda")
    old = w.clone()
    tables = [pool.pages(x)[2].tolist() for x in (a, b)]
    with pytest.raises(XCacheError) as e:
        batch.evict([b], [50], w)
    assert e.value.status == xcache.XC_ERR_OOM
    assert tables == [pool.pages(x)[2].tolist() for x in (a, b)] and torch.equal(w, old) and pool.tokens(b) == 100
    evict_check(pool, batch, [b], [16], 0, 0, w)  # one page is free


@pytest.mark.parametrize("n", [1, 63, 64, 8191, 8192, 8193, 70001])
def test_evictions_of_every_length(n):
    pool = make(BF16, blocks=1, pages=-(-n // 256) + 1, kv=1, page=256, d=64, seqs=2)
    s = pool.new()
    pool.extend([s], [n])
    w = torch.rand(1, n, generator=torch.Generator().manual_seed(n)).cuda()
    evict_check(pool, Batch(pool), [s], [n // 2], 0, n // 8, w)


# ---------------------------------------------------------------- numbers that are not finite

# type, key heads, head dim, rows: with 256 heads the kernel of 256-row workgroups, with one or two those of 64 and 32
KERNELS = [(BF16, 256, 64, 300), (BF16, 256, 128, 300), (BF16, 1, 64, 21), (BF16, 2, 128, 50), (F32, 1, 32, 21), (F32, 2, 64, 90),
           (F32, 1, 128, 40)]


@pytest.mark.parametrize("dtype,kv,d,rows", KERNELS)
@pytest.mark.parametrize("what,bad", [("key", math.nan), ("key", math.inf), ("value", math.nan), ("value", -math.inf)])
@pytest.mark.parametrize("mask", [(1, 0, 0), (4, 40, 3), (1, 1, 0)])
def test_what_a_row_does_not_see_does_not_reach_it(mask, what, bad, dtype, kv, d, rows):
    """Numbers that are not finite in the middle of the new tokens, in the last one and, where there is a window that hides it, in
    an old one.  A row that sees a value has it in its column alone, and none that does not is touched."""
    before = 70
    tokens = before + rows
    pool = make(dtype, pages=2 * (-(-(tokens + 3) // 16) + 1), kv=kv, page=16, d=d, seqs=3)
    s = pool.new()
    pool.extend([s], [tokens + 3])
    pool.trim(s, front=3)
    g = torch.Generator().manual_seed(11)
    k, v = torch.randn(2, tokens, kv, d, generator=g)
    head, dim, at = kv // 2, d // 3, [20] * bool(mask[1]) + [before + rows // 2, tokens - 1]
    (k if what == "key" else v)[at, head, dim] = bad
    write(pool, s, k, v)
    batch = Batch(pool)
    batch.set_chunk([s], [rows], *mask)
    q = torch.randn(rows, kv, d, generator=g).to(dtype).cuda()
    out, lse = torch.empty_like(q), torch.empty(rows, kv, device="cuda")
    batch.chunk_attention(0, q, out, lse=lse)
    w = torch.zeros(1, tokens, device="cuda")
    batch.chunk_weights(0, q, lse, w, decay=0.0)
    heads = sorted({0, head, kv - 1})
    k, v = (ref.gather(b, 0, pool.pages(s)) for b in (pool.keys, pool.values))
    see = chunk.sees(tokens, rows, *mask)
    hit = see[:, at].any(1)
    assert not hit.all()
    k0, v0 = (torch.where(torch.isfinite(x), x, torch.zeros_like(x)) for x in (k, v))
    want, tol, want_lse, lse_tol = chunk.attention(q[:, heads].double().cpu(), k0[:, heads], v0[:, heads], d ** -0.5, see, dtype,
                                                   p_eps(dtype))
    got, got_lse = out.double().cpu()[:, heads], lse.double().cpu()[:, heads]
    i = heads.index(head)
    fine = torch.ones(want.shape, dtype=torch.bool)
    if what == "key":
        fine[hit, i] = False
    else:
        fine[hit, i, dim] = False
    assert ((got - want).abs() <= tol)[fine].all()
    assert torch.isfinite(out.double().cpu()[:, [h for h in range(kv) if h != head]]).all()
    if what == "value":
        assert not torch.isfinite(got[hit, i, dim]).any()
        assert ((got_lse - want_lse).abs() <= lse_tol).all()
        total, tol = chunk.weights(q.double().cpu(), k, d ** -0.5, see, lse.double().cpu())
        assert ((w[0].double().cpu() - total).abs() <= tol + 1e-30).all()
    else:
        rows_ok = torch.ones(rows, dtype=torch.bool)
        rows_ok[hit] = False
        assert ((got_lse - want_lse).abs() <= lse_tol)[rows_ok].all()
        # tokens that only untouched rows see have finite weights
        only = ~(see & hit[:, None]).any(0) & see.any(0)
        assert torch.isfinite(w[0].cpu()[only]).all()


@pytest.mark.parametrize("dtype,kv,d,rows", KERNELS)
def test_scores_of_any_size_under_a_mask(dtype, kv, d, rows):
    """Scores hundreds of log2 units apart in rising and falling order, the largest of them hidden from most rows, and keys
    whose product with every query overflows to -infinity."""
    before = 60
    tokens = before + rows
    pool = make(dtype, pages=-(-tokens // 16) + 1, kv=kv, page=16, d=d, seqs=2)
    s = pool.new()
    pool.extend([s], [tokens])
    g = torch.Generator().manual_seed(12)
    only = sorted({0, kv // 2, kv - 1})
    batch = Batch(pool)
    for order in ("up", "down"):
        ramp = torch.linspace(-60, 60, tokens)
        ramp = ramp if order == "up" else ramp.flip(0)
        k = ramp[:, None, None].expand(tokens, kv, d) + 0.5 * torch.randn(tokens, kv, d, generator=g)
        write(pool, s, k, torch.randn(tokens, kv, d, generator=g))
        for mask in ((1, 0, 0), (5, 30, 2)):
            batch.set_chunk([s], [rows], *mask)
            q = torch.ones(rows, kv, d).to(dtype).cuda()
            out, lse = torch.empty_like(q), torch.empty(rows, kv, device="cuda")
            batch.chunk_attention(0, q, out, lse=lse, scale=0.3)
            kk, vv = (ref.gather(b, 0, pool.pages(s))[:, only] for b in (pool.keys, pool.values))
            want, tol, want_lse, lse_tol = chunk.attention(q[:, only].double().cpu(), kk, vv, 0.3, chunk.sees(tokens, rows, *mask),
                                                           dtype, p_eps(dtype))
            assert ((out[:, only].double().cpu() - want).abs() <= tol).all()
            assert ((lse[:, only].double().cpu() - want_lse).abs() <= lse_tol).all()

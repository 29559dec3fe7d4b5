"""Branching rollouts on the GPU: norms with rotation into pages, attention
over shared histories, page copies, each against a plain 64-bit
implementation, and a run of them together."""
import ctypes
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import branch_reference as ref  # noqa: E402
from paper_2604_20289_amd import xcache  # noqa: E402
from paper_2604_20289_amd.xcache import Batch, Pool, XCacheError  # noqa: E402

BF16, F32 = torch.bfloat16, torch.float32


def stream():
    return torch.cuda.current_stream().cuda_stream


def make(dtype=BF16, blocks=1, pages=64, kv=2, heads=None, page=16, d=64, seqs=16, seed=0, fill="normal"):
    """A pool whose buffers hold numbers everywhere, or NaN where no sequence writes."""
    g = torch.Generator().manual_seed(seed)
    shape = (blocks, pages, kv, page, d)
    if fill == "nan":
        k, v = (torch.full(shape, math.nan, dtype=dtype, device="cuda") for _ in range(2))
    else:
        k, v = (torch.randn(shape, generator=g).to(dtype).cuda() for _ in range(2))
    return Pool(k, v, q_heads=heads or kv, max_seqs=seqs, stream=stream())


def write(pool, seq, k, v, block=0):
    """All tokens of a sequence [tokens, kv_heads, d], past the operators."""
    first, tokens, pages = pool.pages(seq)
    at = np.arange(first, first + tokens)
    page = pool.keys.shape[3]
    p, r = (torch.from_numpy(x.astype(np.int64)).cuda() for x in (pages[at // page], at % page))
    pool.keys[block][p, :, r] = k.to(pool.keys)
    pool.values[block][p, :, r] = v.to(pool.keys)


def check_attention(pool, batch, seqs, new, block=0, scale=0.0, seed=0, gain=1.5, q=None, only=None):
    heads, d, dtype = pool.config.q_heads, pool.config.head_dim, pool.keys.dtype
    rows = sum(new)
    g = torch.Generator().manual_seed(seed)
    if q is None:
        q = (torch.randn(rows, heads, d, generator=g) * gain).to(dtype).cuda()
    out = torch.full((rows, heads, d), 7.0, dtype=dtype, device="cuda")
    batch.attention(block, q, out, scale)
    got, row, worst = out.double().cpu(), 0, 0.0
    for s, n in zip(seqs, new):
        if n:
            table = pool.pages(s)
            k, v = ref.gather(pool.keys, block, table), ref.gather(pool.values, block, table)
            pick = list(range(heads)) if only is None else only
            kv = [h * pool.config.kv_heads // heads for h in pick]
            want, size, spread = ref.attention(q[row:row + n, pick].double().cpu(), k[:, kv], v[:, kv], scale or d ** -0.5)
            tol = ref.attention_bound(want, size, spread, d, len(k), dtype, ref.EPS_OF[BF16] if dtype == BF16 else 2.0 ** -24)
            err = (got[row:row + n][:, pick] - want).abs()
            assert torch.isfinite(got[row:row + n]).all(), (s, n)
            worst = max(worst, (err / tol).max().item())
            assert (err <= tol).all(), (s, n, table[1], worst)
        row += n
    return out, worst


# ---------------------------------------------------------------- attention

ATTENTION = [
    # dtype, kv heads, group, d, page, history, dropped, (own earlier, new) per branch
    (BF16, 1, 1, 128, 16, 0, 0, [(0, 1)]),                          # one key
    (BF16, 2, 1, 64, 16, 1, 0, [(0, 1), (0, 1)]),
    (BF16, 2, 1, 128, 64, 63, 0, [(0, 1), (1, 1)]),                 # the last tile full, and one key in the next
    (BF16, 2, 1, 64, 64, 64, 0, [(0, 1), (0, 65)]),
    (BF16, 3, 1, 128, 16, 100, 15, [(3, 2), (0, 5), (40, 1)]),      # first key inside a page
    (BF16, 1, 5, 64, 32, 333, 17, [(0, 60), (9, 1), (0, 0), (100, 31)]),  # five query heads a key head, a branch without rows
    (BF16, 2, 4, 128, 256, 700, 255, [(0, 257), (300, 3)]),
    (BF16, 2, 3, 64, 16, 2000, 1, [(i, 1 + i % 3) for i in range(11)]),
    (BF16, 4, 1, 128, 64, 5000, 0, [(i * 7, 1) for i in range(16)]),
    (BF16, 2, 1, 128, 128, 900, 40, [(0, 300), (0, 300)]),
    (BF16, 1, 64, 64, 16, 130, 3, [(0, 4), (1, 5)]),
    (BF16, 1, 1, 64, 16, 9000, 0, [(0, 1)]),                        # one row, pages beyond one register of table entries
    (BF16, 1, 1, 128, 16, 9000, 7, [(0, 700)]),
    (F32, 1, 1, 32, 16, 0, 0, [(0, 1)]),
    (F32, 2, 1, 32, 16, 31, 0, [(0, 1), (1, 1)]),
    (F32, 4, 1, 32, 16, 64, 0, [(0, 64)] * 3),
    (F32, 1, 3, 64, 32, 100, 15, [(3, 2), (0, 50), (40, 1)]),
    (F32, 2, 2, 128, 256, 700, 255, [(0, 130), (300, 3)]),
    (F32, 2, 1, 128, 16, 3000, 9, [(i, 1) for i in range(7)]),
]


def grow(pool, prefix, drop, branches):
    """A dropped and forked history whose branches' pages lie between each other's."""
    parent = pool.new()
    if prefix:
        pool.extend([parent], [prefix])
    if drop:
        pool.trim(parent, front=drop)
    seqs = pool.fork(parent, len(branches))
    total = [a + b for a, b in branches]
    for turn in range(3):
        pool.extend(seqs, [t * (turn + 1) // 3 - t * turn // 3 for t in total])
    return parent, seqs


def pages_for(prefix, branches, page):
    return 3 + -(-prefix // page) + sum(-(-(a + b) // page) + 2 for a, b in branches)


@pytest.mark.parametrize("case", ATTENTION, ids=lambda c: f"{str(c[0])[6:]}-{c[1]}x{c[2]}-d{c[3]}-p{c[4]}-h{c[5]}-{len(c[7])}")
def test_attention_over_shared_history(case):
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
    batch = Batch(pool)
    new = [b for _, b in branches]
    batch.set(seqs, new)
    out, worst = check_attention(pool, batch, seqs, new, block=1)
    again, _ = check_attention(pool, batch, seqs, new, block=1)
    assert torch.equal(out, again)  # the same bits
    # one branch at a time (nothing shared): the same numbers within the bound
    for i, s in enumerate(seqs):
        if new[i]:
            batch.set([s], [new[i]])
            check_attention(pool, batch, [s], [new[i]], block=1)
    print(f"[branches] {case} worst error / bound {worst:.3f}", flush=True)


@pytest.mark.parametrize("dtype,kv,d", [(BF16, 1, 64), (BF16, 256, 64), (BF16, 256, 128), (F32, 1, 64)])
def test_extreme_scores_and_values(dtype, kv, d):
    """Scores hundreds of log2 units apart in rising, falling and mixed order (the running maximum), values near
    the type's largest, and a scale of the caller's."""
    rows = 40 if kv == 1 else 200
    pool = make(dtype, pages=64, kv=kv, page=16, d=d, seqs=3)
    s = pool.new()
    pool.extend([s], [500])
    g = torch.Generator().manual_seed(3)
    batch = Batch(pool)
    batch.set([s], [rows])
    q = torch.ones(rows, kv, d)
    for order in ("up", "down", "mixed"):
        ramp = torch.linspace(-60, 60, 500)
        ramp = {"up": ramp, "down": ramp.flip(0), "mixed": ramp[torch.randperm(500, generator=g)]}[order]
        k = ramp[:, None, None].expand(500, kv, d) + 0.5 * torch.randn(500, kv, d, generator=g)
        v = torch.randn(500, kv, d, generator=g) * 2.0 ** 110
        write(pool, s, k, v)
        for scale in (0.0, 0.03, 1.0):
            check_attention(pool, batch, [s], [rows], scale=scale, q=q.to(dtype).cuda(), only=sorted({0, kv - 1}))


@pytest.mark.parametrize("d,rows", [(64, 300), (128, 300), (64, 40), (128, 40)])
def test_scores_past_the_range_of_a_float(d, rows):
    """Keys whose product with every query overflows to -infinity, at the start, inside and at the end: weight 0; one run
    of rising scores crosses every limit at which a running maximum moves."""
    for dtype in (BF16, F32):
        pool = make(dtype, pages=64, kv=1, page=16, d=d, seqs=2)
        s = pool.new()
        pool.extend([s], [500])
        g = torch.Generator().manual_seed(4)
        q = torch.full((rows, 1, d), 2.0 ** 60) * (1 + torch.rand(rows, 1, d, generator=g))
        k = torch.randn(500, 1, d, generator=g).abs() * 2.0 ** -60 * torch.linspace(0.01, 3, 500)[:, None, None]
        k[:130] = -2.0 ** 100
        k[200:210] = -2.0 ** 100
        k[499] = -2.0 ** 100
        write(pool, s, k, torch.randn(500, 1, d, generator=g))
        batch = Batch(pool)
        batch.set([s], [rows])
        q = q.to(dtype).cuda()
        out = torch.empty_like(q)
        batch.attention(0, q, out)
        kk, vv = ref.gather(pool.keys, 0, pool.pages(s)), ref.gather(pool.values, 0, pool.pages(s))
        keep = (kk[:, 0, 0] > 0)
        want, size, spread = ref.attention(q.double().cpu(), kk[keep], vv[keep], d ** -0.5)
        tol = ref.attention_bound(want, size, spread, d, 500, dtype, ref.EPS_OF[BF16] if dtype == BF16 else 2.0 ** -24)
        assert ((out.double().cpu() - want).abs() <= tol).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kv,group,rows", [(1, 1, 200), (1, 1, 511), (256, 1, 65), (256, 1, 200), (256, 1, 257), (256, 4, 3),
                                           (256, 4, 40)])
def test_many_rows_over_every_number_of_tiles(kv, group, rows, d):
    """One to eleven tiles of keys, ending anywhere in a tile, starting anywhere in a page; one to three workgroups of rows
    (with 256 heads: workgroups of 256 rows, tests/test_branch_plan.py).  Three of the heads are compared."""
    heads = sorted({0, kv * group // 2 + 1, kv * group - 1} & set(range(kv * group)))
    for i, more in enumerate((0, 1, 62, 63, 64, 130, 195, 400)):
        keys, drop = rows + more, (0, 1, 15, 7)[i % 4]
        pool = make(BF16, pages=-(-(keys + 16) // 16) + 1, kv=kv, heads=kv * group, page=16, d=d, seqs=2, fill="nan")
        s = pool.new()
        pool.extend([s], [keys + drop])
        pool.trim(s, front=drop)
        g = torch.Generator().manual_seed(i)
        write(pool, s, *torch.randn(2, keys, kv, d, generator=g))
        batch = Batch(pool)
        batch.set([s], [rows])
        check_attention(pool, batch, [s], [rows], seed=i, only=heads)


@pytest.mark.parametrize("dtype,d", [(BF16, 64), (BF16, 128), (F32, 32), (F32, 64), (F32, 128)])
def test_few_rows_over_every_number_of_tiles(dtype, d):
    for rows in (1, 31, 32, 33, 64):
        for i, keys in enumerate((rows, 64, 65, 97, 128, 129, 160, 256, 300, 511)):
            pool = make(dtype, pages=40, kv=2, page=16, d=d, seqs=2, fill="nan")
            s = pool.new()
            drop = (0, 1, 15, 7)[i % 4]
            keys = max(keys, rows)
            pool.extend([s], [keys + drop])
            pool.trim(s, front=drop)
            g = torch.Generator().manual_seed(i)
            write(pool, s, *torch.randn(2, keys, 2, d, generator=g))
            batch = Batch(pool)
            batch.set([s], [rows])
            check_attention(pool, batch, [s], [rows], seed=i)


@pytest.mark.parametrize("dtype,d,kv,group,lengths", ref.LAST_ROUND)
def test_a_cut_last_round(dtype, d, kv, group, lengths):
    """Most rows whole, the last ones in pieces (tests/test_branch_plan.py): both, and the rows between them."""
    pool = make(dtype, pages=sum(-(-sum(x) // 64) for x in lengths), kv=kv, heads=kv * group, page=64, d=d, fill="nan")
    seqs, g = [], torch.Generator().manual_seed(8)
    for before, new in lengths:
        seqs.append(pool.new())
        pool.extend(seqs[-1:], [before + new])
        write(pool, seqs[-1], *torch.randn(2, before + new, kv, d, generator=g))
    batch = Batch(pool)
    new = [n for _, n in lengths]
    batch.set(seqs, new)
    heads = sorted({0, kv * group // 2, kv * group - 1})
    out, _ = check_attention(pool, batch, seqs, new, seed=9, only=heads)
    again, _ = check_attention(pool, batch, seqs, new, seed=9, only=heads)
    assert torch.equal(out, again)


def test_infinite_and_nan_tokens_stay_in_their_branch():
    pool = make(BF16, pages=64, kv=1, page=16, d=64)
    parent, seqs = grow(pool, 100, 0, [(20, 3), (20, 3), (20, 3)])
    first, tokens, pages = pool.pages(seqs[1])
    pool.values[0, pages[-1]] = math.nan
    pool.keys[0, pages[-2]] = math.inf
    batch = Batch(pool)
    batch.set(seqs, [3, 3, 3])
    q = torch.randn(9, 1, 64).to(BF16).cuda()
    out = torch.empty_like(q)
    batch.attention(0, q, out)
    assert torch.isnan(out[3:6]).any()
    assert torch.isfinite(out[:3]).all() and torch.isfinite(out[6:]).all()
    for i in (0, 2):
        one = Batch(pool)
        one.set([seqs[i]], [3])
        check_attention(pool, one, [seqs[i]], [3], q=q[3 * i:3 * i + 3])


def test_strided_rows_and_untouched_surroundings():
    pool = make(BF16, pages=40, kv=2, heads=4, page=16, d=64)
    parent, seqs = grow(pool, 50, 0, [(0, 7), (3, 9)])
    batch = Batch(pool)
    batch.set(seqs, [7, 9])
    big = torch.randn(18, 700).to(BF16).cuda()
    q = big[1:17, 8:8 + 256]
    frame = torch.full((20, 400), 5.0, dtype=BF16, device="cuda")
    with pytest.raises(XCacheError) as e:  # rows of 1400 bytes are not 16-byte aligned
        batch.attention(0, q, frame[2:18, 16:16 + 256])
    assert e.value.status == xcache.XC_ERR_INVALID_ARG and (frame == 5.0).all()
    q = torch.cat((big, big[:, :4]), 1)[1:17, 8:8 + 256]
    batch.attention(0, q, frame[2:18, 16:16 + 256])
    dense = torch.empty(16, 256, dtype=BF16, device="cuda")
    batch.attention(0, q.contiguous(), dense)
    assert torch.equal(frame[2:18, 16:272], dense)
    frame[2:18, 16:272] = 5.0
    assert (frame == 5.0).all()


def test_offsets_past_32_bits():
    """Pages whose bytes and whose elements lie past 2^32: bf16 rows of 8 heads x 128 in 2^31 + elements."""
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
    qkv = torch.randn(305, 3 * kv * d, device="cuda", generator=g).to(BF16)
    gain = torch.ones(d, device="cuda")
    for buf in (k, v):
        buf[0, n_pages - 40:] = torch.randn(40, kv, page, d, device="cuda", generator=g).to(BF16)
    batch = Batch(pool)
    batch.set(seqs, [5, 300])
    q = torch.empty(305, kv, d, dtype=BF16, device="cuda")
    batch.qk_norm_rope(0, qkv, gain, gain, None, 2.0, q)
    first, tokens, pages = pool.pages(seqs[1])
    got = ref.gather(v, 0, pool.pages(seqs[1]))[-300:]
    assert torch.equal(got, qkv[5:, 2 * kv * d:].double().cpu().view(300, kv, d))
    check_attention(pool, batch, seqs, [5, 300], q=q)
    # and the copies: a fork of the far sequence, then compaction into the freed low pages
    more = pool.fork(seqs[0], 1)
    pool.extend(more, [1])
    assert torch.equal(ref.gather(k, 0, pool.pages(more[0]))[:-1], ref.gather(k, 0, pool.pages(seqs[0])))
    before = ref.gather(k, 0, pool.pages(seqs[1]))
    pool.free([low])
    assert pool.compact() > 0 and max(pool.pages(seqs[1])[2]) < 40
    assert torch.equal(ref.gather(k, 0, pool.pages(seqs[1])), before)


# ---------------------------------------------------------------- norms and rotation

NORM_ROPE = [
    # dtype, q heads, kv heads, d, page, axes, rows per branch, first position
    (BF16, 1, 1, 128, 16, 1, [1], 0),
    (BF16, 12, 12, 128, 64, 3, [1] * 8, 10 ** 6),
    (BF16, 16, 4, 64, 16, 1, [1, 15, 16, 17, 400], 2 ** 31 - 500),
    (BF16, 5, 5, 64, 256, 3, [300, 1, 0, 257], -5),
    (BF16, 7, 1, 128, 32, 0, [33, 31], 0),
    (BF16, 3, 3, 128, 128, 3, [5000], 77),
    (F32, 4, 4, 32, 16, 3, [64, 64, 64], 12345),
    (F32, 3, 1, 64, 64, 1, [1, 100], 2 ** 30),
    (F32, 2, 2, 128, 16, 3, [47], 0),
    (F32, 5, 1, 32, 16, 0, [2, 1], 0),
]


@pytest.mark.parametrize("case", NORM_ROPE, ids=lambda c: f"{str(c[0])[6:]}-{c[1]}x{c[2]}-d{c[3]}-p{c[4]}-axes{c[5]}-{sum(c[6])}")
def test_norm_rope_into_pages(case):
    dtype, heads, kv, d, page, axes, new, base = case
    pool = make(dtype, blocks=2, pages=4 + sum(-(-n // page) + 1 for n in new), kv=kv, heads=heads, page=page, d=d)
    parent = pool.new()
    pool.extend([parent], [5])
    seqs = pool.fork(parent, len(new))
    pool.extend(seqs, new)
    batch = Batch(pool)
    batch.set(seqs, new)
    rows, width = sum(new), (heads + 2 * kv) * d
    g = torch.Generator().manual_seed(5)
    wide = torch.randn(rows, width + 64, generator=g) * torch.logspace(-4, 3, rows)[:, None]
    wide[rows // 2, :heads * d] = 0.0  # a row of zeros stays zero
    wide = wide.to(dtype).cuda()
    qkv = wide[:, 32:32 + width]
    gq, gk = 1 + 0.3 * torch.randn(2, d, generator=g)
    pos = None
    if axes:
        pos = (base + torch.arange(rows)[:, None] * torch.tensor([1, 1, 1][:axes]) +
               torch.randint(0, 300, (rows, axes), generator=g)).clamp(max=2 ** 31 - 1).to(torch.int32)
    keys, values = pool.keys.clone(), pool.values.clone()
    frame = torch.full((rows + 2, heads * d + 48), 3.0, dtype=dtype, device="cuda")
    batch.qk_norm_rope(1, qkv, gq.cuda(), gk.cuda(), pos.cuda() if axes else None, 10000.0,
                       frame[1:-1, 16:16 + heads * d])
    x = qkv.double().cpu().view(rows, heads + 2 * kv, d)
    worst = 0.0
    want, tol = ref.norm_rope(x[:, :heads], gq.double(), pos, 10000.0, dtype)
    got = frame[1:-1, 16:16 + heads * d].double().cpu().view(rows, heads, d)
    worst = max(worst, ((got - want).abs() / tol).max().item())
    assert ((got - want).abs() <= tol).all(), worst
    want_k, tol_k = ref.norm_rope(x[:, heads:heads + kv], gk.double(), pos, 10000.0, dtype)
    row = 0
    for s, n in zip(seqs, new):
        table = pool.pages(s)
        if n:
            k, v = (ref.gather(b, 1, table)[-n:] for b in (pool.keys, pool.values))
            assert ((k - want_k[row:row + n]).abs() <= tol_k[row:row + n]).all()
            assert torch.equal(v, x[row:row + n, heads + kv:])
            # what was not to be written is as it was
            at = np.arange(table[0] + table[1] - n, table[0] + table[1])
            p, r = (torch.from_numpy(i.astype(np.int64)).cuda() for i in (table[2][at // page], at % page))
            for buf, old in ((pool.keys, keys), (pool.values, values)):
                old[1][p, :, r] = buf[1][p, :, r]
        row += n
    assert torch.equal(pool.keys, keys) and torch.equal(pool.values, values)
    frame[1:-1, 16:16 + heads * d] = 3.0
    assert (frame == 3.0).all()
    print(f"[branches] {case} worst error / bound {worst:.3f}", flush=True)


def test_norm_rope_agrees_with_the_models_positions():
    """Scores of rotated rows depend on position differences alone (in every axis)."""
    d = 128
    pool = make(F32, pages=8, kv=1, page=16, d=d)
    s = pool.new()
    pool.extend([s], [2])
    batch = Batch(pool)
    batch.set([s], [2])
    x = torch.randn(1, 3 * d).repeat(2, 1).cuda()
    one = torch.ones(d, device="cuda")
    scores = []
    for shift in ([0, 0, 0], [10 ** 6, 5, 9]):
        pos = torch.tensor([[3, 4, 5], [9, 2, 8]]) + torch.tensor(shift)
        q = torch.empty(2, d, device="cuda")
        batch.qk_norm_rope(0, x, one, one, pos.int().cuda(), 10000.0, q)
        k = ref.gather(pool.keys, 0, pool.pages(s))[:, 0]
        scores.append((q.double().cpu() @ k.T)[0, 1].item())
    # each rotated number within 2^-18 of |a| + |b| <= 2 sqrt(d / 2) in norm: d products of numbers of norm sqrt(d)
    assert abs(scores[0] - scores[1]) <= 4 * 2.0 ** -18 * d


@pytest.mark.parametrize("dtype,heads,kv,d", [(BF16, 12, 6, 128), (BF16, 6, 3, 64), (F32, 3, 3, 32), (F32, 6, 2, 64),
                                              (F32, 2, 1, 128)])
def test_norm_rope_of_more_than_a_cache_holds(dtype, heads, kv, d):
    """More than 256 MB in and out; 400 rows from end to end are compared, the values of all of them."""
    row = (heads + 2 * kv) * d * (2 if dtype == BF16 else 4)
    rows, page = (256 << 20) // (2 * row) + 17, 64
    pool = make(dtype, pages=-(-rows // page) + 4, kv=kv, heads=heads, page=page, d=d, fill="nan")
    s = pool.new()
    pool.extend([s], [rows])
    batch = Batch(pool)
    batch.set([s], [rows])
    g = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randn(rows, heads + 2 * kv, d, generator=g, device="cuda").to(dtype)
    gq, gk = 1 + 0.3 * torch.randn(2, d, generator=g, device="cuda")
    pos = torch.randint(0, 10 ** 6, (rows, 3), generator=g, device="cuda").to(torch.int32)
    q = torch.full((rows, heads, d), math.nan, dtype=dtype, device="cuda")
    batch.qk_norm_rope(0, x, gq, gk, pos, 10000.0, q)
    pages = torch.from_numpy(pool.pages(s)[2].astype(np.int64)).cuda()
    keys, values = (b[0][pages].transpose(1, 2).reshape(-1, kv, d)[:rows] for b in (pool.keys, pool.values))
    assert torch.equal(values, x[:, heads + kv:]) and torch.isfinite(keys).all() and torch.isfinite(q).all()
    at = torch.linspace(0, rows - 1, 400, device="cuda").long()
    some = x[at].double().cpu()
    for got, src, gain in ((q, some[:, :heads], gq), (keys, some[:, heads:heads + kv], gk)):
        want, tol = ref.norm_rope(src, gain.double().cpu(), pos[at].cpu(), 10000.0, dtype)
        assert ((got[at].double().cpu() - want).abs() <= tol).all()


# ---------------------------------------------------------------- pages

@pytest.mark.parametrize("dtype,blocks,kv,d,page", [(BF16, 1, 1, 64, 16), (BF16, 3, 4, 128, 64), (F32, 2, 3, 32, 256),
                                                     (BF16, 2, 12, 128, 256)])
def test_page_copies(dtype, blocks, kv, d, page):
    """A search over branches: after every call each sequence reads what a list of its tokens says, in every block
    and both buffers; rows that no copy names are left as they were."""
    n_pages = 40
    pool = make(dtype, blocks=blocks, pages=n_pages, kv=kv, page=page, d=d, seqs=12)
    parent = pool.new()
    pool.extend([parent], [2 * page + page // 2 + 1])
    used = page // 2 + 1
    keys, values = pool.keys.clone(), pool.values.clone()
    tail = int(pool.pages(parent)[2][-1])
    kids = pool.fork(parent, 5)
    pool.extend(kids, [1, 1, 0, page, 2])
    for kid in kids:
        own = int(pool.pages(kid)[2][2])
        for buf, old in ((pool.keys, keys), (pool.values, values)):
            assert (own == tail) == (kid == kids[2])
            old[:, own, :, :used] = old[:, tail, :, :used]
    assert torch.equal(pool.keys, keys) and torch.equal(pool.values, values)
    # compaction: what every survivor reads stays, pages that no sequence holds too
    seen = {s: [pool.pages(s)[2].copy(), pool.pages(s)[1]] for s in (kids[1], kids[3])}
    pool.free([parent, kids[0], kids[2], kids[4]])
    moved = pool.compact()
    info = pool.info()
    assert moved > 0 and info["live_pages"] + info["free_pages"] == n_pages and info["live_seqs"] == 2
    to = {}
    for s, (old_pages, tokens) in seen.items():
        now = pool.pages(s)
        assert now[1] == tokens
        to.update(zip(old_pages.tolist(), now[2].tolist()))
    assert sorted(to.values()) == list(range(info["live_pages"]))
    src = torch.tensor(list(to))
    dst = torch.tensor([to[p] for p in to])
    for buf, old in ((pool.keys, keys), (pool.values, values)):
        new = old.clone()
        new[:, dst] = old[:, src]
        assert torch.equal(buf, new)


def test_copies_of_more_than_a_cache_holds():
    """80 branches, each with its own copy of the last page they share, 255 tokens of it: 2 x 196 MB."""
    pool = make(BF16, blocks=2, pages=84, kv=9, page=256, d=128, seqs=82)
    parent = pool.new()
    pool.extend([parent], [255])
    old = int(pool.pages(parent)[2][0])
    keys, values = pool.keys.clone(), pool.values.clone()
    kids = pool.fork(parent, 80)
    pool.extend(kids, [1] * 80)
    to = torch.tensor([int(pool.pages(k)[2][0]) for k in kids])
    assert old not in to and len(set(to.tolist())) == 80
    for buf, was in ((pool.keys, keys), (pool.values, values)):
        was[:, to, :, :255] = was[:, old:old + 1, :, :255]
        assert torch.equal(buf, was)


def test_many_copies_in_one_call():
    """More copies and moves than one launch takes."""
    pool = make(BF16, pages=2000, kv=1, page=16, d=64, seqs=900)
    parent = pool.new()
    pool.extend([parent], [9])
    kids = pool.fork(parent, 800)
    pool.extend(kids, [1] * 800)
    want = pool.keys[0, 0, :, :9]
    for kid in kids[::97] + kids[-1:]:
        assert torch.equal(pool.keys[0, int(pool.pages(kid)[2][0]), :, :9], want)
    assert len({int(pool.pages(k)[2][0]) for k in kids}) == 800
    ids = torch.tensor([int(pool.pages(k)[2][0]) for k in kids[1::2]])
    before = pool.keys[0, ids].clone()
    pool.free([parent] + kids[::2])
    assert pool.compact() > 100
    assert torch.equal(pool.keys[0, torch.tensor([int(pool.pages(k)[2][0]) for k in kids[1::2]])], before)
    long = pool.new()
    pool.extend([long], [16 * 700 - 3])
    first, tokens, pages = pool.pages(long)
    live = pool.info()["live_pages"] - 700
    assert (first, tokens) == (0, 16 * 700 - 3) and pages.tolist() == list(range(live, live + 700))


# ---------------------------------------------------------------- together

@pytest.mark.parametrize("dtype", [BF16, F32])
def test_a_search_over_futures(dtype):
    """Three generations of branching: every branch grows by a chunk, writes its keys and values over two passes, attends, the worst
    futures go, the best fork, the window rolls, the pool is compacted.  The reference keeps a list of tokens per branch."""
    blocks, kv, group, page, d, chunk, window = 2, 2, 2, 16, 64, 37, 90
    heads = kv * group
    pool = make(dtype, blocks=blocks, pages=120, kv=kv, heads=heads, page=page, d=d, seqs=10, fill="nan")
    width = (heads + 2 * kv) * d
    g = torch.Generator().manual_seed(11)
    gq, gk = (1 + 0.2 * torch.randn(2, d, generator=g)).cuda()
    batch, root = Batch(pool), pool.new()
    live, history, clock = [root], {root: [[] for _ in range(blocks)]}, 0
    for generation in range(4):
        pool.extend(live, [chunk] * len(live))
        batch.set(live, [chunk] * len(live))
        rows = chunk * len(live)
        t = clock + torch.arange(chunk).repeat(len(live))
        pos = torch.stack((t // 6, t % 6 // 3, t % 3), 1).int()
        for step in range(2):  # the second pass replaces the first one's keys and values
            for b in range(blocks):
                qkv = torch.randn(rows, width, generator=g).to(dtype).cuda()
                q = torch.empty(rows, heads, d, dtype=dtype, device="cuda")
                batch.qk_norm_rope(b, qkv, gq, gk, pos.cuda(), 100.0, q)
                x = qkv.double().cpu().view(rows, heads + 2 * kv, d)
                k, tol = ref.norm_rope(x[:, heads:heads + kv], gk.double().cpu(), pos, 100.0, dtype)
                for i, s in enumerate(live):
                    part = slice(i * chunk, (i + 1) * chunk)
                    past = history[s][b][:len(history[s][b]) - chunk * step]
                    history[s][b] = past + list(zip(k[part], tol[part], x[part, heads + kv:]))
                    kept = history[s][b][-min(len(history[s][b]), pool.pages(s)[1]):]
                    got = ref.gather(pool.keys, b, pool.pages(s))
                    assert len(kept) == len(got)
                    assert ((got - torch.stack([a for a, _, _ in kept])).abs() <= torch.stack([e for _, e, _ in kept])).all()
                    assert torch.equal(ref.gather(pool.values, b, pool.pages(s)), torch.stack([v for _, _, v in kept]))
                check_attention(pool, batch, live, [chunk] * len(live), block=b, q=q)
        clock += chunk
        # the first of the branches survives with the last one; both fork
        kept = sorted({live[0], live[-1]})
        gone = [s for s in live if s not in kept]
        pool.free(gone)
        for s in gone:
            del history[s]
        for s in kept:
            over = pool.pages(s)[1] - window
            if over > 0:
                pool.trim(s, front=over)
        pool.compact()
        live = list(kept)
        for s in kept:
            for c in pool.fork(s, 2):
                history[c] = [list(x) for x in history[s]]
                live.append(c)


def test_shared_pages_are_not_written():
    """Right after a fork the last tokens are shared: writing them again is refused until the other is gone."""
    pool = make(BF16, pages=16, kv=1, page=16, d=64)
    s = pool.new()
    pool.extend([s], [20])
    batch = Batch(pool)
    batch.set([s], [20])
    x, one = torch.randn(20, 192).to(BF16).cuda(), torch.ones(64, device="cuda")
    q = torch.empty(20, 64, dtype=BF16, device="cuda")
    batch.qk_norm_rope(0, x, one, one, None, 2.0, q)
    kid, = pool.fork(s, 1)
    keys = pool.keys.clone()
    with pytest.raises(XCacheError) as e:
        batch.qk_norm_rope(0, x * 2, one, one, None, 2.0, q)
    assert e.value.status == xcache.XC_ERR_STATE
    assert torch.equal(pool.keys, keys)
    # its attention is still that of the same tokens
    check_attention(pool, batch, [s], [20])
    pool.free([kid])
    batch.qk_norm_rope(0, x, one, one, None, 2.0, q)
    # a child that grew owns its last page, its first is shared: only rows in its own may be written
    kid, = pool.fork(s, 1)
    pool.extend([kid], [3])
    batch.set([kid], [7])
    batch.qk_norm_rope(0, x[:7], one, one, None, 2.0, q[:7])
    batch.set([kid], [8])
    with pytest.raises(XCacheError):
        batch.qk_norm_rope(0, x[:8], one, one, None, 2.0, q[:8])


def test_forks_that_did_not_grow_attend_to_the_same_tokens():
    """Every token shared, whole pages and the partly filled last one."""
    pool = make(BF16, pages=32, kv=2, page=16, d=64)
    s = pool.new()
    pool.extend([s], [200])
    kids = pool.fork(s, 3)
    batch = Batch(pool)
    for new in ([1, 1, 1], [200, 3, 64]):
        batch.set(kids, new)
        check_attention(pool, batch, kids, new)
    pool.trim(kids[1], front=30)
    pool.trim(kids[2], back=193)
    batch.set(kids, [2, 2, 2])
    check_attention(pool, batch, kids, [2, 2, 2])


# ---------------------------------------------------------------- streams, graphs, errors

def test_graph_replays_follow_their_inputs():
    """Norms, rotation and attention of a batch in one graph, replayed with new inputs, eager work between."""
    pool = make(BF16, pages=200, kv=4, page=16, d=128, seqs=20)
    st = torch.cuda.Stream()
    pool2 = Pool(pool.keys, pool.values, q_heads=4, max_seqs=20, stream=st.cuda_stream)
    parent, seqs = grow(pool2, 1500, 0, [(i, 2) for i in range(8)])
    torch.cuda.synchronize()
    batches = []
    for part in (seqs[:4], seqs[4:]):
        with torch.cuda.stream(st):
            b = Batch(pool2)
            b.set(part, [2] * 4)
            x = torch.randn(8, 12 * 128, device="cuda").to(BF16)
            q, out = (torch.empty(8, 4, 128, dtype=BF16, device="cuda") for _ in range(2))
            pos, one = torch.arange(8, device="cuda").int()[:, None], torch.ones(128, device="cuda")

            def call(b=b, x=x, q=q, out=out, pos=pos, one=one):
                b.qk_norm_rope(0, x, one, one, pos, 100.0, q)
                b.attention(0, q, out)

            call()
            st.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=st):
                call()
            batches.append((b, x, out, call, g))
    for turn in range(4):
        for b, x, out, call, g in batches:
            with torch.cuda.stream(st):
                x.copy_(torch.randn(8, 12 * 128, device="cuda"))
                g.replay()
                st.synchronize()
                got = out.clone()
                out.zero_()
                call()
                st.synchronize()
                assert torch.equal(got, out) and got.abs().sum() > 0


def test_changes_are_refused_inside_a_capture():
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        pool = make(BF16, pages=16, kv=1, page=16, d=64)
        s = pool.new()
        pool.extend([s], [5])
        batch = Batch(pool)
        batch.set([s], [1])
        q, out = (torch.ones(1, 64, dtype=BF16, device="cuda") for _ in range(2))
        st.synchronize()
        g = torch.cuda.CUDAGraph()
        refused = []
        with torch.cuda.graph(g, stream=st):
            for call in (lambda: pool.extend([s], [1]), lambda: batch.set([s], [1]), pool.compact):
                with pytest.raises(XCacheError) as e:
                    call()
                refused.append(e.value.status)
            batch.attention(0, q, out)
        assert refused == [xcache.XC_ERR_STATE] * 3
        g.replay()
        st.synchronize()
        assert torch.equal(out[0].cpu(), pool.values[0, 0, 0, :5].float().mean(0).to(BF16).cpu()) or torch.isfinite(out).all()
        pool.extend([s], [1])  # outside it works again


def test_batches_out_of_date_are_refused():
    pool = make(BF16, pages=32, kv=1, page=16, d=64)
    q, out = (torch.zeros(1, 64, dtype=BF16, device="cuda") for _ in range(2))
    batch = Batch(pool)
    with pytest.raises(ValueError):
        batch.attention(0, q, out)  # no rows yet
    lib = xcache.load_library()
    call = lambda: lib.xc_branch_attention(batch.b, 0, q.data_ptr(), 64, 0.0, out.data_ptr(), 64)  # noqa: E731
    assert call() == xcache.XC_ERR_STATE
    low = pool.new()
    pool.extend([low], [20])
    s, other = pool.new(), pool.new()
    for change in (lambda: pool.extend([s], [1]), lambda: pool.trim(s, 1, 0), lambda: (pool.free([low]), pool.compact()),
                   lambda: pool.free([s])):
        pool.extend([s, other], [3, 3])
        batch.set([s], [1])
        assert call() == xcache.XC_OK
        pool.fork(s, 1)
        pool.extend([other], [1])
        assert call() == xcache.XC_OK  # others' tables
        change()
        assert call() == xcache.XC_ERR_STATE
    # the number is used again: still refused
    assert pool.new() == s
    pool.extend([s], [3])
    assert call() == xcache.XC_ERR_STATE


def test_refused_arguments():
    pool = make(BF16, blocks=2, pages=16, kv=2, heads=4, page=16, d=64)
    s = pool.new()
    pool.extend([s], [5])
    batch = Batch(pool)
    batch.set([s], [5])
    lib, INVALID = xcache.load_library(), xcache.XC_ERR_INVALID_ARG
    x = torch.zeros(5, 512, dtype=BF16, device="cuda")
    q, out = (torch.zeros(5, 256, dtype=BF16, device="cuda") for _ in range(2))
    g = torch.ones(64, device="cuda")
    pos = torch.zeros(5, 3, dtype=torch.int32, device="cuda")
    good_a = dict(b=batch.b, block=0, q=q.data_ptr(), q_ld=256, scale=0.0, out=out.data_ptr(), ld=256)
    good_n = dict(b=batch.b, block=1, x=x.data_ptr(), ld=512, gq=g.data_ptr(), gk=g.data_ptr(), pos=pos.data_ptr(),
                  axes=3, theta=10000.0, q=q.data_ptr(), q_ld=256)
    assert lib.xc_branch_attention(*good_a.values()) == xcache.XC_OK
    assert lib.xc_qk_norm_rope(*good_n.values()) == xcache.XC_OK
    for bad in (dict(b=None), dict(block=-1), dict(block=2), dict(q=None), dict(out=None), dict(q_ld=255), dict(q_ld=248),
                dict(q_ld=260), dict(ld=-256), dict(ld=1 << 62), dict(scale=math.nan), dict(scale=math.inf), dict(scale=-1.0),
                dict(scale=1e-45), dict(scale=3.4e38), dict(q=q.data_ptr() + 2), dict(out=out.data_ptr() + 8),
                dict(out=q.data_ptr()), dict(out=q.data_ptr() + 4 * 512), dict(out=pool.keys.data_ptr()),
                dict(out=pool.values.data_ptr() + 4096)):
        assert lib.xc_branch_attention(*{**good_a, **bad}.values()) == INVALID, bad
    for bad in (dict(b=None), dict(block=2), dict(x=None), dict(gq=None), dict(gk=None), dict(q=None), dict(ld=511),
                dict(ld=504), dict(ld=516), dict(q_ld=0), dict(axes=2), dict(axes=0), dict(theta=1.0),
                dict(theta=math.nan), dict(theta=math.inf), dict(x=x.data_ptr() + 4), dict(q=q.data_ptr() + 4),
                dict(q=x.data_ptr(), q_ld=512), dict(q=pool.values.data_ptr()), dict(x=pool.keys.data_ptr())):
        assert lib.xc_qk_norm_rope(*{**good_n, **bad}.values()) == INVALID, bad
    ints = lambda *v: (ctypes.c_int32 * len(v))(*v)  # noqa: E731
    for seqs, new in (((s,), (6,)), ((s,), (-1,)), ((s, s), (1, 1)), ((9,), (0,)), ((-1,), (0,)), ((99,), (0,))):
        assert lib.xc_batch_set(batch.b, len(seqs), ints(*seqs), ints(*new)) == INVALID
    assert lib.xc_batch_set(batch.b, -1, None, None) == INVALID
    # the earlier rows are still there
    assert lib.xc_branch_attention(*good_a.values()) == xcache.XC_OK
    # the binding: shapes, types, places
    for bad in (q[:4], q.float(), q.cpu(), q.view(5, 8, 32)[:, :4], q.T):
        with pytest.raises(ValueError):
            batch.attention(0, bad, out)
    for bad in (dict(gq=g.double()), dict(gk=g[:32]), dict(positions=pos.long()), dict(positions=pos[:4]),
                dict(positions=pos[0]), dict(qkv=x[:, :504])):
        with pytest.raises(ValueError):
            batch.qk_norm_rope(**{**dict(block=0, qkv=x, gq=g, gk=g, positions=pos, theta=2.0, q_out=q), **bad})
    with pytest.raises(XCacheError):
        batch.qk_norm_rope(0, x, g, g, pos[:, :2].contiguous(), 2.0, q)
    with pytest.raises(XCacheError) as e:
        pool.extend([s], [17 * 16])
    assert e.value.status == xcache.XC_ERR_OOM and pool.pages(s)[1] == 5
    with pytest.raises(XCacheError):
        pool.fork(s, 16)
    # no rows: nothing to do, no refusal
    batch.set([s], [0])
    batch.attention(0, q[:0], out[:0])
    batch.qk_norm_rope(0, x[:0], g, g, pos[:0], 2.0, q[:0])
    batch.set([], [])
    batch.attention(0, q[:0], out[:0])


def test_a_batch_outlives_its_pool():
    pool = make(BF16, pages=16, kv=1, page=16, d=64)
    s = pool.new()
    pool.extend([s], [5])
    batch = Batch(pool)
    batch.set([s], [2])
    want = torch.empty(2, 64, dtype=BF16, device="cuda")
    q, out = torch.randn(2, 64).to(BF16).cuda(), torch.empty_like(want)
    batch.attention(0, q, want)
    pool.close()
    batch.attention(0, q, out)
    assert torch.equal(out, want)
    batch.close()


def test_batches_grow_and_shrink():
    """The tables and pieces of earlier, larger and smaller rows leave no trace."""
    pool = make(BF16, pages=700, kv=2, page=16, d=64, seqs=40)
    parent, seqs = grow(pool, 4000, 0, [(i % 5, 3) for i in range(32)])
    batch = Batch(pool)
    for part in (seqs[:1], seqs, seqs[3:5], seqs[1:30], []):
        new = [1 + i % 3 for i in range(len(part))]
        batch.set(part, new)
        if part:
            check_attention(pool, batch, part, new)


# ---------------------------------------------------------------- from a rollout

@pytest.mark.parametrize("grid", [None, (1, 5, 7), (3, 9, 11)])
@pytest.mark.parametrize("dtype,generations", [("f32", 1), ("f32", 3), ("bf16", 2), ("bf16", 5)])
def test_a_rollouts_history_is_shared_by_branches(dtype, generations, grid):
    """A model handle's window, imported: the tokens of the kept chunks, oldest first, in every block; then
    branches of it."""
    import synth
    from paper_2604_20289_amd.xcache import XC_CACHE_KEYS, XC_CACHE_VALUES, XCache
    w = synth.workload(0)
    w = synth.with_model(w, rope=1, kv_window=3, n_heads=4, head_dim=64 if dtype == "bf16" else 32,
                         hidden=256 if dtype == "bf16" else 128, mlp_hidden=512, dtype=dtype)
    if grid:  # an odd number of tokens
        w = synth.with_model(w, groups=(synth.ViewGroup(1, *grid),))
    m = w.model
    L, D, H = m.tokens, m.head_dim, m.n_heads
    h = XCache(m, w.gate, synth.make_weights(m), stream())
    taus = synth.timesteps(m)
    eps, acts = synth.latent_stream(m, w.stream, 0, generations), synth.action_stream(m, w.stream, 0, generations)
    y = torch.empty(L, m.hidden, device="cuda")
    for e, a in zip(eps, acts):
        x = torch.from_numpy(e).cuda()
        h.forward_chunk(0, taus[0], a, x, y)
        h.kv_update(0.0, a, y)
    torch_dtype = BF16 if dtype == "bf16" else F32
    pool = make(torch_dtype, blocks=m.n_blocks, pages=64, kv=H, page=16, d=D)
    seq = pool.new()
    pool.extend([seq], [5])
    kid, = pool.fork(seq, 1)
    pool.import_window(kid, h)  # after five tokens of its own: the shared page is copied first
    chunks = min(generations, 2)
    assert pool.pages(kid)[1] == 5 + chunks * L
    for b in range(m.n_blocks):
        for kind, buf in ((XC_CACHE_KEYS, pool.keys), (XC_CACHE_VALUES, pool.values)):
            ring = torch.empty(H, m.kv_window * L, D, device="cuda")
            h.read_cache(kind, 0, b, ring)
            got = ref.gather(buf, b, pool.pages(kid))
            assert torch.equal(got[:5], ref.gather(buf, b, pool.pages(seq)))
            for i in range(chunks):
                slot = (generations - chunks + i) % m.kv_window
                want = ring[:, slot * L:(slot + 1) * L].double().cpu().transpose(0, 1)
                assert torch.equal(got[5 + i * L:5 + (i + 1) * L], want)
    branches = pool.fork(kid, 3)
    pool.extend(branches, [1, 20, L])
    batch = Batch(pool)
    batch.set(branches, [1, 20, L])
    for b in range(m.n_blocks):
        check_attention(pool, batch, branches, [1, 20, L], block=b)
    # a handle of another shape or stream is refused
    other = make(torch_dtype, blocks=m.n_blocks + 1, pages=64, kv=H, page=16, d=D)
    with pytest.raises(XCacheError) as e:
        other.import_window(other.new(), h)
    assert e.value.status == xcache.XC_ERR_INVALID_ARG
    st = torch.cuda.Stream()
    third = Pool(pool.keys, pool.values, q_heads=H, stream=st.cuda_stream)
    with pytest.raises(XCacheError) as e:
        third.import_window(third.new(), h)
    assert e.value.status == xcache.XC_ERR_INVALID_ARG
    h.close()

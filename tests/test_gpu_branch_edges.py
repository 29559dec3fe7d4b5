"""Branch attention at the edges of its numbers and of its memory: tokens and queries that are not finite, scores past the
range of a float and the worst roundings of the probabilities, in every kernel; rows beside each other in one buffer;
buffers that grow under work in flight; a capture in which changes were refused."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import branch_reference as ref  # noqa: E402
from paper_2604_20289_amd import xcache  # noqa: E402
from paper_2604_20289_amd.xcache import Batch, XCacheError  # noqa: E402
from test_gpu_branches import BF16, F32, check_attention, grow, make, write  # noqa: E402

# type, key heads, head dim, rows per branch: with 256 heads the kernel of 256-row workgroups, with one the kernel of 64
# (tests/test_branch_plan.py)
KERNELS = [(BF16, 256, 64, 90), (BF16, 256, 128, 90), (BF16, 1, 64, 21), (BF16, 1, 128, 21), (BF16, 1, 64, 7), (BF16, 1, 128, 3),
           (F32, 1, 32, 21), (F32, 3, 64, 40), (F32, 1, 128, 9)]


def p_eps(dtype):
    return ref.EPS_OF[BF16] if dtype == BF16 else 2.0 ** -24


def expected(pool, seq, q, heads, weightless=None):
    """64-bit values and bounds of the given heads of one sequence's rows q; the bounds without a key that either weighs
    nothing or leaves nothing finite."""
    kv = pool.config.kv_heads
    k, v = (ref.gather(b, 0, pool.pages(seq)) for b in (pool.keys, pool.values))
    d, dtype = pool.config.head_dim, pool.keys.dtype
    kv_of, q = [h * kv // pool.config.q_heads for h in heads], q[:, heads].double().cpu()
    want, size, spread = ref.attention(q, k[:, kv_of], v[:, kv_of], d ** -0.5)
    if weightless is not None:
        keep = torch.arange(len(k)) != weightless
        _, size, spread = ref.attention(q, k[keep][:, kv_of], v[keep][:, kv_of], d ** -0.5)
    return want, ref.attention_bound(want, size, spread, d, len(k), dtype, p_eps(dtype))


@pytest.mark.parametrize("dtype,kv,d,rows", KERNELS)
@pytest.mark.parametrize("what", ["nan key", "inf key", "nan value", "inf value", "nan last value", "nan query", "inf query"])
def test_what_is_not_finite_stays_in_its_rows(what, dtype, kv, d, rows):
    """One number of the second of three branches: NaN and infinity come out where the formula has them, everything else
    is as it would be (an infinite key may weigh nothing in every row)."""
    pool = make(dtype, pages=4 * (-(-(300 + rows) // 16) + 2), kv=kv, page=16, d=d, seqs=4)
    parent, seqs = grow(pool, 130, 3, [(170, rows)] * 3)
    g = torch.Generator().manual_seed(21)
    head, dim = kv // 2, d // 3
    q = (torch.randn(3 * rows, kv, d, generator=g) * 0.7).to(dtype)
    bad = math.nan if "nan" in what else math.inf
    first, tokens, pages = pool.pages(seqs[1])
    place = first + (tokens - 1 if "last" in what else 200)  # one of its own, in a page of its own
    at = (0, int(pages[place // 16]), head, place % 16, dim)
    if "key" in what:
        pool.keys[at] = bad
    elif "value" in what:
        pool.values[at] = bad
    else:
        q[rows + 2, head, dim] = bad
    q = q.cuda()
    batch = Batch(pool)
    batch.set(seqs, [rows] * 3)
    out = torch.empty_like(q)
    batch.attention(0, q, out)
    got = out.double().cpu()
    heads = sorted({0, head, kv - 1})
    for i, s in enumerate(seqs):
        part = slice(i * rows, (i + 1) * rows)
        want, tol = expected(pool, s, q[part], heads, 200 if i == 1 and what == "inf key" else None)
        have = got[part][:, heads]
        finite = torch.isfinite(want)
        assert finite.all() or i == 1
        assert ((have - want)[finite].abs() <= tol[finite]).all(), (i, (have - want)[finite].abs().max())
        assert torch.equal(torch.isnan(have), torch.isnan(want)) and torch.equal(have[~finite].nan_to_num(), want[~finite].nan_to_num())
    assert what == "inf key" or not torch.isfinite(got[rows:2 * rows]).all()
    assert torch.isfinite(got[:rows]).all() and torch.isfinite(got[2 * rows:]).all()
    others = [h for h in range(kv) if h != head]
    assert torch.isfinite(got[:, others]).all()


@pytest.mark.parametrize("d,rows", [(64, 70), (128, 70), (64, 257), (128, 257)])
def test_scores_past_the_range_of_a_float_in_wide_workgroups(d, rows):
    """As tests/test_gpu_branches.py has it for the other kernels: keys whose product overflows to -infinity, whole tiles of
    them first, weigh nothing."""
    kv, keys = 256, 600
    pool = make(BF16, pages=40, kv=kv, page=16, d=d, seqs=2)
    s = pool.new()
    pool.extend([s], [keys])
    g = torch.Generator().manual_seed(4)
    q = (torch.full((rows, kv, d), 2.0 ** 60) * (1 + torch.rand(rows, 1, d, generator=g))).to(BF16).cuda()
    k = torch.randn(keys, 1, d, generator=g).abs() * 2.0 ** -60 * torch.linspace(0.01, 3, keys)[:, None, None]
    k[:130] = -2.0 ** 100
    k[200:210] = -2.0 ** 100
    k[keys - 1] = -2.0 ** 100
    write(pool, s, k.expand(keys, kv, d), torch.randn(keys, kv, d, generator=g))
    batch = Batch(pool)
    batch.set([s], [rows])
    out = torch.empty_like(q)
    batch.attention(0, q, out)
    kk, vv = ref.gather(pool.keys, 0, pool.pages(s)), ref.gather(pool.values, 0, pool.pages(s))
    keep = kk[:, 0, 0] > 0
    pick = [0, 100, kv - 1]
    want, size, spread = ref.attention(q[:, pick].double().cpu(), kk[keep][:, pick], vv[keep][:, pick], d ** -0.5)
    tol = ref.attention_bound(want, size, spread, d, keys, BF16, p_eps(BF16))
    assert torch.isfinite(out).all() and ((out[:, pick].double().cpu() - want).abs() <= tol).all()


def _worst_step(sign):
    """x in [0, 1), a bf16 number, whose 2^-x is rounded to bf16 by most in this direction."""
    x = torch.arange(128, dtype=torch.float64) / 128
    p = 2.0 ** -x
    err = (p.to(BF16).double() - p) / p * sign
    i = int(err.argmax())
    return x[i].item(), err[i].item()


@pytest.mark.parametrize("dtype,kv,d,rows", KERNELS)
def test_the_worst_roundings_of_the_probabilities(dtype, kv, d, rows):
    """Two kinds of keys, the probabilities of one all rounded up, of the other all down, by nearly half a step.

    With p(1 + e), |e| <= u, in the numerator alone the result is off by u sum p |v|.  Where the denominator sums the rounded
    ones too (256-row workgroups, d = 64) it is off by another u |o|, both times 1 / (1 - u)."""
    (up, e_up), (down, e_down) = _worst_step(1), _worst_step(-1)
    assert min(e_up, e_down) > 0.9 * 2.0 ** -9
    keys, u = max(300, rows), p_eps(dtype)
    pool = make(dtype, pages=40, kv=kv, page=16, d=d, seqs=2)
    s = pool.new()
    pool.extend([s], [keys])
    rare = torch.arange(keys) % 9 == 4
    k = torch.zeros(keys, kv, d)
    k[:, :, 0] = torch.where(rare, -up, -down - 1)[:, None]
    k[0, :, 0] = 0.0  # the maximum, a power of two
    v = torch.zeros(keys, kv, d)
    v[:, :, 1::2] = rare.float()[:, None, None]
    v[:, :, 0::2] = torch.where(rare, 1.0, -1.0)[:, None, None]
    write(pool, s, k, v)
    q = torch.zeros(rows, kv, d)
    q[:, :, 0] = 1.0
    q, scale = q.to(dtype).cuda(), math.log(2.0)
    out = torch.empty_like(q)
    batch = Batch(pool)
    batch.set([s], [rows])
    batch.attention(0, q, out, scale)
    want, size, spread = ref.attention(q.double().cpu(), k.double(), v.double(), scale)
    tol = ref.attention_bound(want, size, spread, d, keys, dtype, u)
    if kv == 256 and d == 64:
        tol = tol + u * (1 + 4 * u) * (want.abs() + u * size) + u * u * size
    err = (out.double().cpu() - want).abs()
    print(f"[branches] {dtype} {kv} heads of {d}: worst error / bound {(err / tol).max():.3f}", flush=True)
    assert (err <= tol).all()


@pytest.mark.parametrize("dtype,kv,d,rows", [(BF16, 2, 64, 33), (BF16, 4, 128, 5), (F32, 2, 32, 40)])
def test_rows_beside_each_other_in_one_buffer(dtype, kv, d, rows):
    """[qkv | q | out] of every row in one buffer: norms from the first to the second, attention from the second to the third."""
    def run(qkv, q, out):
        pool = make(dtype, pages=40, kv=kv, page=16, d=d, seqs=3)
        parent, (s,) = grow(pool, 100, 5, [(9, rows)])
        batch = Batch(pool)
        batch.set([s], [rows])
        one = torch.ones(d, device="cuda")
        batch.qk_norm_rope(0, qkv, one, one, torch.arange(rows, device="cuda").int()[:, None], 100.0, q)
        batch.attention(0, q, out)
        return pool.keys.clone(), q.clone(), out.clone()

    w = kv * d
    x = torch.randn(rows, 5 * w + 16).to(dtype).cuda()
    frame = x[:, 5 * w:].clone()
    want = run(x[:, :3 * w].clone(), *(torch.empty(rows, w, dtype=dtype, device="cuda") for _ in range(2)))
    got = run(x[:, :3 * w], x[:, 3 * w:4 * w], x[:, 4 * w:5 * w])
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(x[:, 5 * w:], frame)


def test_buffers_grow_under_work_in_flight():
    """Rows set anew, more each time, while the attention of the earlier ones is still running: both are right."""
    pool = make(BF16, pages=2200, kv=8, page=16, d=128, seqs=70)
    parent, seqs = grow(pool, 30000, 0, [(i % 4, 2) for i in range(64)])
    batch, single = Batch(pool), Batch(pool)
    g = torch.Generator(device="cuda").manual_seed(2)
    q = torch.randn(128, 8, 128, device="cuda", generator=g).to(BF16)
    outs, parts = [], (1, 2, 5, 12, 30, 64, 3, 64)
    for n in parts:
        batch.set(seqs[:n], [2] * n)
        for _ in range(3):
            out = torch.empty(2 * n, 8, 128, dtype=BF16, device="cuda")
            batch.attention(0, q[:2 * n], out)
        outs.append(out)
    for n, out in zip(parts, outs):
        single.set(seqs[:n], [2] * n)
        torch.cuda.synchronize()
        again = torch.empty_like(out)
        single.attention(0, q[:2 * n], again)
        assert torch.equal(out, again)
    check_attention(pool, single, seqs, [2] * 64, q=q, only=[0, 7])


def test_an_attention_captured_after_refused_changes_is_right():
    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        pool = make(BF16, pages=16, kv=1, page=16, d=64)
        s = pool.new()
        pool.extend([s], [5])
        batch = Batch(pool)
        batch.set([s], [2])
        q = torch.randn(2, 1, 64).to(BF16).cuda()
        out = torch.full((2, 1, 64), math.nan, dtype=BF16, device="cuda")
        st.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=st):
            for call in (lambda: pool.extend([s], [1]), lambda: batch.set([s], [1]), pool.compact):
                with pytest.raises(XCacheError) as e:
                    call()
                assert e.value.status == xcache.XC_ERR_STATE
            batch.attention(0, q, out)
        assert torch.isnan(out).all() and pool.pages(s)[1] == 5
        for turn in range(3):
            q.copy_(torch.randn(2, 1, 64))
            out.fill_(math.nan)
            graph.replay()
            st.synchronize()
            want, tol = expected(pool, s, q, [0])
            assert ((out.double().cpu() - want).abs() <= tol).all()
            eager = torch.empty_like(out)
            batch.attention(0, q, eager)
            st.synchronize()
            assert torch.equal(out, eager)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_chunk_of_more_pages_than_one_launch_fills(dtype):
    """15 635 tokens behind nine others, in pages of 16: the second launch begins at an odd token."""
    import synth
    from paper_2604_20289_amd.xcache import XC_CACHE_KEYS, XC_CACHE_VALUES, XCache
    w = synth.workload(0)
    d = 64 if dtype == "bf16" else 32
    w = synth.with_model(w, rope=1, kv_window=2, n_heads=2, head_dim=d, hidden=2 * d, mlp_hidden=128, dtype=dtype, n_blocks=2,
                         groups=(synth.ViewGroup(1, 5, 59, 53),))
    m = w.model
    L = m.tokens
    h = XCache(m, w.gate, synth.make_weights(m), torch.cuda.current_stream().cuda_stream)
    (e,), (a,) = synth.latent_stream(m, w.stream, 0, 1), synth.action_stream(m, w.stream, 0, 1)
    x, y = torch.from_numpy(e).cuda(), torch.empty(L, m.hidden, device="cuda")
    h.forward_chunk(0, synth.timesteps(m)[0], a, x, y)
    h.kv_update(0.0, a, y)
    pool = make(BF16 if dtype == "bf16" else F32, blocks=2, pages=1000, kv=2, page=16, d=d)
    keys, values = pool.keys.clone(), pool.values.clone()
    s = pool.new()
    pool.extend([s], [9])
    pool.import_window(s, h)
    first, tokens, pages = pool.pages(s)
    assert (first, tokens, len(pages)) == (0, 9 + L, 978)
    for kind, buf, old in ((XC_CACHE_KEYS, pool.keys, keys), (XC_CACHE_VALUES, pool.values, values)):
        for b in range(2):
            ring = torch.empty(2, 2 * L, d, device="cuda")
            h.read_cache(kind, 0, b, ring)
            rows = old[b, :978].transpose(1, 2).reshape(978 * 16, 2, d).clone()  # in order of place
            rows[9:9 + L] = ring[:, :L].transpose(0, 1).to(buf.dtype)
            old[b, :978] = rows.view(978, 16, 2, d).transpose(1, 2)
        assert torch.equal(buf, old)  # the tokens where they belong, everything else as it was
    h.close()


def test_another_streams_capture_is_left_alone():
    """While another stream is captured, a pool's calls on its own stream work, allocations among them, and the graph is whole."""
    own, other = torch.cuda.Stream(), torch.cuda.Stream()
    with torch.cuda.stream(own):
        pool = make(BF16, pages=400, kv=4, page=16, d=64, seqs=12)
        parent, seqs = grow(pool, 3000, 0, [(3, 2)] * 8)
        batch, gone = Batch(pool), Batch(pool)
        batch.set(seqs[:1], [1])
        gone.set(seqs[:1], [1])
        q = torch.randn(16, 4, 64).to(BF16).cuda()
        out = torch.zeros_like(q)
    x, y = torch.ones(8, device="cuda"), torch.zeros(8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=other):
        y.copy_(x * 2)
        batch.set(seqs, [2] * 8)
        batch.attention(0, q, out)
        gone.close()
        kid, = pool.fork(seqs[0], 1)
        pool.extend([kid], [1])
        y.add_(1)
    for turn in range(3):
        x.fill_(turn)
        graph.replay()
        torch.cuda.synchronize()
        assert (y == 2 * turn + 1).all()
    for i, s in enumerate(seqs):
        want, tol = expected(pool, s, q[2 * i:2 * i + 2], [0, 3])
        assert ((out[2 * i:2 * i + 2, [0, 3]].double().cpu() - want).abs() <= tol).all()

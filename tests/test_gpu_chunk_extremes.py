"""Weights of keys where one row's scores are as large as no sum of exponentials can follow, on the GPU: whatever that row gives to the
token that it attends to, the other tokens' weights are those of the other rows."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import branch_reference as ref  # noqa: E402
import chunk_reference as chunk  # noqa: E402
from paper_2604_20289_amd.xcache import Batch  # noqa: E402
from test_gpu_branches import BF16, F32, make, write  # noqa: E402


@pytest.mark.parametrize("dtype,d,rows", [(BF16, 64, 40), (BF16, 128, 40), (BF16, 64, 300), (BF16, 128, 300), (F32, 32, 40),
                                          (F32, 64, 70), (F32, 128, 300)])
@pytest.mark.parametrize("size", [3e8, -3e8, 7e9, -7e9, 1.1e10, 6e10, -6e10, 2e30, -2e30, 2.5e38])
def test_one_row_of_enormous_scores(size, dtype, d, rows):
    """Token t has all of its size in the first dim, so has the row at hand, and nobody else has anything there; -size: the first
    row, which sees the first token alone."""
    kv = 2
    pool = make(dtype, pages=-(-rows // 16) + 1, kv=kv, page=16, d=d, seqs=2)
    s = pool.new()
    pool.extend([s], [rows])
    g = torch.Generator().manual_seed(5)
    k, v = torch.randn(2, rows, kv, d, generator=g)
    q = torch.randn(rows, kv, d, generator=g)
    q[..., 0] = k[..., 0] = 0
    row = 0 if size < 0 else rows // 2
    t = 0 if size < 0 else row // 2
    q[row, :, 0], k[t, :, 0] = abs(size) ** 0.5, (abs(size) ** 0.5) * (1 if size > 0 else -1)
    write(pool, s, k, v)
    q = q.to(dtype).cuda()
    batch = Batch(pool)
    batch.set_chunk([s], [rows])
    k = ref.gather(pool.keys, 0, pool.pages(s))
    see = chunk.sees(rows, rows, 1, 0, 0)
    lse = torch.logsumexp(chunk.scores(q.double().cpu(), k, 1.0, see)[0], -1).T.float().cuda()  # of 64-bit scores
    assert (lse[row].cpu() / size - 1).abs().max() < 0.02  # (the square root's rounding to bf16, twice)
    w = torch.full((1, rows), 7.0, device="cuda")
    batch.chunk_weights(0, q, lse.contiguous(), w, decay=0.0, scale=1.0)
    others = [r for r in range(rows) if r != row]
    total, tol = chunk.weights(q.double().cpu()[others], k, 1.0, see[others], lse.double().cpu()[others])
    got = w[0].double().cpu()
    rest = torch.arange(rows) != t
    assert ((got - total).abs() <= tol + 1e-30)[rest].all()


@pytest.mark.parametrize("dtype,d,rows,kv", [(BF16, 64, 40, 2), (BF16, 128, 40, 2), (BF16, 64, 300, 256), (BF16, 128, 300, 256),
                                             (F32, 32, 40, 2), (F32, 64, 70, 2), (F32, 128, 300, 2)])
@pytest.mark.parametrize("size", [3e8, -3e8, 1.06e9, -1.06e9])
def test_scores_of_up_to_2_to_the_30(size, dtype, d, rows, kv):
    """As above: the row's result is the value of the token with all of its weight, through a probability and a result that are
    rounded once each; its log-sum-exp is the score, through a dozen roundings of 2^-24."""
    pool = make(dtype, pages=-(-rows // 16) + 1, kv=kv, page=16, d=d, seqs=2)
    s = pool.new()
    pool.extend([s], [rows])
    g = torch.Generator().manual_seed(9)
    k, v = torch.randn(2, rows, kv, d, generator=g)
    q = torch.randn(rows, kv, d, generator=g)
    q[..., 0] = k[..., 0] = 0
    row, t = (0, 0) if size < 0 else (rows // 2, rows // 4)
    root = 2.0 ** 15 if abs(size) > 1e9 else 2.0 ** 14
    q[row, :, 0], k[t, :, 0] = root, size / root
    write(pool, s, k, v)
    q = q.to(dtype).cuda()
    batch = Batch(pool)
    batch.set_chunk([s], [rows])
    out, lse = torch.empty_like(q), torch.empty(rows, kv, device="cuda")
    batch.chunk_attention(0, q, out, lse=lse, scale=1.0)
    k, v = (ref.gather(b, 0, pool.pages(s)) for b in (pool.keys, pool.values))
    score = (q[row].double().cpu() * k[t]).sum(-1)
    assert (score.abs() < 2.0 ** 30).all()
    assert ((out[row].double().cpu() - v[t]).abs() <= (2 * torch.finfo(dtype).eps / 2 + 2.0 ** -20) * v[t].abs()).all()
    assert ((lse[row].double().cpu() - score).abs() <= 12 * 2.0 ** -24 * score.abs()).all()
    assert torch.isfinite(out.double()).all() and torch.isfinite(lse).all()

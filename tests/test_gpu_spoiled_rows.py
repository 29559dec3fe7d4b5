"""Values that are not finite, in whole tokens and in the first place that some rows see, on the GPU: every row that sees one
has it in every column, in results and in pieces of results, and no other row has."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import branch_reference as ref  # noqa: E402
import chunk_reference as chunk  # noqa: E402
from paper_2604_20289_amd.xcache import Batch  # noqa: E402
from test_gpu_branches import BF16, F32, make, write  # noqa: E402
from test_gpu_chunks import p_eps  # noqa: E402


@pytest.mark.parametrize("dtype,d,rows", [(BF16, 64, 32), (BF16, 64, 64), (BF16, 128, 31), (BF16, 128, 64), (F32, 32, 32),
                                          (F32, 64, 32), (F32, 128, 29)])
@pytest.mark.parametrize("history", [5, 4000])
@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_every_row_that_sees_one_has_it(bad, history, dtype, d, rows):
    """One workgroup's rows (with 4000 tokens before them in pieces), a window whose first place the first rows see and the
    later ones do not, and a token in the middle of the new ones, which the later rows see."""
    tokens, kv = history + rows, 2
    pool = make(dtype, pages=-(-tokens // 16) + 1, kv=kv, page=16, d=d, seqs=2)
    s = pool.new()
    pool.extend([s], [tokens])
    g = torch.Generator().manual_seed(3)
    k, v = torch.randn(2, tokens, kv, d, generator=g)
    window = history + rows // 3
    at = [0, history + rows // 2]
    v[at, 1] = bad
    write(pool, s, k, v)
    batch = Batch(pool)
    batch.set_chunk([s], [rows], 1, window, 0)
    q = torch.randn(rows, kv, d, generator=g).to(dtype).cuda()
    out, lse = torch.empty_like(q), torch.empty(rows, kv, device="cuda")
    see = chunk.sees(tokens, rows, 1, window, 0)
    hit = see[:, at].any(1)
    assert see[:, 0].any() and not see[:, 0].all() and hit.any() and not hit.all()
    k, v = (ref.gather(b, 0, pool.pages(s)) for b in (pool.keys, pool.values))
    v0 = torch.where(torch.isfinite(v), v, torch.zeros_like(v))
    want, tol, want_lse, lse_tol = chunk.attention(q.double().cpu(), k, v0, d ** -0.5, see, dtype, p_eps(dtype))
    for _ in range(20):
        out.fill_(7.0)
        batch.chunk_attention(0, q, out, lse=lse)
        got = out.double().cpu()
        assert not torch.isfinite(got[hit, 1]).any()
        assert ((got - want).abs() <= tol)[:, 0].all() and ((got - want).abs() <= tol)[~hit, 1].all()
        assert ((lse.double().cpu() - want_lse).abs() <= lse_tol).all()

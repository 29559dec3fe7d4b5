"""Chunks under a mask through the binding, on the CPU (tests/chunk_host.py): what its checks of tensors refuse before the
library is called."""
import contextlib

import pytest

torch = pytest.importorskip("torch")

import chunk_host as chunk  # noqa: E402
import pool_host as host  # noqa: E402
from paper_2604_20289_amd import xcache  # noqa: E402
from paper_2604_20289_amd.xcache import Batch, Pool, XCacheError  # noqa: E402

pytestmark = pytest.mark.skipif(host.shutil.which("g++") is None, reason="no host compiler")


class Tensor(host.Tensor):
    """What the binding asks of rows and tables."""

    def __init__(self, at, shape, dtype="bfloat16", stride=None, device=0):
        super().__init__(at, shape, device)
        self.dtype = getattr(torch, dtype)
        self.steps = list(stride) if stride else [torch.empty(shape[i + 1:], device="meta").numel() for i in range(len(shape))]

    def stride(self, i=None):
        return self.steps if i is None else self.steps[i]

    def is_contiguous(self):
        return self.steps == [torch.empty(self.shape[i + 1:], device="meta").numel() for i in range(len(self.shape))]


@pytest.fixture
def made(monkeypatch):
    out = chunk.lib()
    out.xc_status_string.restype = xcache.load_library().xc_status_string.restype
    out.fake_reset()
    monkeypatch.setattr(xcache, "_lib", out)
    monkeypatch.setattr(torch.cuda, "device", lambda d: contextlib.nullcontext())
    shape = (1, 64, 2, 16, 64)
    pool = Pool(Tensor(host.KEYS, shape), Tensor(host.VALUES, shape), q_heads=4)
    a = pool.new()
    pool.extend([a], [100])
    b, = pool.fork(a, 1)
    pool.extend([b], [20])
    batch = Batch(pool)
    yield pool, batch, a, b
    batch.close()


def rows(n, width=256, at=chunk.ROWS, **kw):
    return Tensor(at, (n, width), **kw)


def lse(n, heads=4, dtype="float32", **kw):
    return Tensor(chunk.LSE, (n, heads), dtype, **kw)


def table(n, cols, dtype="float32", at=chunk.WEIGHTS, **kw):
    return Tensor(at, (n, cols), dtype, **kw)


def test_rows_and_tables_are_checked(made):
    pool, batch, a, b = made
    batch.set_chunk([a, b], [3, 5])
    out = rows(8, at=chunk.ROWS + (1 << 30))
    for bad in (rows(7), rows(8, 255), rows(8, device=1), rows(8, dtype="float32")):
        for call in (lambda: batch.chunk_attention(0, bad, out), lambda: batch.chunk_attention(0, out, bad),
                     lambda: batch.chunk_weights(0, bad, lse(8), table(2, 120))):
            with pytest.raises(ValueError):
                call()
    for bad in (lse(7), lse(8, 2), lse(8, device=1), lse(8, dtype="bfloat16"), lse(8, stride=(8, 1)), lse(8, stride=(1, 8))):
        for call in (lambda: batch.chunk_attention(0, rows(8), out, lse=bad),
                     lambda: batch.chunk_weights(0, rows(8), bad, table(2, 120))):
            with pytest.raises(ValueError):
                call()
    for bad in (table(2, 119), table(1, 120), table(3, 120), Tensor(chunk.WEIGHTS, (240,), "float32"), table(2, 120, "bfloat16"),
                table(2, 120, device=1), table(2, 120, stride=(1, 2))):
        for call in (lambda: batch.chunk_weights(0, rows(8), lse(8), bad), lambda: batch.evict([a, b], [10, 10], bad)):
            with pytest.raises(ValueError):
                call()
    for bad in (table(2, 29, "int32"), table(1, 30, "int32"), table(2, 30), table(2, 30, "int64"), table(2, 30, "int32", device=1),
                table(2, 30, "int32", stride=(1, 2))):
        with pytest.raises(ValueError):
            batch.evict([a, b], [10, 30], table(2, 120), bad)
    with pytest.raises(ValueError):
        batch.evict([a, b], [10], table(2, 120))
    with pytest.raises(ValueError):
        batch.set_chunk([a, b], [10])
    assert chunk.info()["last_launch"] == 2 and pool.tokens(a) == 100 and pool.tokens(b) == 120
    # what is allowed: heads apart, wider tables, rows further apart, no table where nothing shrinks
    batch.chunk_attention(0, Tensor(chunk.ROWS, (8, 4, 64), stride=(512, 64, 1)), out, lse=lse(8), scale=0.5)
    batch.chunk_weights(0, rows(8, stride=(264, 1)), lse(8), table(2, 120, stride=(500, 1)), decay=0.5)
    batch.evict([a, b], [100, 300], None)
    batch.evict([a, b], [100, 300], None, table(2, 120, "int32", chunk.KEPT))
    batch.evict([a, b], [10, 30], table(2, 130), table(2, 30, "int32", chunk.KEPT), sinks=4, recent=6)
    assert pool.tokens(a) == 10 and pool.tokens(b) == 30
    batch.evict([], [], None)


def test_rows_follow_the_batch(made):
    pool, batch, a, b = made
    with pytest.raises(XCacheError) as e:  # no rows yet
        batch.chunk_attention(0, rows(0), rows(0))
    assert e.value.status == xcache.XC_ERR_STATE
    batch.set_chunk([b], [120], group=7, window=50, sinks=3)
    assert batch.rows == 120
    batch.chunk_weights(0, rows(120), lse(120), table(1, 120))
    for bad in (dict(group=-1), dict(window=-1), dict(sinks=-1)):
        with pytest.raises(XCacheError) as e:
            batch.set_chunk([a], [1], **bad)
        assert e.value.status == xcache.XC_ERR_INVALID_ARG and batch.rows == 120
    batch.chunk_weights(0, rows(120), lse(120), table(1, 120))  # still the rows set before
    chunk.lib().fake_faults(0, -1, -1)
    with pytest.raises(XCacheError) as e:
        batch.set_chunk([a, b], [100, 120])
    chunk.lib().fake_faults(-1, -1, -1)
    assert e.value.status == xcache.XC_ERR_OOM and batch.rows == 0
    with pytest.raises(XCacheError) as e:
        batch.chunk_attention(0, rows(0), rows(0))
    assert e.value.status == xcache.XC_ERR_STATE
    batch.set_chunk([], [])
    batch.chunk_attention(0, rows(0), rows(0))
    batch.set_chunk([a, b], [0, 2])
    batch.chunk_attention(0, rows(2), rows(2, at=chunk.ROWS + (1 << 30)))

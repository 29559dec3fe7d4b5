"""Pool and Batch of the binding over the host side of the cache (tests/pool_host.py), on the CPU."""
import contextlib
import gc
import os
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")

import pool_host as host  # noqa: E402
from paper_2604_20289_amd import xcache  # noqa: E402
from paper_2604_20289_amd.xcache import Batch, Pool, XCacheError  # noqa: E402

pytestmark = pytest.mark.skipif(host.shutil.which("g++") is None, reason="no host compiler")


@pytest.fixture
def lib(monkeypatch):
    out = host.lib()
    out.xc_status_string.restype = xcache.load_library().xc_status_string.restype
    out.fake_reset()
    monkeypatch.setattr(xcache, "_lib", out)

    @contextlib.contextmanager
    def on(device):
        before = host.info()["device"]
        out.fake_set(device.index, 0)
        yield
        out.fake_set(before, 0)

    monkeypatch.setattr(torch.cuda, "device", on)
    yield out
    gc.collect()
    out.fake_set(0, 0)


def pool(device=0, **kw):
    shape = (1, 64, 2, 16, 64)
    return Pool(host.Tensor(host.KEYS, shape, device), host.Tensor(host.VALUES, shape, device), q_heads=2, **kw)


def test_a_batch_collected_during_a_capture_is_released_after_it(lib):
    p = pool()
    s = p.new()
    p.extend([s], [5])
    lost, kept = Batch(p), Batch(p)
    lost.set([s], [2])
    kept.set([s], [1])
    each = host.info()["live_bytes"] // 2
    lib.fake_set(0, 1)
    with pytest.raises(XCacheError) as e:  # asked for by name it is refused, and the batch stays
        kept.close()
    assert e.value.status == xcache.XC_ERR_STATE and kept.b
    del lost
    gc.collect()
    assert host.info()["live_bytes"] == 2 * each
    lib.fake_set(0, 0)
    kept.set([s], [2])
    assert host.info()["live_bytes"] == each and host.info()["freed_in_use"] == 0
    kept.close()
    assert host.info()["live_bytes"] == 0
    # the last one of all: whatever comes next releases it
    last = Batch(p)
    last.set([s], [1])
    lib.fake_set(0, 1)
    del last
    gc.collect()
    assert host.info()["live_bytes"] > 0
    lib.fake_set(0, 0)
    Batch(p)
    gc.collect()
    assert host.info()["live_bytes"] == 0 and host.info()["freed_unknown"] == 0


def test_a_pool_is_on_the_device_of_its_buffers(lib):
    """Another device is current when the pool is made: its work goes to the buffers' device, and the other stays current."""
    lib.fake_set(0, 0)
    p = pool(device=3)
    assert host.info()["device"] == 0
    s = p.new()
    p.extend([s], [5])
    kid, = p.fork(s, 1)
    p.extend([kid], [1])  # a copy of the shared page
    assert host.info()["launches"] == 1 and host.info()["launched_on"] == 3 and host.info()["device"] == 0


def test_batches_alive_at_the_end_of_the_program_end_quietly():
    code = """
import sys
sys.path[:0] = [{root!r}, {tests!r}]
import torch, contextlib
import pool_host as host
from paper_2604_20289_amd import xcache
lib = host.lib()
xcache._lib = lib
torch.cuda.device = lambda d: contextlib.nullcontext()
shape = (1, 64, 2, 16, 64)
p = xcache.Pool(host.Tensor(host.KEYS, shape), host.Tensor(host.VALUES, shape), q_heads=2)
s = p.new()
p.extend([s], [5])
b = xcache.Batch(p)
b.set([s], [2])
import builtins
builtins.held = b  # outlives the module
""".format(root=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), tests=os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True)
    assert r.returncode == 0 and r.stderr == "", r.stderr


def test_batches_released_later_are_released_once(lib, monkeypatch):
    """A collection in the middle of releasing them ends another batch, which comes by the same list."""
    p = pool()
    s = p.new()
    p.extend([s], [5])
    lost = [Batch(p) for _ in range(4)]
    extra = [Batch(p)]
    for b in lost + extra:
        b.set([s], [1])
    lib.fake_set(0, 1)
    lost.clear()
    del b
    gc.collect()
    lib.fake_set(0, 0)
    seen, destroy = [], lib.xc_batch_destroy

    class Lib:
        def __getattr__(self, name):
            return getattr(lib, name)

        def xc_batch_destroy(self, b):
            seen.append(b)
            assert seen.count(b) == 1  # (a second time would free it twice)
            if extra:
                extra.pop().__del__()
            return destroy(b)

    monkeypatch.setattr(xcache, "_lib", Lib())
    xcache._release_later()
    assert len(seen) == 5 and host.info()["live_bytes"] == 0 and not xcache._LATER

"""In which order the binding lets streams do things, shown on the CPU with
stand-ins for streams and the library: nothing here touches a GPU."""
import types

import pytest

torch = pytest.importorskip("torch")
mlkv = pytest.importorskip("paper_2406_09297_amd")

CURRENT, SIDE = 0x100, 0x200  # handles


class FakeStream:
    def __init__(self, handle, log, device_index=0):
        self.cuda_stream, self.log, self.device_index = handle, log, device_index

    def __eq__(self, other):
        return self.cuda_stream == other.cuda_stream

    def __hash__(self):
        return hash(self.cuda_stream)

    def wait_stream(self, other):
        self.log.append(("wait", self.cuda_stream, other.cuda_stream))


@pytest.fixture
def world(monkeypatch):
    """Streams, the allocator's record_stream and launches as entries of a log."""
    log = []
    current = FakeStream(CURRENT, log)
    monkeypatch.setattr(torch.cuda, "Stream", FakeStream)
    monkeypatch.setattr(torch.cuda, "ExternalStream",
                        lambda handle, device=None: FakeStream(handle, log))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: FakeStream(0, log))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: current)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: CURRENT, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch.Tensor, "record_stream",
                        lambda t, s: log.append(("record", s.cuda_stream)))
    empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, **k: (log.append(("empty",)), empty(*a, **k))[1])

    monkeypatch.setattr(mlkv, "_dev_ptr", lambda t, dtype, name: t.data_ptr())

    def launch(*args):
        log.append(("launch", args[-1]))
        return mlkv.MLKV_OK

    library = types.SimpleNamespace(
        mlkv_cache_read_rows=launch, mlkv_qcache_read_rows=launch, mlkv_workspace_init=launch,
        mlkv_workspace_bytes=lambda *a: 64, mlkv_workspace_bytes_window=lambda *a: 64)
    monkeypatch.setattr(mlkv, "lib", lambda: library)
    return types.SimpleNamespace(log=log, current=current, side=FakeStream(SIDE, log))


def _cache(kind):
    cache = object.__new__(kind)
    cache.n_kv, cache.batch, cache.capacity, cache.head_dim, cache._device = 1, 1, 32, 64, 0
    cache.data = cache.k = torch.zeros(1)
    cache._c = mlkv._Cache() if kind is mlkv.Cache else mlkv._QCache()
    return cache


MAP = types.SimpleNamespace(handle=None, workspace_bytes=lambda *a: 64)
MAKERS = [lambda s: _cache(mlkv.Cache).read_rows(stream=s),
          lambda s: _cache(mlkv.QCache).read_rows(stream=s),
          lambda s: mlkv.workspace(MAP, 1, 32, 64, device="cpu", stream=s),
          lambda s: mlkv.window_workspace(MAP, 1, 32, 64, device="cpu", stream=s)]


@pytest.mark.parametrize("make", MAKERS)
def test_what_a_call_allocates_is_written_in_order(make, world):
    """Memory from the current stream's pool is written on another stream only
    behind the work that the current one was given, and the allocator is told
    (or, for a bare handle, the current stream waits) before it can be reused."""
    for stream in (None, world.current, CURRENT):
        world.log.clear()
        make(stream)
        assert [e for e in world.log if e[0] != "empty"] == [("launch", CURRENT)]
    world.log.clear()
    make(world.side)
    made = world.log.count(("empty",))
    assert world.log[:made + 1] == [("empty",)] * made + [("wait", SIDE, CURRENT)]
    assert sorted(world.log[made + 1:]) == [("launch", SIDE)] + [("record", SIDE)] * made
    for handle in (SIDE, 0):  # 0: the default stream
        world.log.clear()
        make(handle)
        assert world.log == [("empty",)] * made + [("wait", handle, CURRENT), ("launch", handle),
                                                   ("wait", CURRENT, handle)]

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
        **{name: launch for name in mlkv.EXPORTS if name.startswith("mlkv_qcache_")
           or name.endswith("_window") or name == "mlkv_norm_rope_append"})
    library.__dict__.update(
        mlkv_cache_read_rows=launch, mlkv_workspace_init=launch,
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
def test_what_a_call_allocates_is_written_in_order(make, world, monkeypatch):
    """Memory from the current stream's pool is written on another stream only
    behind the work that the current one was given, and the allocator is told
    (or, for a bare handle, the current stream waits) before it can be reused."""
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)
    for stream in (None, world.current, CURRENT):
        world.log.clear()
        make(stream)
        assert [e for e in world.log if e[0] != "empty"] == [("launch", CURRENT)]
    world.log.clear()
    make(world.side)
    made = world.log.count(("empty",))
    assert world.log[:made + 1] == [("empty",)] * made + [("wait", SIDE, CURRENT)]
    assert sorted(world.log[made + 1:]) == [("launch", SIDE)] + [("record", SIDE)] * made
    with pytest.raises(ValueError, match="stream on device 1"):
        make(FakeStream(SIDE, world.log, device_index=1))
    for handle in (SIDE, 0):  # 0: the default stream
        world.log.clear()
        make(handle)
        assert world.log == [("empty",)] * made + [("wait", handle, CURRENT), ("launch", handle),
                                                   ("wait", CURRENT, handle)]


def _calls():
    """Every long-context call whose tensors the caller has made, on fakes."""
    B, h, D, S = 1, 2, 64, 32
    mp = types.SimpleNamespace(handle=None, _h=None, _heads=h, _owned=[1])
    bf16 = dict(dtype=torch.bfloat16)
    q, rows, lens = torch.zeros((B, h, D), **bf16), torch.zeros((1, B, S, D), **bf16), \
        torch.zeros(B, dtype=torch.int32)
    q4, new = torch.zeros((B, 1, h, D), **bf16), torch.zeros((B, 1, 1, D), **bf16)
    four, two = _cache(mlkv.QCache), _cache(mlkv.Cache)
    return [
        lambda s: four.write_rows(rows, rows, stream=s),
        lambda s: mlkv.qcache_append_rows(0, mp, four, new, new, lens, stream=s),
        lambda s: mlkv.qcache_decode_attention(0, q, four, mp, lens, q, stream=s),
        lambda s: mlkv.decode_attention_window(0, q, two, mp, lens, q, 8, stream=s),
        lambda s: mlkv.prefill_attention_window(0, q4, two, mp, lens, q4, 8, stream=s),
        lambda s: mlkv.norm_rope_append(0, mp, two, q4, new, new, lens, q4, stream=s),
        lambda s: mlkv.norm_rope_append(0, mp, four, q4, new, new, lens, q4, stream=s)]


@pytest.mark.parametrize("n", range(7))
def test_a_call_on_another_stream_comes_after_its_tensors(n, world, monkeypatch):
    """A torch Stream waits for the current one, which made the arguments, and the
    allocator keeps their memory for it; a bare handle and the current stream itself
    are launched on as they are."""
    monkeypatch.setattr(torch.Tensor, "get_device", lambda t: 0)
    call = _calls()[n]
    world.log.clear()
    for stream, handle in ((None, CURRENT), (world.current, CURRENT), (CURRENT, CURRENT),
                           (SIDE, SIDE)):
        call(stream)
        assert world.log == [("launch", handle)]
        world.log.clear()
    call(world.side)
    kept = world.log.count(("record", SIDE))  # the tensors passed, whatever becomes of them after
    assert kept == (2, 3, 3, 3, 3, 5, 5)[n]
    assert world.log == [("wait", SIDE, CURRENT)] + [("record", SIDE)] * kept + [("launch", SIDE)]
    with pytest.raises(ValueError, match="stream on device 1"):
        call(FakeStream(SIDE, world.log, device_index=1))


def test_a_workspace_elsewhere_is_refused(world, monkeypatch):
    """Its size is the current device's, and its fill would run there."""
    for device in (-1, 1):
        monkeypatch.setattr(torch.Tensor, "get_device", lambda t: device)
        with pytest.raises(ValueError, match="not the current one"):
            mlkv.window_workspace(MAP, 1, 32, 64, device="cpu")
    assert ("launch", CURRENT) not in world.log

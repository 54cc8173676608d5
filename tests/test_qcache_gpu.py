"""The 4-bit cache on the GPU: rows in and out against the plain statement of
its values and layout (tests/serve_ref.py), byte for byte."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import serve_ref  # noqa: E402
import synth  # noqa: E402
from gpu_util import say  # noqa: E402

pytestmark = pytest.mark.gpu

mlkv = pytest.importorskip("paper_2406_09297_amd")

POISON = 0xA5


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    mlkv.lib()
    yield


def _poisoned(n_kv, B, S, D):
    host = np.full((n_kv, B, S // 32, 34 * D), POISON, np.uint8)
    return mlkv.QCache(torch.from_numpy(host).cuda()), host


def _awkward_rows(seed, shape):
    """Rows with blocks of zeros, ties, values that round across a binade,
    negative zeros, the smallest and largest numbers, infinities and NaN."""
    bits = synth.normal_bf16(seed, 0, shape)
    flat = bits.reshape(-1, 32)
    one = synth.f32_to_bf16(np.array([0, .25, .5, .75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6,
                                      6.97, -.25, -.75, -2.5, -3.5, -5, -6, -0.0, .24, .26, .74,
                                      1.24, 1.76, 4.99, 5.01, 3.49, 2.49], np.float32))
    special = [np.zeros(32, np.uint16), np.full(32, 0x8000, np.uint16), one,
               synth.f32_to_bf16(synth.bf16_to_f32(one) * np.float32(2.0 ** 40)),
               np.arange(1, 33, dtype=np.uint16),            # subnormal numbers
               np.arange(0x0080, 0x0080 + 32 * 16, 16, dtype=np.uint16),
               np.full(32, 0x7F7F, np.uint16)]               # the largest
    for value in (0x7F80, 0xFF80, 0x7FC0):                   # not finite, among others
        row = flat[9].copy()
        row[11] = value
        special.append(row)
    for n, row in enumerate(special):
        flat[(n * 7 + 3) % flat.shape[0]] = row
    return bits


@pytest.mark.parametrize("D,n_kv,B,S", [(64, 3, 2, 96), (128, 2, 3, 64)])
def test_whole_cache_written_and_read_back(D, n_kv, B, S):
    say(f"qcache rows D={D}")
    k, v = _awkward_rows(11, (n_kv, B, S, D)), _awkward_rows(12, (n_kv, B, S, D))
    cache, ref = _poisoned(n_kv, B, S, D)
    cache.write_rows(mlkv.bf16_tensor(k, "cuda"), mlkv.bf16_tensor(v, "cuda"))
    for kv in range(n_kv):
        for b in range(B):
            serve_ref.store(ref, kv, b, 0, k[kv, b], v[kv, b])
    assert np.array_equal(cache.data.cpu().numpy(), ref)
    kr, vr = cache.read_rows()
    for got, want in zip((kr, vr), serve_ref.load(ref)):
        assert np.array_equal(got.double().cpu().numpy(), want, equal_nan=True)
    # What was read, stored again, is the same cache (NaN blocks included).
    again, _ = _poisoned(n_kv, B, S, D)
    again.write_rows(kr, vr)
    assert np.array_equal(again.data.cpu().numpy(), ref)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T", [1, 2, 7, 31, 32, 33, 70])
def test_append_touches_only_its_slots(D, T):
    """Ragged contexts across tile edges and past the cache's end, rows that are
    columns of wider ones, the second of two groups' heads."""
    g, S = 2, 128
    ctx = np.array([0, 1, 7, 31, 32, 33, 63, S - T, S - T // 2, S, S + 40, -5], np.int32)
    B = ctx.size
    say(f"qcache append D={D} T={T}")
    mp = mlkv.Map.uniform(4, 4, 2, g)
    wide = _awkward_rows(21, (B, T, 3 * g * D + 32))  # multiples of 32: whole blocks
    dev = mlkv.bf16_tensor(wide, "cuda")
    k_new = dev[..., :g * D].unflatten(-1, (g, D))
    v_new = dev[..., 2 * g * D:3 * g * D].unflatten(-1, (g, D))
    cache, ref = _poisoned(2 * g, B, S, D)
    lens = torch.from_numpy(ctx).cuda()
    mlkv.qcache_append_rows(2, mp, cache, k_new, v_new, lens)
    for b in range(B):
        for c in range(g):
            serve_ref.store(ref, g + c, b, int(ctx[b]), wide[b, :, c * D:(c + 1) * D],
                            wide[b, :, (2 * g + c) * D:(2 * g + c + 1) * D])
    assert np.array_equal(cache.data.cpu().numpy(), ref)
    k, v = cache.read_rows(g, g, starts=lens, T=T)
    want = serve_ref.load(ref)
    for got, rows in zip((k, v), want):
        got = got.double().cpu().numpy()
        for b in range(B):
            for t in range(T):
                slot = int(ctx[b]) + t
                exp = rows[g:, b, slot] if 0 <= slot < S else np.zeros((g, D))
                assert np.array_equal(got[:, b, t], exp, equal_nan=True), (b, t)


def test_rows_written_from_a_start_of_their_own():
    D, B, S, T = 64, 3, 96, 40
    say("qcache rows from starts")
    k, v = _awkward_rows(31, (1, B, T, D)), _awkward_rows(32, (1, B, T, D))
    starts = np.array([0, 29, 70], np.int32)
    cache, ref = _poisoned(2, B, S, D)
    cache.write_rows(mlkv.bf16_tensor(k, "cuda"), mlkv.bf16_tensor(v, "cuda"), 1,
                     starts=torch.from_numpy(starts).cuda())
    for b in range(B):
        serve_ref.store(ref, 1, b, int(starts[b]), k[0, b], v[0, b])
    assert np.array_equal(cache.data.cpu().numpy(), ref)


def test_token_by_token_is_the_same_cache_as_at_once():
    D, B, T = 128, 2, 45
    say("qcache token by token")
    k, v = _awkward_rows(41, (B, T, 1, D)), _awkward_rows(42, (B, T, 1, D))
    mp = mlkv.Map.uniform(2, 8, 1, 1)
    kd, vd = mlkv.bf16_tensor(k, "cuda"), mlkv.bf16_tensor(v, "cuda")
    ctx = torch.tensor([3, 30], dtype=torch.int32, device="cuda")
    at_once, _ = _poisoned(1, B, 96, D)
    mlkv.qcache_append_rows(0, mp, at_once, kd, vd, ctx)
    single, _ = _poisoned(1, B, 96, D)
    for t in range(T):
        mlkv.qcache_append_rows(0, mp, single, kd[:, t:t + 1], vd[:, t:t + 1], ctx + t)
    assert torch.equal(single.data, at_once.data)


def test_a_layer_without_heads_of_its_own_stores_nothing():
    mp = mlkv.Map.uniform(4, 4, 2, 1)
    cache, ref = _poisoned(2, 1, 32, 64)
    ctx = torch.zeros(1, dtype=torch.int32, device="cuda")
    rows = torch.zeros((1, 1, 0, 64), dtype=torch.bfloat16, device="cuda")
    mlkv.qcache_append_rows(1, mp, cache, rows, rows, ctx)
    torch.cuda.synchronize()
    assert np.array_equal(cache.data.cpu().numpy(), ref)


@pytest.mark.parametrize("as_handle", [False, True])
def test_rows_on_a_stream_of_their_own(as_handle):
    """Written and read on a stream that is not the current one."""
    D, B, S = 64, 2, 64
    k, v = (mlkv.bf16_tensor(_awkward_rows(s, (1, B, S, D)), "cuda") for s in (41, 42))
    cache, _ = _poisoned(1, B, S, D)
    cache.write_rows(k, v)
    want = cache.read_rows()
    other = mlkv.QCache.empty(1, B, S, D)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    stream = side.cuda_stream if as_handle else side
    other.write_rows(k, v, stream=stream)
    got = other.read_rows(stream=stream)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(got, want):
        assert torch.equal(a.view(torch.int16), b.view(torch.int16))

"""Argument checks of the long-context serving operators, which need no GPU:
every refusal happens before any HIP call."""
import ctypes

import pytest

mlkv = pytest.importorskip("paper_2406_09297_amd")
torch = pytest.importorskip("torch")

P = 0x10000  # stands for device memory: 16-byte aligned, never read
F32 = 0


def _name(status):
    return mlkv.STATUS_NAMES[status]


def _q(n_kv=4, B=2, S=64, D=64, data=P):
    return ctypes.byref(mlkv._QCache(data, n_kv, B, S, D))


def _c(n_kv=4, B=2, S=64, D=64, k=P, v=P):
    return ctypes.byref(mlkv._Cache(k, v, n_kv, B, S, D))


MAP = mlkv.Map.uniform(12, 12, 4, 1)  # layers 0, 3, 6, 9 own a head


def test_qcache_bytes():
    L = mlkv.lib()
    assert L.mlkv_qcache_bytes(MAP.handle, 3, 96, 64) == 4 * 3 * 3 * 34 * 64
    assert L.mlkv_qcache_bytes(MAP.handle, 64, 1 << 20, 128) == 4 * 64 * (1 << 15) * 34 * 128
    bf16 = MAP.cache_bytes(8, 2048, 128)
    assert abs(bf16 / L.mlkv_qcache_bytes(MAP.handle, 8, 2048, 128) - 64 / 17) < 1e-9
    for args in ((None, 3, 96, 64), (MAP.handle, 0, 96, 64), (MAP.handle, 3, 95, 64),
                 (MAP.handle, 3, 96, 96), (MAP.handle, 3, -32, 64)):
        assert L.mlkv_qcache_bytes(*args) == 0


BAD_QCACHES = [(dict(S=48), "MLKV_ERR_CAPACITY"), (dict(D=96), "MLKV_ERR_UNSUPPORTED"),
               (dict(data=P + 8), "MLKV_ERR_ALIGNMENT"), (dict(data=None), "MLKV_ERR_INVALID_ARG"),
               (dict(n_kv=3), "MLKV_ERR_INVALID_ARG"), (dict(B=0), "MLKV_ERR_INVALID_ARG"),
               (dict(S=0), "MLKV_ERR_INVALID_ARG")]


@pytest.mark.parametrize("change,want", BAD_QCACHES)
def test_a_bad_4_bit_cache_is_refused_everywhere(change, want):
    L, c, m = mlkv.lib(), _q(**change), MAP.handle
    nr = ctypes.byref(mlkv._NormRope(None, None, 0.0, 0, 1e4))
    assert _name(L.mlkv_qcache_append_rows(0, m, c, P, P, 1, 64, P, None)) == want
    assert _name(L.mlkv_qcache_decode_attention(0, P, c, m, P, 0, 0, P, F32, 0, P, 1 << 40,
                                                None)) == want
    assert _name(L.mlkv_qcache_norm_rope_append(0, m, c, P, 768, P, P, 64, 1, P, nr, P,
                                                None)) == want
    if change != dict(n_kv=3):  # no map: any number of heads
        for f in (L.mlkv_qcache_write_rows, L.mlkv_qcache_read_rows):
            assert _name(f(c, 0, 1, None, 1, P, P, None)) == want
    for f in (L.mlkv_qcache_write_rows, L.mlkv_qcache_read_rows):
        assert _name(f(None, 0, 1, None, 1, P, P, None)) == "MLKV_ERR_INVALID_ARG"


@pytest.mark.parametrize("args,want", [
    (dict(layer=12), "MLKV_ERR_INVALID_ARG"), (dict(layer=-1), "MLKV_ERR_INVALID_ARG"),
    (dict(k=None), "MLKV_ERR_INVALID_ARG"), (dict(v=P + 4), "MLKV_ERR_ALIGNMENT"),
    (dict(T=65), "MLKV_ERR_CAPACITY"), (dict(T=-1), "MLKV_ERR_CAPACITY"),
    (dict(stride=60), "MLKV_ERR_INVALID_ARG"), (dict(stride=68), "MLKV_ERR_INVALID_ARG"),
    (dict(ctx=None), "MLKV_ERR_INVALID_ARG"), (dict(ctx=P + 2), "MLKV_ERR_ALIGNMENT"),
    (dict(T=0, k=None, ctx=None), "MLKV_OK"), (dict(layer=1, k=None, ctx=None), "MLKV_OK")])
def test_append_rows(args, want):
    a = dict(layer=0, k=P, v=P, T=2, stride=64, ctx=P)
    a.update(args)
    assert _name(mlkv.lib().mlkv_qcache_append_rows(a["layer"], MAP.handle, _q(), a["k"], a["v"],
                                                    a["T"], a["stride"], a["ctx"], None)) == want


@pytest.mark.parametrize("args,want", [
    ((3, 2, None, 1, P, P), "MLKV_ERR_INVALID_ARG"), ((-1, 1, None, 1, P, P), "MLKV_ERR_INVALID_ARG"),
    ((2 ** 31 - 1, 2 ** 31 - 1, None, 1, P, P), "MLKV_ERR_INVALID_ARG"),
    ((0, 1, None, 65, P, P), "MLKV_ERR_CAPACITY"), ((0, 1, P + 1, 1, P, P), "MLKV_ERR_ALIGNMENT"),
    ((0, 1, None, 1, None, P), "MLKV_ERR_INVALID_ARG"), ((0, 1, None, 1, P, P + 8), "MLKV_ERR_ALIGNMENT"),
    ((2, 0, None, 1, None, None), "MLKV_OK"), ((0, 1, None, 0, None, None), "MLKV_OK")])
def test_rows(args, want):
    for f in (mlkv.lib().mlkv_qcache_write_rows, mlkv.lib().mlkv_qcache_read_rows):
        assert _name(f(_q(), *args, None)) == want


@pytest.mark.parametrize("four_bits", [True, False])
@pytest.mark.parametrize("args,want", [
    (dict(layer=12), "MLKV_ERR_INVALID_ARG"), (dict(q=None), "MLKV_ERR_INVALID_ARG"),
    (dict(q=P + 8), "MLKV_ERR_ALIGNMENT"), (dict(lens=None), "MLKV_ERR_INVALID_ARG"),
    (dict(lens=P + 2), "MLKV_ERR_ALIGNMENT"), (dict(out=P + 4), "MLKV_ERR_ALIGNMENT"),
    (dict(dtype=7), "MLKV_ERR_INVALID_ARG"), (dict(window=-1), "MLKV_ERR_INVALID_ARG"),
    (dict(sinks=-1), "MLKV_ERR_INVALID_ARG"), (dict(hint=4097), "MLKV_ERR_CAPACITY"),
    (dict(ws=None), "MLKV_ERR_WORKSPACE"), (dict(n=1000), "MLKV_ERR_WORKSPACE"),
    (dict(ws=P + 8), "MLKV_ERR_ALIGNMENT")])
def test_decode_attention(four_bits, args, want):
    a = dict(layer=0, q=P, lens=P, window=0, sinks=0, out=P, dtype=F32, hint=0, ws=P, n=1 << 40)
    a.update(args)
    L = mlkv.lib()
    f = L.mlkv_qcache_decode_attention if four_bits else L.mlkv_decode_attention_window
    c = _q(S=4096) if four_bits else _c(S=4096)
    assert _name(f(a["layer"], a["q"], c, MAP.handle, a["lens"], a["window"], a["sinks"], a["out"],
                   a["dtype"], a["hint"], a["ws"], a["n"], None)) == want
    assert _name(f(0, P, None, MAP.handle, P, 0, 0, P, F32, 0, P, 1 << 40, None)) == \
        "MLKV_ERR_INVALID_ARG"
    assert _name(f(0, P, c, None, P, 0, 0, P, F32, 0, P, 1 << 40, None)) == "MLKV_ERR_INVALID_ARG"


def test_more_units_than_a_launch_takes():
    mp = mlkv.Map.uniform(1, 8, 1, 8)
    c = _q(n_kv=8, B=1 << 21, S=32)
    assert _name(mlkv.lib().mlkv_qcache_decode_attention(0, P, c, mp.handle, P, 0, 0, P, F32, 0, P,
                                                         1 << 40, None)) == "MLKV_ERR_UNSUPPORTED"


def test_workspace_covers_every_call():
    """No call is refused for a workspace of mlkv_workspace_bytes_window bytes:
    each passes its checks and reaches the launch, which fails here (no GPU)."""
    if torch.cuda.is_available():
        pytest.skip("needs a machine without a GPU: the pointers are not memory")
    L = mlkv.lib()
    for l, h, m, g in ((12, 12, 4, 1), (2, 70, 1, 2), (4, 32, 2, 8), (1, 128, 1, 1)):
        mp = mlkv.Map.uniform(l, h, m, g)
        for B, S, D in ((1, 32, 64), (1, 32768, 128), (8, 4096, 64), (300, 2048, 64), (31, 640, 128)):
            n = L.mlkv_workspace_bytes_window(mp.handle, B, S, D)
            for hint in (0, 1, 33, S // 2, S):
                for window, sinks in ((0, 0), (1, 0), (100, 4), (S, S), (2 ** 31 - 1, 2 ** 31 - 1)):
                    if hint > S:
                        continue
                    st = L.mlkv_qcache_decode_attention(l - 1, P, _q(m * g, B, S, D), mp.handle, P,
                                                        window, sinks, P, F32, hint, P, n, None)
                    assert _name(st) == "MLKV_ERR_HIP", (l, h, B, S, D, hint, window)
    assert L.mlkv_workspace_bytes_window(MAP.handle, 0, 64, 64) == 0
    assert L.mlkv_workspace_bytes_window(MAP.handle, 1, 64, 80) == 0
    assert L.mlkv_workspace_bytes_window(None, 1, 64, 64) == 0


@pytest.mark.parametrize("args,want", [
    (dict(layer=12), "MLKV_ERR_INVALID_ARG"), (dict(q=None), "MLKV_ERR_INVALID_ARG"),
    (dict(q=P + 8), "MLKV_ERR_ALIGNMENT"), (dict(ctx=P + 2), "MLKV_ERR_ALIGNMENT"),
    (dict(T=65), "MLKV_ERR_CAPACITY"), (dict(T=-1), "MLKV_ERR_CAPACITY"),
    (dict(window=-1), "MLKV_ERR_INVALID_ARG"), (dict(sinks=-4), "MLKV_ERR_INVALID_ARG"),
    (dict(out=None), "MLKV_ERR_INVALID_ARG"), (dict(dtype=2), "MLKV_ERR_INVALID_ARG"),
    (dict(T=0), "MLKV_OK")])
def test_prefill_attention(args, want):
    a = dict(layer=0, q=P, ctx=P, T=2, window=8, sinks=1, out=P, dtype=F32)
    a.update(args)
    assert _name(mlkv.lib().mlkv_prefill_attention_window(
        a["layer"], a["q"], _c(), MAP.handle, a["ctx"], a["T"], a["window"], a["sinks"], a["out"],
        a["dtype"], None)) == want


def test_prefill_attention_beyond_a_grid():
    L = mlkv.lib()
    mq = mlkv.Map.uniform(1, 256, 1, 1)
    assert _name(L.mlkv_prefill_attention_window(0, P, _c(1, 1, 1 << 17), mq.handle, P, 70000, 8, 0,
                                                 P, F32, None)) == "MLKV_ERR_UNSUPPORTED"
    m8 = mlkv.Map.uniform(1, 8, 1, 8)
    assert _name(L.mlkv_prefill_attention_window(0, P, _c(8, 1 << 20, 32), m8.handle, P, 1, 8, 0, P,
                                                 F32, None)) == "MLKV_ERR_UNSUPPORTED"


@pytest.mark.parametrize("four_bits", [True, False])
@pytest.mark.parametrize("args,want", [
    (dict(layer=12), "MLKV_ERR_INVALID_ARG"), (dict(q=None), "MLKV_ERR_INVALID_ARG"),
    (dict(q=P + 8), "MLKV_ERR_ALIGNMENT"), (dict(qs=760), "MLKV_ERR_INVALID_ARG"),
    (dict(qs=772), "MLKV_ERR_INVALID_ARG"), (dict(k=None), "MLKV_ERR_INVALID_ARG"),
    (dict(v=P + 8), "MLKV_ERR_ALIGNMENT"), (dict(ns=56), "MLKV_ERR_INVALID_ARG"),
    (dict(T=65), "MLKV_ERR_CAPACITY"), (dict(ctx=None), "MLKV_ERR_INVALID_ARG"),
    (dict(ctx=P + 1), "MLKV_ERR_ALIGNMENT"), (dict(out=None), "MLKV_ERR_INVALID_ARG"),
    (dict(nr=None), "MLKV_ERR_INVALID_ARG"), (dict(nr=(P + 8, None, 0.0, 0, 1e4)), "MLKV_ERR_ALIGNMENT"),
    (dict(nr=(P, P, -1.0, 0, 1e4)), "MLKV_ERR_INVALID_ARG"),
    (dict(nr=(P, P, float("nan"), 0, 1e4)), "MLKV_ERR_INVALID_ARG"),
    (dict(nr=(P, P, 0.0, 8, 1e4)), "MLKV_ERR_UNSUPPORTED"),
    (dict(nr=(P, P, 0.0, 80, 1e4)), "MLKV_ERR_UNSUPPORTED"),
    (dict(nr=(P, P, 0.0, -16, 1e4)), "MLKV_ERR_UNSUPPORTED"),
    (dict(nr=(P, P, 0.0, 16, 0.0)), "MLKV_ERR_INVALID_ARG"),
    (dict(nr=(P, P, 0.0, 16, float("inf"))), "MLKV_ERR_INVALID_ARG"),
    (dict(T=0, q=None, k=None), "MLKV_OK")])
def test_norm_rope_append(four_bits, args, want):
    a = dict(layer=0, q=P, qs=768, k=P, v=P, ns=64, T=2, ctx=P, nr=(P, P, 1e-6, 16, 1e4), out=P)
    a.update(args)
    L = mlkv.lib()
    f = L.mlkv_qcache_norm_rope_append if four_bits else L.mlkv_norm_rope_append
    nr = None if a["nr"] is None else ctypes.byref(mlkv._NormRope(*a["nr"]))
    assert _name(f(a["layer"], MAP.handle, _q() if four_bits else _c(), a["q"], a["qs"], a["k"],
                   a["v"], a["ns"], a["T"], a["ctx"], nr, a["out"], None)) == want


def test_binding_checks_strides():
    rows = torch.zeros((2, 3, 10, 64), dtype=torch.bfloat16)
    shape = (2, 3, 10, 64)
    for bad in (rows.transpose(1, 2), rows[..., :32], rows.float(), rows[:1]):
        with pytest.raises(ValueError):
            mlkv._rows_arg(bad, shape, rows.get_device(), "k_new")
    with pytest.raises(ValueError):  # not a device tensor
        mlkv._rows_arg(rows, shape, 0, "k_new")
    wide = torch.zeros((2, 3, 1024), dtype=torch.bfloat16)[..., 64:704].unflatten(-1, (10, 64))
    assert mlkv._rows_arg(wide, shape, -1, "q") == (wide.data_ptr(), 1024)
    with pytest.raises(ValueError):  # sequences farther apart than their rows
        mlkv._rows_arg(torch.zeros((2, 4, 10, 64), dtype=torch.bfloat16)[:, :3], shape, -1, "q")
    for bad in (rows[0], rows.float(), rows.transpose(0, 1)):
        with pytest.raises(ValueError):
            mlkv._arg(bad, shape, torch.bfloat16, -1, "q")
    with pytest.raises(ValueError):
        mlkv.QCache.empty(1, 1, 40, 64, device="cpu")
    with pytest.raises(ValueError):
        mlkv.QCache(torch.zeros((1, 1, 1, 34 * 96), dtype=torch.uint8))

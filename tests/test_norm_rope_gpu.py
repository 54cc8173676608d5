"""Norm and rotation of queries and keys with the append, against the plain
64-bit statement (tests/serve_ref.py), and the operators together as one
layer of a serving program uses them."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import serve_ref  # noqa: E402
import synth  # noqa: E402
from gpu_util import say  # noqa: E402

pytestmark = pytest.mark.gpu

mlkv = pytest.importorskip("paper_2406_09297_amd")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    mlkv.lib()
    yield


def _projected(seed, B, T, h, g, D, scale=1.0):
    """One projection's rows [B][T][(h + 2 g) D], host bits and device columns."""
    bits = synth.normal_bf16(seed, 0, (B, T, (h + 2 * g) * D), scale=scale)
    dev = mlkv.bf16_tensor(bits, "cuda")
    cut = [(0, h), (h, g), (h + g, g)]
    return ([bits[..., a * D:(a + n) * D].reshape(B, T, n, D) for a, n in cut],
            [dev[..., a * D:(a + n) * D].unflatten(-1, (n, D)) for a, n in cut])


def _weight(seed, D):
    return synth.f32_to_bf16((1 + 0.1 * synth.bf16_to_f32(synth.normal_bf16(seed, 9, (D,)))))


def _check(got, bits, weight, eps, dims, base, pos, label):
    ref, bound = serve_ref.norm_rope(bits, weight, eps, dims, base, pos)
    d = np.abs(got - ref)
    assert np.all(d <= bound), (label, np.unravel_index(np.argmax(d - bound), d.shape), d.max())


@pytest.mark.parametrize("D,h,g,T,dims,normed", [
    (64, 12, 1, 1, 16, True), (64, 12, 4, 45, 64, True), (64, 7, 7, 3, 48, True),
    (128, 32, 8, 1, 128, True), (128, 8, 2, 33, 32, True), (64, 12, 3, 9, 0, True),
    (128, 4, 1, 70, 112, False), (64, 12, 1, 8, 16, False), (64, 1, 1, 17, 0, False)])
def test_queries_and_keys(D, h, g, T, dims, normed):
    """Odd head counts, partial and full rotation, either step left out, columns
    of a projection; contexts at tile edges and far positions."""
    S = 160
    ctx = np.array([0, 1, 31, 32, S - T], np.int32)
    B, eps, base = ctx.size, 1e-5, 500000.0
    label = f"norm D{D} h{h} g{g} T{T} dims{dims}"
    say(label)
    (q, k, v), (qd, kd, vd) = _projected(71, B, T, h, g, D, 2.0)
    wq, wk = (_weight(s, D) if normed else None for s in (1, 2))
    wd = [None if w is None else mlkv.bf16_tensor(w, "cuda") for w in (wq, wk)]
    mp = mlkv.Map.uniform(4, h, 2, g)
    cache = mlkv.Cache.empty(2 * g, B, S, D)
    cache.k.fill_(5.0)
    cache.v.fill_(6.0)
    q_out = torch.empty((B, T, h, D), dtype=torch.bfloat16, device="cuda")
    lens = torch.from_numpy(ctx).cuda()
    mlkv.norm_rope_append(2, mp, cache, qd, kd, vd, lens, q_out, q_norm=wd[0], k_norm=wd[1],
                          eps=eps, rotary_dims=dims, rotary_base=base)
    pos = ctx[:, None] + np.arange(T)
    _check(q_out.double().cpu().numpy(), q, wq, eps, dims, base, pos, label + " q")
    rows_k, rows_v = (x.double().cpu().numpy() for x in cache.read_rows())
    kept = np.ones((B, S), bool)
    for b in range(B):
        at = slice(ctx[b], ctx[b] + T)
        kept[b, at] = False
        _check(rows_k[g:, b, at].transpose(1, 0, 2), k[b], wk, eps, dims, base, pos[b], label + " k")
        assert np.array_equal(rows_v[g:, b, at].transpose(1, 0, 2), serve_ref.f64(v[b]))
    assert np.all(rows_k[:g] == 5) and np.all(rows_v[:g] == 6)
    assert np.all(rows_k[g:][:, kept] == 5) and np.all(rows_v[g:][:, kept] == 6)
    # The 4-bit cache holds the same bf16 rows' values, and the queries are the same.
    four = mlkv.QCache.empty(2 * g, B, S, D)
    four.data.fill_(0x11)
    q_four = torch.empty_like(q_out)
    mlkv.norm_rope_append(2, mp, four, qd, kd, vd, lens, q_four, q_norm=wd[0], k_norm=wd[1],
                          eps=eps, rotary_dims=dims, rotary_base=base)
    assert torch.equal(q_four, q_out)
    two = mlkv.QCache.empty(2 * g, B, S, D)
    two.data.fill_(0x11)
    k_rows = torch.stack([cache.read_rows(g, g)[0][:, b, ctx[b]:ctx[b] + T] for b in range(B)], 1)
    v_rows = vd.permute(2, 0, 1, 3).contiguous()
    two.write_rows(k_rows.contiguous(), v_rows, g, starts=lens)
    assert torch.equal(four.data, two.data)


@pytest.mark.parametrize("pos", [0, 1000, 131071, 10 ** 6, 2 * 10 ** 9])
def test_far_positions(pos):
    """The queries of a layer without heads of its own: positions alone count,
    up to the largest an int32 holds."""
    D, h = 64, 3
    (q, _, _), (qd, _, _) = _projected(72, 1, 1, h, 1, D)
    mp = mlkv.Map.uniform(2, h, 1, 1)
    cache = mlkv.Cache.empty(1, 1, 32, D)
    q_out = torch.empty((1, 1, h, D), dtype=torch.bfloat16, device="cuda")
    mlkv.norm_rope_append(1, mp, cache, qd, None, None,
                          torch.tensor([pos], dtype=torch.int32, device="cuda"), q_out,
                          rotary_dims=D)
    _check(q_out.double().cpu().numpy(), q, None, 0.0, D, 10000.0, np.array([[pos]]), f"pos {pos}")


def test_queries_in_place_and_rows_of_zeros():
    D, h, B, T = 128, 5, 2, 11
    (q, _, _), _ = _projected(73, B, T, h, 1, D)
    q[0, 3] = 0
    qd = mlkv.bf16_tensor(q, "cuda")
    mp = mlkv.Map.uniform(2, h, 1, 1)
    cache = mlkv.Cache.empty(1, B, 32, D)
    ctx = torch.tensor([4, 9], dtype=torch.int32, device="cuda")
    w = _weight(3, D)
    mlkv.norm_rope_append(1, mp, cache, qd, None, None, ctx, qd, q_norm=mlkv.bf16_tensor(w, "cuda"),
                          rotary_dims=64)
    pos = np.array([[4], [9]]) + np.arange(T)
    got = qd.double().cpu().numpy()
    _check(got, q, w, 1e-6, 64, 10000.0, pos, "in place")
    assert not got[0, 3].any()


def test_slots_outside_the_cache_are_skipped():
    D, g, S, T = 64, 1, 32, 4
    (q, k, v), (qd, kd, vd) = _projected(74, 3, T, 2, g, D)
    mp = mlkv.Map.uniform(2, 2, 1, g)
    ctx = torch.tensor([-2, 30, 500], dtype=torch.int32, device="cuda")
    for cache in (mlkv.Cache.empty(1, 3, S, D), mlkv.QCache.empty(1, 3, S, D)):
        planes = [cache.data] if isinstance(cache, mlkv.QCache) else [cache.k, cache.v]
        for p in planes:
            p.fill_(3)
        q_out = torch.empty((3, T, 2, D), dtype=torch.bfloat16, device="cuda")
        mlkv.norm_rope_append(0, mp, cache, qd, kd, vd, ctx, q_out)
        rows = cache.read_rows()[1].cpu()
        before = mlkv.QCache(torch.full_like(cache.data, 3)) if isinstance(cache, mlkv.QCache) \
            else None
        empty = before.read_rows()[1].cpu() if before else torch.full_like(rows, 3)
        assert torch.equal(rows[0, 0, 2:], empty[0, 0, 2:])
        assert torch.equal(rows[0, 1, :30], empty[0, 1, :30])
        assert torch.equal(rows[0, 2], empty[0, 2])
        if not before:
            assert torch.equal(rows[0, 0, :2], vd[0, 2:, 0].cpu())
            assert torch.equal(rows[0, 1, 30:], vd[1, :2, 0].cpu())


@pytest.mark.parametrize("D,h,g,window,sinks", [(64, 12, 1, 24, 3), (128, 8, 4, 0, 0)])
def test_a_layer_of_a_serving_loop(D, h, g, window, sinks):
    """A prompt of 40 tokens and ten single tokens through an owning layer and
    one that reads its heads: norm, rotation and append, then attention, from a
    bf16 cache and from the 4-bit cache, with the queries the calls made."""
    say(f"serving loop D{D} w{window}")
    B, T, S, eps = 3, 40, 96, 1e-6
    start = np.array([0, 5, 20], np.int32)
    mp = mlkv.Map.uniform(2, h, 1, g)
    bf16, four = mlkv.Cache.empty(g, B, S, D), mlkv.QCache.empty(g, B, S, D)
    bf16.k.fill_(float("nan"))
    bf16.v.fill_(float("nan"))
    four.data.fill_(0xFF)
    old_k, old_v = (synth.normal_bf16(75, s, (g, B, 20, D)) for s in (1, 2))
    zero = torch.zeros(B, dtype=torch.int32, device="cuda")
    bf = [mlkv.bf16_tensor(x, "cuda") for x in (old_k, old_v)]
    four.write_rows(*bf, starts=zero)  # slots up to 20 filled; a sequence attends its own
    full = [torch.zeros((g, B, S, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for x, rows in zip(full, bf):
        x[:, :, :20] = rows
    bf16.write_rows(*full)
    ws = mlkv.window_workspace(mp, B, S, D)
    w = [mlkv.bf16_tensor(_weight(s, D), "cuda") for s in (5, 6)]
    ctx = torch.from_numpy(start).cuda()

    def values():
        k, v = (x.double().cpu().numpy() for x in bf16.read_rows())
        return (k, v), tuple(x.double().cpu().numpy() for x in four.read_rows())

    def check(out, q, cached, n0, tokens, label):
        q, out = q.double().cpu().numpy(), out.double().cpu().numpy()
        G = h // g
        for b in range(B):
            for t in range(tokens):
                at = serve_ref.attended(int(n0[b]) + t, window, sinks)
                for r in range(g):
                    hs = slice(r * G, (r + 1) * G)
                    ref, bound = serve_ref.attend(q[b, t, hs], cached[0][r, b], cached[1][r, b], at)
                    assert np.all(np.abs(out[b, t, hs] - ref) <= bound), (label, b, t)

    for step in range(11):
        n = T if step == 0 else 1
        for layer in (0, 1):
            _, (qd, kd, vd) = _projected(80 + 2 * step + layer, B, n, h, g, D)
            new = (kd, vd) if layer == 0 else (None, None)
            q_bf16 = torch.empty((B, n, h, D), dtype=torch.bfloat16, device="cuda")
            q_four = torch.empty_like(q_bf16)
            kw = dict(q_norm=w[0], k_norm=w[1], eps=eps, rotary_dims=32)
            mlkv.norm_rope_append(layer, mp, bf16, qd, *new, ctx, q_bf16, **kw)
            mlkv.norm_rope_append(layer, mp, four, qd, *new, ctx, q_four, **kw)
            assert torch.equal(q_bf16, q_four)
            cached, cached4 = values()
            n0 = ctx.cpu().numpy()
            out = torch.empty((B, n, h, D), dtype=torch.float32, device="cuda")
            if n > 1:
                mlkv.prefill_attention_window(layer, q_bf16, bf16, mp, ctx, out, window, sinks)
                check(out, q_bf16, cached, n0, n, f"prompt layer {layer}")
                continue
            q1, o1 = q_bf16.view(B, h, D), out.view(B, h, D)
            mlkv.decode_attention_window(layer, q1, bf16, mp, ctx + 1, o1, window, sinks, ws=ws)
            check(out, q_bf16, cached, n0, 1, f"step {step} layer {layer}")
            mlkv.qcache_decode_attention(layer, q1, four, mp, ctx + 1, o1, window, sinks, ws=ws)
            check(out, q_bf16, cached4, n0, 1, f"step {step} layer {layer} 4-bit")
        ctx = ctx + n


@pytest.mark.parametrize("four_bits", [True, False])
def test_a_decode_step_captured_in_a_graph(four_bits):
    """Norm, rotation, append and attention of a layer as one graph: each replay
    follows the new projections and lengths, as the eager calls do on a cache of
    their own; split runs, several replays, eager work in between."""
    D, h, g, B, S, window = 64, 12, 4, 2, 1024, 500
    mp = mlkv.Map.uniform(2, h, 1, g)
    kind = mlkv.QCache if four_bits else mlkv.Cache
    caches = [kind.empty(g, B, S, D) for _ in range(2)]
    k, v = (mlkv.bf16_tensor(synth.normal_bf16(90, s, (g, B, S, D)), "cuda") for s in (1, 2))
    for cache in caches:
        cache.write_rows(k, v)
    w = mlkv.bf16_tensor(_weight(8, D), "cuda")
    x = torch.empty((B, 1, (h + 2 * g) * D), dtype=torch.bfloat16, device="cuda")
    ctx = torch.tensor([900, 30], dtype=torch.int32, device="cuda")
    lens = ctx + 1
    workspaces = [mlkv.window_workspace(mp, B, S, D) for _ in range(2)]
    attend = mlkv.qcache_decode_attention if four_bits else mlkv.decode_attention_window

    def step(cache, ws, q_out, out):
        q, kn, vn = (x[..., a * D:(a + n) * D].unflatten(-1, (n, D))
                     for a, n in ((0, h), (h, g), (h + g, g)))
        mlkv.norm_rope_append(0, mp, cache, q, kn, vn, ctx, q_out, q_norm=w, k_norm=w,
                              rotary_dims=D)
        attend(0, q_out.view(B, h, D), cache, mp, lens, out, window=window, sinks=4, ws=ws)

    outs = [torch.empty((B, h, D), dtype=torch.float32, device="cuda") for _ in range(2)]
    qs = [torch.empty((B, 1, h, D), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    x.normal_()
    step(caches[0], workspaces[0], qs[0], outs[0])
    step(caches[1], workspaces[1], qs[1], outs[1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(caches[0], workspaces[0], qs[0], outs[0])
    for n in range(4):
        x.copy_(mlkv.bf16_tensor(synth.normal_bf16(91 + n, 0, tuple(x.shape)), "cuda"))
        ctx.add_(1)
        lens.add_(1)
        graph.replay()
        step(caches[1], workspaces[1], qs[1], outs[1])
        torch.cuda.synchronize()
        assert torch.equal(qs[0], qs[1]) and torch.equal(outs[0], outs[1]), n
        pairs = [(caches[0].data, caches[1].data)] if four_bits else \
            [(caches[0].k, caches[1].k), (caches[0].v, caches[1].v)]
        for a, b in pairs:
            assert torch.equal(a, b)


def test_prompt_calls_on_a_stream_of_their_own_and_in_a_graph():
    """Append, norm and windowed prefill of a prompt: on another stream and
    replayed from a graph, the same results."""
    D, h, g, B, T, S = 128, 8, 2, 2, 70, 128
    mp = mlkv.Map.uniform(2, h, 1, g)
    _, (q, k, v) = _projected(95, B, T, h, g, D)
    ctx = torch.tensor([3, 40], dtype=torch.int32, device="cuda")
    old = [mlkv.bf16_tensor(synth.normal_bf16(96, s, (g, B, S, D)), "cuda") for s in (1, 2)]

    def run(stream=None):
        bf16, four = mlkv.Cache.empty(g, B, S, D), mlkv.QCache.empty(g, B, S, D)
        bf16.write_rows(*old, stream=stream)
        four.write_rows(*old, stream=stream)
        q_out = torch.empty((B, T, h, D), dtype=torch.bfloat16, device="cuda")
        out = torch.empty((B, T, h, D), dtype=torch.bfloat16, device="cuda")

        def calls():
            mlkv.norm_rope_append(0, mp, bf16, q, k, v, ctx, q_out, rotary_dims=32, stream=stream)
            mlkv.prefill_attention_window(0, q_out, bf16, mp, ctx, out, 33, 2, stream=stream)
            mlkv.qcache_append_rows(0, mp, four, k, v, ctx, stream=stream)
        return calls, (bf16.k, bf16.v, four.data, q_out, out)

    calls, want = run()
    calls()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    calls, got = run(side)
    calls()
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    calls, got = run()
    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for _ in range(3):
        got[3].zero_()
        got[4].zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("four_bits", [True, False])
def test_no_new_tokens_change_nothing(four_bits):
    B, h, g, D, S = 3, 4, 2, 64, 64
    mp = mlkv.Map.uniform(2, h, 1, g)
    cache = (mlkv.QCache if four_bits else mlkv.Cache).empty(g, B, S, D)
    planes = [cache.data] if four_bits else [cache.k, cache.v]
    for p in planes:
        p.fill_(3)
    empty = lambda n: torch.empty((B, 0, n, D), dtype=torch.bfloat16, device="cuda")  # noqa: E731
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")
    mlkv.norm_rope_append(0, mp, cache, empty(h), empty(g), empty(g), lens, empty(h),
                          rotary_dims=16)
    if four_bits:
        mlkv.qcache_append_rows(0, mp, cache, empty(g), empty(g), lens)
    for p in planes:
        assert (p == 3).all()


def test_rows_further_apart_than_a_c_int_are_refused():
    B, h, D = 2, 2, 64
    mp = mlkv.Map.uniform(2, h, 1, 1)
    cache = mlkv.Cache.empty(1, B, 32, D)
    q = torch.empty(2 ** 32 + 256, dtype=torch.bfloat16, device="cuda").as_strided(
        (B, 1, h, D), (2 ** 32, 2 ** 32, D, 1))
    with pytest.raises(ValueError, match="evenly spaced"):
        mlkv.norm_rope_append(1, mp, cache, q, None, None,
                              torch.zeros(B, dtype=torch.int32, device="cuda"),
                              torch.empty((B, 1, h, D), dtype=torch.bfloat16, device="cuda"))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("eps", [0.0, 1e-6])
def test_rows_whose_squares_leave_fp32(D, eps):
    """Rows up to bf16's largest and down to its smallest normal numbers, side
    by side: a row times a power of two has the same norm where eps is small
    beside it (below, the formula's 64 bits say what it has)."""
    h, B = 6, 11
    say(f"norm of extreme rows D={D} eps={eps}")
    powers = np.array([125, 100, 64, 63, 30, 0, -30, -44, -46, -70, -118])
    f = synth.bf16_to_f32(synth.normal_bf16(75, 0, (B, 1, h, D)))
    f = np.clip(f, -3.9, 3.9)  # 3.9 2^125 < 2^127
    f = np.where(np.abs(f) < 2.0 ** -8, np.float32(2.0 ** -8), f)  # normal numbers all
    bits = synth.f32_to_bf16(np.ldexp(f, powers[:, None, None, None]).astype(np.float32))
    w = _weight(3, D)
    mp = mlkv.Map.uniform(2, h, 1, 1)
    cache = mlkv.Cache.empty(1, B, 32, D)
    q_out = torch.empty((B, 1, h, D), dtype=torch.bfloat16, device="cuda")
    ctx = np.arange(B, dtype=np.int32)
    mlkv.norm_rope_append(1, mp, cache, mlkv.bf16_tensor(bits, "cuda"), None, None,
                          torch.from_numpy(ctx).cuda(), q_out, q_norm=mlkv.bf16_tensor(w, "cuda"),
                          eps=eps, rotary_dims=32)
    got = q_out.double().cpu().numpy()
    for b in range(B):
        if eps == 0 or powers[b] > -70:  # others leave bf16's normal numbers in the result
            _check(got[b:b + 1], bits[b:b + 1], w, eps, 32, 10000.0, ctx[b:b + 1, None],
                   f"row of 2^{powers[b]}")
    assert np.isfinite(got).all()

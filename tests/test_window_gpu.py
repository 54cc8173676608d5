"""Attention over the 4-bit cache and within a window, decode and prefill,
against the plain 64-bit statement (tests/serve_ref.py), each element within
the bound that bf16 weights and fp32 sums allow."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import serve_ref  # noqa: E402
import synth  # noqa: E402
from gpu_util import BOUND_MAX_POSITIONS, say  # noqa: E402

pytestmark = pytest.mark.gpu

mlkv = pytest.importorskip("paper_2406_09297_amd")

NAN = 0x7FC0


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    mlkv.lib()
    yield


class Case:
    """A layer's cache, 4-bit or bf16, of two groups of g heads, the second
    read by `layer`; slots that no sequence attends hold NaN."""

    def __init__(self, four_bits, h, g, D, lens, S, seed, k_scale=1.0, T=1, window=0, sinks=0):
        self.four_bits, self.h, self.g, self.D, self.T = four_bits, h, g, D, T
        self.lens = np.asarray(lens, np.int32)
        self.B, self.S, self.window, self.sinks = self.lens.size, S, window, sinks
        self.map = mlkv.Map.uniform(4, h, 2, g)
        shape = (g, self.B, S, D)
        k, v = synth.normal_bf16(seed, 1, shape, scale=k_scale), synth.normal_bf16(seed, 2, shape)
        self.attended = []
        for b, L in enumerate(self.lens):  # positions any of the T tokens (the last: L - 1) attends
            at = [serve_ref.attended(int(n), window, sinks) for n in range(L - T, L)]
            self.attended.append(at)
            off = np.setdiff1d(np.arange(S), np.concatenate(at + [np.zeros(0, int)]))
            k[:, b, off] = NAN
            v[:, b, off] = NAN
        kd, vd = mlkv.bf16_tensor(k, "cuda"), mlkv.bf16_tensor(v, "cuda")
        if four_bits:
            self.cache = mlkv.QCache.empty(2 * g, self.B, S, D)
            self.cache.data.fill_(0xFF)
            self.k, self.v = serve_ref.held(k), serve_ref.held(v)
        else:
            self.cache = mlkv.Cache.empty(2 * g, self.B, S, D)
            self.cache.k.fill_(float("nan"))
            self.cache.v.fill_(float("nan"))
            self.k, self.v = serve_ref.f64(k), serve_ref.f64(v)
        self.cache.write_rows(kd, vd, g)
        self.layer = 3
        qs = (self.B, T, h, D) if T > 1 else (self.B, h, D)
        self.q_bits = synth.normal_bf16(seed, 3, qs)
        self.q = mlkv.bf16_tensor(self.q_bits, "cuda")
        self.seq_lens = torch.from_numpy(self.lens).cuda()
        self.ws = mlkv.window_workspace(self.map, self.B, S, D)

    def decode(self, dtype=torch.float32, hint=0, stream=None):
        out = torch.full(self.q.shape, 7.0, dtype=dtype, device="cuda")
        f = mlkv.qcache_decode_attention if self.four_bits else mlkv.decode_attention_window
        f(self.layer, self.q, self.cache, self.map, self.seq_lens, out, window=self.window,
          sinks=self.sinks, max_len_hint=hint, ws=self.ws, stream=stream)
        return out

    def prefill(self, dtype=torch.float32):
        out = torch.full(self.q.shape, 7.0, dtype=dtype, device="cuda")
        mlkv.prefill_attention_window(self.layer, self.q, self.cache, self.map,
                                      self.seq_lens - self.T, out, window=self.window,
                                      sinks=self.sinks)
        return out

    def check(self, out, label, tokens=None):
        G = self.h // self.g
        out = out.double().cpu().numpy().reshape(self.B, self.T, self.h, self.D)
        q = serve_ref.f64(self.q_bits).reshape(out.shape)
        worst = 0.0
        for b in range(self.B):
            for t in range(self.T) if tokens is None else tokens:
                at = self.attended[b][t]
                for r in range(self.g):
                    hs = slice(r * G, (r + 1) * G)
                    ref, bound = serve_ref.attend(q[b, t, hs], self.k[r, b], self.v[r, b], at)
                    d = np.abs(out[b, t, hs] - ref)
                    if at.size > BOUND_MAX_POSITIONS:  # the bar of longer rows
                        bound = np.full(ref.shape, 2e-3 * max(1.0, np.abs(ref).max()))
                    assert np.all(d <= bound), (label, b, t, r, d.max(), bound.min())
                    worst = max(worst, float((d / np.maximum(bound, 1e-300)).max(initial=0.0)))
        say(f"  {label}: max|d|/bound={worst:.3f}")


WINDOWS = [(0, 0), (1, 0), (1, 1), (5, 0), (32, 0), (33, 32), (31, 3), (64, 40), (100, 200),
           (10 ** 9, 10 ** 9)]
LENS = [0, 1, 2, 31, 32, 33, 63, 64, 65, 96, 127, 160]


@pytest.mark.parametrize("four_bits", [True, False])
@pytest.mark.parametrize("D,h,g", [(64, 12, 1), (128, 8, 2)])
@pytest.mark.parametrize("window,sinks", WINDOWS)
def test_decode_lengths_and_windows_across_tile_edges(four_bits, D, h, g, window, sinks):
    label = f"decode {'4-bit' if four_bits else 'bf16'} D{D} w{window} s{sinks}"
    say(label)
    c = Case(four_bits, h, g, D, LENS, 160, 51, window=window, sinks=sinks)
    c.check(c.decode(), label)


@pytest.mark.parametrize("four_bits", [True, False])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("G", [1, 3, 16, 17, 24, 33, 70])
def test_decode_group_sizes(four_bits, D, G):
    """One to many query heads per KV head: one block of rows, two, and several
    chunks; long enough for split runs."""
    label = f"decode {'4-bit' if four_bits else 'bf16'} D{D} G{G}"
    say(label)
    c = Case(four_bits, 2 * G, 2, D, [700, 33, 1], 704, 52, window=0 if G % 2 else 530, sinks=4)
    c.check(c.decode(), label)


@pytest.mark.parametrize("four_bits", [True, False])
@pytest.mark.parametrize("D,lens,window,sinks", [
    (64, [6000, 40, 0, 2500], 0, 0), (64, [9000], 4000, 70), (128, [3000, 2999], 0, 0),
    (128, [5000], 2049, 1), (64, [33] * 40 + [3000], 0, 0)])
def test_decode_split_runs(four_bits, D, lens, window, sinks):
    """Few long sequences are cut into many runs and merged in place: within the
    bound, the same bits every time, also from another stream and after other
    calls on the same workspace."""
    label = f"decode split {'4-bit' if four_bits else 'bf16'} D{D} {lens[:4]} w{window}"
    say(label)
    S = (max(lens) + 63) // 32 * 32
    c = Case(four_bits, 12, 4, D, lens, S, 53, k_scale=3.0, window=window, sinks=sinks)
    out = c.decode(hint=max(lens))
    c.check(out, label)
    for _ in range(5):
        assert torch.equal(c.decode(hint=max(lens)), out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = c.decode(hint=max(lens), stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, out)
    # The counters are left at zero for whoever uses the workspace next.
    assert not c.ws[:262144].any() or c.ws.numel() <= 16
    bf16 = c.decode(torch.bfloat16, hint=max(lens))
    assert torch.equal(bf16, out.bfloat16())


@pytest.mark.parametrize("four_bits", [True, False])
@pytest.mark.parametrize("D,B,g,window", [(64, 70, 4, 0), (64, 70, 4, 2100), (128, 35, 4, 0)])
def test_more_long_sequences_than_compute_units(four_bits, D, B, g, window):
    """Grids of several rounds of the compute units, whose long units are cut too."""
    say(f"span rounds D={D} B={B} window={window} four_bits={four_bits}")
    lens = np.array([(1, 2145, 40, 1100, 0, 2176, 2079, 300)[b % 8] for b in range(B)])
    c = Case(four_bits, h=2 * g, g=g, D=D, lens=lens, S=2176, seed=83, window=window,
             sinks=3 if window else 0)
    c.check(c.decode(), "rounds")


def test_lengths_above_the_hint_are_truncated_to_it():
    c = Case(True, 12, 1, 64, [300, 100], 320, 54)
    out = c.decode(hint=100)
    c.attended = [[np.arange(100)], [np.arange(100)]]
    c.check(out, "decode truncated")


@pytest.mark.parametrize("four_bits", [True, False])
def test_lengths_outside_the_cache_are_clamped(four_bits):
    c = Case(four_bits, 12, 1, 64, [64, 64], 64, 55)
    want = c.decode()
    c.seq_lens = torch.tensor([2 ** 31 - 1, -3], dtype=torch.int32, device="cuda")
    got = c.decode()
    assert torch.equal(got[0], want[0]) and not got[1].any()


@pytest.mark.parametrize("four_bits", [True, False])
@pytest.mark.parametrize("window", [0, 40])
def test_what_is_attended_and_not_finite_comes_through(four_bits, window):
    """A NaN key makes its heads NaN; a value that is not finite makes its
    channels so (in 4 bits: its block of 32); other sequences keep theirs."""
    D = 64
    c = Case(four_bits, 4, 1, D, [90, 90, 90, 90], 96, 56, window=window)
    clean = c.decode()
    k, v = (t.clone() for t in c.cache.read_rows(1, 1)[:2]) if four_bits else \
        (t.clone() for t in c.cache.read_rows(1, 1))
    k[0, 0, 70, 5] = float("nan")
    v[0, 1, 70, 40] = float("inf")
    v[0, 2, 70, 40] = float("nan")
    c.cache.write_rows(k, v, 1)
    out = c.decode()
    assert out[0].isnan().all()
    block = slice(32, 64) if four_bits else slice(40, 41)
    rest = [d for d in range(D) if not block.start <= d < block.stop]
    for b in (1, 2):
        assert not out[b][:, block].isfinite().any()
        assert torch.equal(out[b][:, rest], clean[b][:, rest])
    assert torch.equal(out[3], clean[3])


@pytest.mark.parametrize("four_bits", [True, False])
def test_decode_captured_in_a_graph_follows_the_lengths(four_bits):
    c = Case(four_bits, 12, 4, 64, [1500, 900], 1600, 57, window=1000, sinks=5)
    c.decode()
    out = torch.empty(c.q.shape, dtype=torch.float32, device="cuda")
    f = mlkv.qcache_decode_attention if four_bits else mlkv.decode_attention_window
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        f(c.layer, c.q, c.cache, c.map, c.seq_lens, out, window=1000, sinks=5, ws=c.ws)
    for lens in ([1500, 900], [1400, 1], [1500, 900], [0, 1203]):
        # Shorter sequences only: every attended slot of theirs is filled.
        c.cache.k.nan_to_num_(0) if not four_bits else c.cache.data.copy_(
            torch.where(c.cache.data == 255, torch.zeros_like(c.cache.data), c.cache.data))
        c.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        if not four_bits:
            c.cache.v.nan_to_num_(0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, c.decode())


def test_two_graphs_share_a_workspace():
    """Calls of other shapes, split into other runs, replayed in turn."""
    say("two graphs, one workspace")
    cases = [Case(True, 12, 2, 64, [3000, 5, 900], 3008, 86),
             Case(False, 8, 4, 128, [1500, 2000], 2016, 87, window=1700, sinks=9)]
    ws = max((c.ws for c in cases), key=lambda t: t.numel())
    outs, graphs, want = [], [], []
    for c in cases:
        c.ws = ws
        want.append(c.decode())
        f = mlkv.qcache_decode_attention if c.four_bits else mlkv.decode_attention_window
        outs.append(torch.empty_like(want[-1]))
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            f(c.layer, c.q, c.cache, c.map, c.seq_lens, outs[-1], window=c.window, sinks=c.sinks,
              ws=ws)
    for turn in range(4):
        for g, out, w, c in zip(graphs, outs, want, cases):
            out.fill_(7.0)
            g.replay()
            assert torch.equal(out, w), turn
            if turn % 2:
                assert torch.equal(c.decode(), w)


@pytest.mark.parametrize("L", [40, 700])
def test_scores_that_are_all_minus_infinity_give_nan(L):
    """The quotient is 0 / 0; a sequence with one finite score has its value."""
    c = Case(False, 4, 1, 64, [L, L, 0], 704, 58)
    k, v = (t.clone() for t in c.cache.read_rows(1, 1))
    c.q[:, :, 0] = 1.0
    k[0, :, :L, 0] = -float("inf")
    k[0, 1, L - 7, 0] = 1.0
    c.cache.write_rows(k, v, 1)
    out = c.decode()
    assert out[0].isnan().all() and not out[2].any()
    assert torch.equal(out[1], v[0, 1, L - 7].float().expand(4, 64))
    pre = torch.empty((3, 1, 4, 64), dtype=torch.float32, device="cuda")
    c.seq_lens[2] = 1  # prefill has a token in every sequence
    mlkv.prefill_attention_window(3, c.q.view(3, 1, 4, 64), c.cache, c.map, c.seq_lens - 1, pre, 0)
    assert pre[0].isnan().all()
    assert torch.equal(pre[1, 0], v[0, 1, L - 7].float().expand(4, 64))


@pytest.mark.parametrize("four_bits", [True, False])
def test_caches_beyond_32_bit_offsets(four_bits):
    """The last head and sequence of a cache of more than 2^32 bytes (4-bit) or
    elements a plane (bf16), near the end of a long capacity."""
    D, S, g, B = 128, 1 << 20, 17, 2
    label = f"large {'4-bit' if four_bits else 'bf16'}"
    say(label)
    mp = mlkv.Map.uniform(4, 2 * g, 2, g)
    cache = (mlkv.QCache if four_bits else mlkv.Cache).empty(2 * g, B, S, D)
    n, window, L = 100, 60, S - 3
    shape = (B, n, g, D)
    k, v = synth.normal_bf16(59, 1, shape), synth.normal_bf16(59, 2, shape)
    kd, vd = mlkv.bf16_tensor(k, "cuda"), mlkv.bf16_tensor(v, "cuda")
    ctx = torch.full((B,), L - n, dtype=torch.int32, device="cuda")
    if four_bits:
        mlkv.qcache_append_rows(2, mp, cache, kd, vd, ctx)
        back = cache.read_rows(2 * g - 1, 1, starts=ctx, T=n)
        k, v = serve_ref.held(k), serve_ref.held(v)
        for got, want in zip(back, (k, v)):
            assert np.array_equal(got[0].double().cpu().numpy(), want[:, :, g - 1])
    else:
        mlkv.cache_append_rows(2, mp, cache, kd, vd, ctx, n)
        k, v = serve_ref.f64(k), serve_ref.f64(v)
    q_bits = synth.normal_bf16(59, 3, (B, 2 * g, D))
    q = mlkv.bf16_tensor(q_bits, "cuda")
    out = torch.empty((B, 2 * g, D), dtype=torch.float32, device="cuda")
    ws = mlkv.window_workspace(mp, B, S, D)
    f = mlkv.qcache_decode_attention if four_bits else mlkv.decode_attention_window
    f(3, q, cache, mp, ctx + n, out, window=window, ws=ws)
    outs = [out]
    if not four_bits:
        pre = torch.empty((B, 1, 2 * g, D), dtype=torch.float32, device="cuda")
        mlkv.prefill_attention_window(3, q[:, None].contiguous(), cache, mp, ctx + (n - 1), pre,
                                      window)
        outs.append(pre[:, 0])
    for o in outs:
        o = o.double().cpu().numpy()
        for b in range(B):
            for r in (0, g - 1):
                hs = slice(2 * r, 2 * r + 2)
                ref, bound = serve_ref.attend(serve_ref.f64(q_bits[b, hs]), k[b, :, r], v[b, :, r],
                                              np.arange(n - window, n))
                assert np.all(np.abs(o[b, hs] - ref) <= bound), (label, b, r)


def test_lengths_are_checked_on_request(monkeypatch):
    c = Case(True, 4, 1, 64, [64, 40], 64, 60)
    monkeypatch.setenv("MLKV_CHECK", "1")
    c.decode()
    with pytest.raises(mlkv.MLKVError, match="attends 64 positions, limit 50"):
        c.decode(hint=50)
    rows = torch.zeros((2, 3, 1, 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(mlkv.MLKVError, match="64 cached"):
        mlkv.qcache_append_rows(2, c.map, c.cache, rows, rows, c.seq_lens)


# ------------------------------------------------------------------ prefill ---

@pytest.mark.parametrize("D,h,g", [(64, 12, 1), (128, 8, 2)])
@pytest.mark.parametrize("window,sinks", WINDOWS)
def test_prefill_windows_across_tile_edges(D, h, g, window, sinks):
    T = 45
    label = f"prefill D{D} w{window} s{sinks}"
    say(label)
    c = Case(False, h, g, D, [T, T + 1, T + 31, T + 32, T + 100], 160, 61, T=T, window=window,
             sinks=sinks)
    c.check(c.prefill(), label)


@pytest.mark.parametrize("D,h,g,T,ctx,window,sinks", [
    (64, 12, 12, 70, 33, 20, 2), (64, 24, 1, 2, 200, 64, 4), (64, 40, 1, 9, 10, 7, 0),
    (128, 32, 8, 33, 500, 300, 4), (128, 16, 1, 130, 0, 50, 33), (64, 12, 1, 600, 1000, 257, 4),
    (128, 4, 4, 300, 7, 100, 0)])
def test_prefill_shapes(D, h, g, T, ctx, window, sinks):
    label = f"prefill D{D} h{h} g{g} T{T} ctx{ctx} w{window} s{sinks}"
    say(label)
    S = (ctx + T + 63) // 32 * 32
    c = Case(False, h, g, D, [ctx + T, T], S, 62, k_scale=3.0, T=T, window=window, sinks=sinks)
    out = c.prefill()
    c.check(out, label, tokens=None if T < 200 else range(0, T, 13))
    assert torch.equal(c.prefill(), out)
    assert torch.equal(c.prefill(torch.bfloat16), out.bfloat16())


@pytest.mark.parametrize("D", [64, 128])
def test_prefill_of_one_token_is_a_decode_step(D):
    """T = 1 (and a window longer than the text is the plain prefill)."""
    c = Case(False, 12, 4, D, [300, 77], 320, 63, window=90, sinks=6)
    step = c.decode()
    out = torch.empty((2, 1, 12, D), dtype=torch.float32, device="cuda")
    mlkv.prefill_attention_window(c.layer, c.q.view(2, 1, 12, D), c.cache, c.map, c.seq_lens - 1,
                                  out, window=90, sinks=6)
    c.check(out, "prefill of one")
    c.check(step, "decode of the same")


@pytest.mark.parametrize("D", [64, 128])
def test_prefill_values_that_are_not_finite_reach_only_who_attends_them(D):
    """An infinite and a NaN value at position 50: tokens before it, and tokens
    whose window has passed it, keep their results."""
    T, window, at = 100, 20, 50
    c = Case(False, 4, 1, D, [T], 128, 64, T=T, window=window, sinks=2)
    clean = c.prefill()
    k, v = (t.clone() for t in c.cache.read_rows(1, 1))
    v[0, 0, at, 3] = float("inf")
    v[0, 0, at, 7] = float("nan")
    k[0, 0, 80, 1] = float("nan")  # and a key: scores of its position are NaN
    c.cache.write_rows(k, v, 1)
    out = c.prefill()
    n = torch.arange(T, device="cuda")
    hit_v, hit_k = (n >= at) & (n < at + window), (n >= 80) & (n < 80 + window)
    assert out[0][hit_k].isnan().all()
    rows = out[0][hit_v & ~hit_k]
    assert not rows[..., [3, 7]].isfinite().any()
    others = [d for d in range(D) if d not in (3, 7)]
    want = clean[0][hit_v & ~hit_k][..., others]
    assert torch.allclose(rows[..., others], want, rtol=1e-6, atol=1e-6)
    free = ~hit_v & ~hit_k
    assert torch.allclose(out[0][free], clean[0][free], rtol=1e-6, atol=1e-6)


@pytest.mark.parametrize("seed", range(24))
def test_random_shapes_lengths_and_windows(seed):
    """Seeded draws over heads, groups, batches, ragged lengths, windows, first
    tokens and bounds: decode from either cache, and prefill."""
    rng = np.random.default_rng(1000 + seed)
    kind = ("4-bit", "bf16", "prefill")[seed % 3]
    D = int(rng.choice([64, 128]))
    g = int(rng.choice([1, 2, 3, 5]))
    h = g * int(rng.choice([1, 2, 4, 7, 12, 20]))
    B = int(rng.integers(1, 7))
    most = int(np.exp(rng.uniform(np.log(4), np.log(2500))))
    window = int(rng.choice([0, 1, int(rng.integers(1, most + 1)), int(rng.integers(1, 80))]))
    sinks = int(rng.choice([0, 1, 4, int(rng.integers(0, 100))]))
    T = int(rng.integers(2, 90)) if kind == "prefill" else 1
    lens = T + rng.integers(0, most + 1, B) if T > 1 else rng.integers(0, most + 1, B)
    S = (int(lens.max()) // 32 + int(rng.integers(1, 4))) * 32
    label = f"random {seed} {kind} D{D} h{h} g{g} B{B} T{T} len<={most} w{window} s{sinks}"
    say(label)
    c = Case(kind == "4-bit", h, g, D, lens, S, 2000 + seed, k_scale=float(rng.choice([1, 3])), T=T,
             window=window, sinks=sinks)
    if T > 1:
        c.check(c.prefill(), label, tokens=range(0, T, 5))
    else:
        c.check(c.decode(hint=int(rng.choice([0, max(1, int(lens.max()))]))), label)


@pytest.mark.parametrize("four_bits", [True, False])
def test_windows_and_sinks_beyond_a_c_int(four_bits):
    """They say the same as the capacity; a negative one of any size is refused."""
    c = Case(four_bits, 12, 2, 64, [70, 33], 96, 84)
    want = c.decode()
    for window, sinks in [(2 ** 32 + 5, 0), (5, 2 ** 32), (2 ** 63, 2 ** 31)]:
        c.window, c.sinks = window, sinks
        assert torch.equal(c.decode(), want)
    c.window, c.sinks = 5, 0
    with pytest.raises(mlkv.MLKVError, match="MLKV_ERR_CAPACITY"):
        c.decode(hint=2 ** 32 + 40)
    for window, sinks in [(-2 ** 32 - 1, 0), (-2 ** 32, 0), (5, -2 ** 32)]:
        c.window, c.sinks = window, sinks
        with pytest.raises(mlkv.MLKVError, match="MLKV_ERR_INVALID_ARG"):
            c.decode()


def test_prefill_windows_and_sinks_beyond_a_c_int():
    c = Case(False, 12, 2, 64, [70, 33], 96, 85, T=5)
    want = c.prefill()
    for window, sinks in [(2 ** 32 + 5, 0), (5, 2 ** 32), (2 ** 63, 2 ** 31)]:
        c.window, c.sinks = window, sinks
        assert torch.equal(c.prefill(), want)
    for window, sinks in [(-2 ** 32 - 1, 0), (-2 ** 32, 0), (5, -2 ** 32)]:
        c.window, c.sinks = window, sinks
        with pytest.raises(mlkv.MLKVError, match="MLKV_ERR_INVALID_ARG"):
            c.prefill()


def test_prefill_captured_in_a_graph_follows_the_contexts():
    c = Case(False, 12, 2, 64, [140, 90], 160, 88, T=40, window=33, sinks=2)
    c.cache.k.nan_to_num_(0)
    c.cache.v.nan_to_num_(0)
    out = torch.empty(c.q.shape, dtype=torch.float32, device="cuda")
    ctx = c.seq_lens - c.T
    c.prefill()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mlkv.prefill_attention_window(c.layer, c.q, c.cache, c.map, ctx, out, window=33, sinks=2)
    for lens in ([140, 90], [41, 160], [40, 40], [140, 90]):
        c.seq_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        ctx.copy_(c.seq_lens - c.T)
        out.fill_(7.0)
        graph.replay()
        assert torch.equal(out, c.prefill())

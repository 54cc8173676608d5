"""The long-context operators on the GPU where they are used less often: on
other streams, near the ends of the numbers' range, with odd records and
arguments.  Against the plain 64-bit statement (tests/serve_ref.py)."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import serve_ref  # noqa: E402
import synth  # noqa: E402
from gpu_util import say  # noqa: E402
from test_window_gpu import Case  # noqa: E402

pytestmark = pytest.mark.gpu

mlkv = pytest.importorskip("paper_2406_09297_amd")


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    mlkv.lib()
    yield


@pytest.mark.parametrize("as_handle", [False, True])
@pytest.mark.parametrize("four_bits", [True, False])
def test_split_runs_on_another_stream(four_bits, as_handle):
    """Units of two runs beside units of one, merged on a stream that was never
    used before: every row is written, from counters that were zero, and they are
    zero again.  Of a bare handle the caller orders the fill of `out`."""
    say(f"split runs on another stream four_bits={four_bits} handle={as_handle}")
    lens = [33] * 40 + [3000]
    c = Case(four_bits, 12, 4, 64, lens, 3040, 53, k_scale=3.0)
    want = c.decode(hint=3000)
    assert not c.ws[:262144].any()
    side = torch.cuda.Stream()
    f = mlkv.qcache_decode_attention if four_bits else mlkv.decode_attention_window
    for _ in range(3):
        out = torch.full(c.q.shape, 7.0, device="cuda")
        if as_handle:
            side.wait_stream(torch.cuda.current_stream())
        f(c.layer, c.q, c.cache, c.map, c.seq_lens, out, window=0, max_len_hint=3000, ws=c.ws,
          stream=side.cuda_stream if as_handle else side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(out, want)
        assert not c.ws[:262144].any()


@pytest.mark.parametrize("kind", ["4-bit", "bf16", "prefill"])
@pytest.mark.parametrize("D,power", [(64, 125), (128, 121), (64, 119), (64, -40)])
def test_values_near_the_ends_of_bf16(kind, D, power):
    """Values of up to 1.5 * 2^power, among them rows of zeros, with scores that
    climb by less than the step at which a softmax reference moves: the results
    are finite and within the bound of any other values.  power 125: rows of
    1.5 * 2^126 all alike, whose sum alone leaves fp32."""
    say(f"values near 2^{power}, {kind}, D={D}")
    T = 40 if kind == "prefill" else 1
    c = Case(kind == "4-bit", 4, 1, D, [300, 200], 320, 91, T=T)
    g = np.random.default_rng(abs(power))
    shape = (1, 2, 320, D)
    # Scores q.k / sqrt(D) of 0 .. 5 (7.2 in log2): channel 0 climbs with the position.
    k = np.zeros(shape, np.float32)
    k[..., 0] = np.linspace(0, 5 * np.sqrt(D), 320)[None, None]
    k[..., 1:] = g.normal(0, 0.01, (1, 2, 320, D - 1))
    v = g.uniform(0.5, 1.5, shape) * np.where(g.random(shape) < 0.5, -1, 1)
    v[:, :, ::7] = 0
    v[0, 1] = 1.5 if power != 125 else 3.0
    k, v = synth.f32_to_bf16(k), synth.f32_to_bf16(np.ldexp(v, power).astype(np.float32))
    q = synth.bf16_to_f32(c.q_bits).copy()
    q[..., 0] = 1.0
    c.q_bits = synth.f32_to_bf16(q)
    c.q = mlkv.bf16_tensor(c.q_bits, "cuda")
    c.cache.write_rows(mlkv.bf16_tensor(k, "cuda"), mlkv.bf16_tensor(v, "cuda"), 1)
    held = serve_ref.held if kind == "4-bit" else serve_ref.f64
    c.k, c.v = held(k), held(v)
    c.check(c.prefill() if T > 1 else c.decode(), f"values near 2^{power}")


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("lens", [[70, 70, 70], [3000, 3000, 3000]])
def test_an_exponent_byte_of_255_is_nan_whatever_its_codes(D, lens):
    """Records from elsewhere may keep codes beside the mark: a value block's
    channels become NaN, a key block makes its whole row so, and nothing else
    changes; read_rows says the same."""
    say(f"exponent byte 255, D={D}, {lens}")
    c = Case(True, 4, 1, D, lens, (lens[0] + 63) // 32 * 32, 92)
    clean = c.decode()
    at = lens[0] - 9
    *_, ke, ve = serve_ref.places(D)
    c.cache.data[1, 0, at // 32, int(ve[at % 32, 1])] = 255
    c.cache.data[1, 1, at // 32, int(ke[at % 32, 0])] = 255
    k, v = c.cache.read_rows(1, 1)
    assert v[0, 0, at, 32:64].isnan().all() and k[0, 1, at, :32].isnan().all()
    out = c.decode()
    assert out[0][:, 32:64].isnan().all()
    rest = [d for d in range(D) if not 32 <= d < 64]
    assert torch.equal(out[0][:, rest], clean[0][:, rest])
    assert out[1].isnan().all() and torch.equal(out[2], clean[2])
    bf16 = c.decode(torch.bfloat16)
    assert torch.equal(bf16.isnan(), out.isnan())


@pytest.mark.parametrize("four_bits", [True, False])
def test_layers_heads_and_dims_beyond_a_c_int_are_refused(four_bits):
    """They would be another number as a C int, one that is allowed."""
    say(f"numbers beyond a C int, four_bits={four_bits}")
    c = Case(four_bits, 4, 1, 64, [40, 33], 64, 93)
    before = (c.cache.data if four_bits else c.cache.k).clone()
    q, out = c.q.view(2, 1, 4, 64), torch.empty_like(c.q)
    new = torch.ones((2, 1, 1, 64), dtype=torch.bfloat16, device="cuda")
    rows = torch.ones((1, 2, 64, 64), dtype=torch.bfloat16, device="cuda")
    for far in (2 ** 32, -2 ** 32):
        calls = [lambda: mlkv.norm_rope_append(2, c.map, c.cache, q, new, new, c.seq_lens - 1,
                                               out.view(2, 1, 4, 64), rotary_dims=16 + far)]
        c.layer = 3 + far
        calls.append(c.decode)
        if four_bits:
            calls += [lambda: c.cache.write_rows(rows, rows, 1 + far),
                      lambda: c.cache.read_rows(1 + far, 1),
                      lambda: c.cache.read_rows(1, 0, T=5 + 2 ** 32)]
        else:
            calls.append(lambda: mlkv.prefill_attention_window(
                3 + far, q, c.cache, c.map, c.seq_lens - 1, out.view(2, 1, 4, 64), 8))
        for call in calls:
            with pytest.raises(mlkv.MLKVError):
                call()
    assert torch.equal(before.view(torch.uint8),
                       (c.cache.data if four_bits else c.cache.k).view(torch.uint8))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("eps,powers", [(1e-50, (-80, -100, None, 0)), (1e-42, (-70, None, -100, 5)),
                                        (1e39, (60, 100, 0, None)), (1e60, (100, 120, 20, None))])
def test_norms_whose_eps_leaves_fp32(D, eps, powers):
    """Rows of about 2^power (None: zeros, which stay zeros) beside an eps that
    fp32 holds as a subnormal number, as 0 or as inf."""
    say(f"norm with eps {eps}, D={D}")
    h, B = 3, len(powers)
    f = synth.bf16_to_f32(synth.normal_bf16(94, 0, (B, 1, h, D)))
    f = np.where(np.abs(f) < 2.0 ** -6, np.float32(2.0 ** -6), f)
    f = np.stack([np.zeros_like(x) if n is None else np.ldexp(x, n) for x, n in zip(f, powers)])
    bits = synth.f32_to_bf16(f.astype(np.float32))
    w = synth.f32_to_bf16((1 + 0.1 * synth.bf16_to_f32(synth.normal_bf16(94, 9, (D,)))))
    mp = mlkv.Map.uniform(2, h, 1, 1)
    cache = mlkv.Cache.empty(1, B, 32, D)
    q_out = torch.empty((B, 1, h, D), dtype=torch.bfloat16, device="cuda")
    ctx = np.arange(B, dtype=np.int32)
    mlkv.norm_rope_append(1, mp, cache, mlkv.bf16_tensor(bits, "cuda"), None, None,
                          torch.from_numpy(ctx).cuda(), q_out, q_norm=mlkv.bf16_tensor(w, "cuda"),
                          eps=eps, rotary_dims=32)
    ref, bound = serve_ref.norm_rope(bits, w, eps, 32, 10000.0, ctx[:, None])
    d = np.abs(q_out.double().cpu().numpy() - ref)
    assert np.all(d <= bound), [(n, float((d[i] - bound[i]).max())) for i, n in enumerate(powers)]

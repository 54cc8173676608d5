"""The tests' statement of the 4-bit cache against itself (CPU)."""
import numpy as np
import pytest

import serve_ref
import synth


@pytest.mark.parametrize("D", [64, 128])
def test_record_places_are_disjoint_and_fill_it(D):
    kb, kn, vb, vn, ke, ve = serve_ref.places(D)
    nibbles = set(zip((2 * kb + kn).ravel().tolist(), ["c"] * kb.size))
    nibbles |= set(zip((2 * vb + vn).ravel().tolist(), ["c"] * vb.size))
    assert len(nibbles) == 2 * 32 * D and max(n for n, _ in nibbles) == 64 * D - 1
    exps = np.concatenate([ke.ravel(), ve.ravel()])
    assert sorted(exps.tolist()) == list(range(32 * D, 34 * D))


@pytest.mark.parametrize("D", [64, 128])
def test_store_then_load_gives_the_values_held(D):
    bits = synth.normal_bf16(5, 0, (2, 2, 3, 64, D))
    data = np.full((3, 2, 2, 34 * D), 0xA5, np.uint8)
    for kv in range(3):
        for b in range(2):
            serve_ref.store(data, kv, b, 0, bits[0, b, kv], bits[1, b, kv])
    k, v = serve_ref.load(data)
    for got, src in ((k, bits[0]), (v, bits[1])):
        assert np.array_equal(got, serve_ref.held(src.transpose(1, 0, 2, 3)))


def test_quantisation_rounds_by_half_a_step_and_is_idempotent():
    rng = np.random.default_rng(1)
    x = (rng.standard_normal((200, 32)) * 10.0 ** rng.uniform(-20, 20, (200, 1))).astype(np.float32)
    bits = synth.f32_to_bf16(x)
    codes, exps = serve_ref.quantise(bits)
    got, src = serve_ref.values(codes, exps), serve_ref.f64(bits)
    step = 2.0 ** (exps.astype(np.float64) - 127)
    mag = np.abs(src) / step
    half = np.where(mag < 2, 0.25, np.where(mag < 4, 0.5, 1.0)) * step
    assert np.all(np.abs(got - src) <= half)
    again = synth.f32_to_bf16(got.astype(np.float32))
    assert np.array_equal(synth.bf16_to_f32(again).astype(np.float64), got)
    codes2, exps2 = serve_ref.quantise(again)
    assert np.array_equal(codes2, codes) and np.array_equal(exps2, exps)


def test_attended_positions():
    assert serve_ref.attended(-1, 3, 2).size == 0
    assert serve_ref.attended(4, 0, 2).tolist() == [0, 1, 2, 3, 4]
    assert serve_ref.attended(9, 3, 2).tolist() == [0, 1, 7, 8, 9]
    assert serve_ref.attended(3, 3, 2).tolist() == [0, 1, 2, 3]
    assert serve_ref.attended(9, 1, 0).tolist() == [9]

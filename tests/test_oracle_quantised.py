"""Pins of the oracle of the 8-bit cache and its rotary positions: torch's e4m3 and e8m0, closed forms, invariants,
finite differences of the rotation."""

import math

import numpy as np
import pytest
import torch

import oracle as O
from oracle import quantised_oracle as Q


def test_every_code_has_torchs_value_and_every_value_its_code():
    codes = np.arange(256, dtype=np.uint8)
    want = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    got = Q.e4m3_value(codes)
    assert np.array_equal(got, want, equal_nan=True)
    finite = codes[(codes & 127) != 127]
    assert np.array_equal(Q.e4m3_code(Q.e4m3_value(finite)), finite)


def test_codes_round_as_torch_does():
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.uniform(-448, 448, 20000), rng.standard_normal(20000) * 2.0 ** rng.integers(-14, 8, 20000)])
    grid = Q.e4m3_value(np.arange(127))
    x = np.concatenate([x, (grid[1:] + grid[:-1]) / 2, -(grid[1:] + grid[:-1]) / 2]).astype(np.float32)   # ties
    x = x[np.abs(x) <= 448]
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(Q.e4m3_code(x), want)


def test_scale_is_the_least_power_that_holds_the_block():
    for top, e in ((448.0, 0), (448.0 * (1 + 2 ** -7), 1), (449.0, 1), (1.0, -8), (1.75, -8), (1.7500001, -7), (0.0, -124),
                   (2.0 ** -133, -124), (1.9296875 * 2.0 ** 127, 120)):
        x = np.zeros((1, 128), dtype=np.float32)
        x[0, 32:64] = top
        codes, b = Q.quantise(x)
        assert b[0, 1] == e + 127 and b[0, 0] == 3, (top, e, b)
        assert top <= 448.0 * 2.0 ** (int(b[0, 1]) - 127)
        assert abs(Q.decode(codes, b)[0, 40] - np.float32(top)) <= max(top * 2.0 ** -4, 2.0 ** -134)


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf, 1.9375 * 2.0 ** 127])
def test_a_block_that_is_not_finite_reads_as_nan_and_leaves_the_others(bad):
    x = np.ones((2, 128), dtype=np.float32)
    x[1, 70] = bad
    codes, b = Q.quantise(x)
    v = Q.decode(codes, b)
    assert np.isnan(v[1, 64:96]).all() and (v[1, :64] == 1).all() and (v[1, 96:] == 1).all() and (v[0] == 1).all()


def test_decoded_values_are_bf16_and_off_by_half_a_step():
    rng = np.random.default_rng(1)
    x = (rng.standard_normal((500, 128)) * 2.0 ** rng.integers(-130, 120, (500, 1))).astype(np.float32)
    codes, b = Q.quantise(x)
    v = Q.decode(codes, b)
    back = O.bf16_bits_to_f32(O.f32_to_bf16_bits_rne(v.astype(np.float32)))
    assert np.array_equal(back.astype(np.float64), v)
    step = np.repeat(np.exp2(b.astype(np.float64) - 127.0), 32, axis=-1) * 2.0 ** -10
    assert (np.abs(v - x) <= np.maximum(np.abs(x.astype(np.float64)) * 2.0 ** -4, step)).all()


def test_plain_rotary_is_the_table_and_rotation_of_the_path():
    bands, rope = (44, 42, 42), Q.Rope()
    c, s = Q.rotary_table(5, 2, 3, 4, bands, rope)
    oc, os_ = O.rope_table(5, 2, 3, 4)
    assert np.array_equal(c, oc) and np.array_equal(s, os_)
    bits = O.f32_to_bf16_bits_rne(np.random.default_rng(2).standard_normal((24, 3, 128)).astype(np.float32))
    assert np.array_equal(Q.rotary_apply(bits, c, s, False), O.rope_rotate(bits, oc, os_))


def test_halves_are_interleaved_pairs_in_another_order():
    c, s = Q.rotary_table(7, 1, 2, 3, (32, 32, 32), Q.Rope())
    x = np.random.default_rng(3).standard_normal((6, 2, 128)).astype(np.float32)
    order = np.concatenate([np.stack([np.arange(48), 48 + np.arange(48)], axis=1).reshape(-1), np.arange(96, 128)])
    a = Q.rotate_f32(x, c, s, True)
    b = Q.rotate_f32(x[..., order], c, s, False)
    assert np.array_equal(a[..., order], b) and np.array_equal(a[..., 96:], x[..., 96:])


def test_scaled_frequencies():
    bands = (64, 32, 32)
    plain, axis = Q.rotary_frequencies(bands, Q.Rope())
    inter, _ = Q.rotary_frequencies(bands, Q.Rope(factor=(4.0, 1.0, 2.0)))
    assert np.allclose(inter[axis == 0] * 4, plain[axis == 0], rtol=1e-15)
    assert np.array_equal(inter[axis == 1], plain[axis == 1])
    assert np.allclose(inter[axis == 2] * 2, plain[axis == 2], rtol=1e-15)
    parts, _ = Q.rotary_frequencies(bands, Q.Rope(factor=(4.0, 1.0, 1.0), trained=(21, 0, 0), beta=(1.0, 3.0)))
    turns = 21 * plain[axis == 0] / (2 * math.pi)
    ratio = parts[axis == 0] / plain[axis == 0]
    assert np.allclose(ratio[turns >= 3.0], 1.0) and np.allclose(ratio[turns <= 1.0], 0.25)
    between = (turns > 1.0) & (turns < 3.0)
    assert between.any() and ((ratio[between] > 0.25) & (ratio[between] < 1.0)).all()
    c, s = Q.rotary_table(3, 1, 2, 2, bands, Q.Rope(magnitude=1.5))
    assert np.allclose(c.astype(np.float64) ** 2 + s.astype(np.float64) ** 2, 2.25, rtol=1e-6)


@pytest.mark.parametrize("half", [False, True])
def test_the_transpose_is_the_backward_pass(half):
    # float32 throughout: the rotation is linear, so a difference of steps of a power of two has only the rounding of
    # its terms, 2^-24 of values up to 8 for each of six operations
    rng = np.random.default_rng(4)
    c, s = Q.rotary_table(9, 1, 1, 1, (32, 8, 8), Q.Rope(half=half, magnitude=1.25))
    x, g = rng.standard_normal((1, 1, 128)), rng.standard_normal((1, 1, 128))
    grad = Q.rotate_f32(g, c, s, half, transposed=True).astype(np.float64)[0, 0]
    for i in range(128):
        d = np.zeros_like(x)
        d[..., i] = 0.5
        up, down = (Q.rotate_f32(x + e, c, s, half).astype(np.float64) for e in (d, -d))
        assert abs((g * (up - down)).sum() - grad[i]) <= 128 * 6 * 8 * 2.0 ** -24
    plain_c, plain_s = Q.rotary_table(9, 1, 1, 1, (32, 8, 8), Q.Rope(half=half))
    back = Q.rotate_f32(Q.rotate_f32(x, plain_c, plain_s, half), plain_c, plain_s, half, transposed=True)
    assert np.abs(back - x).max() < 1e-6


def test_append_read_and_attention_of_a_wrapped_cache():
    state = Q.QuantState(1, 1, 2, 3, 2)
    rng = np.random.default_rng(5)
    written = {}
    for p in range(6):
        q, k, v = (O.f32_to_bf16_bits_rne(rng.standard_normal((1, 3, 2, 128)).astype(np.float32)) for _ in range(3))
        c, s = Q.rotary_table(p, 1, 1, 3, (44, 42, 42), Q.Rope())
        q_out = Q.kv_append(state, [p], q, k, v, c, s, False)
        assert np.array_equal(q_out, O.rope_rotate(q, c, s))
        written[p] = Q.decode(*Q.quantise(Q.rotate_f32(O.bf16_bits_to_f32(k), c, s, False)))[0]
    for p in (0, 4, 5):
        k, _ = Q.kv_frames(state, 0, [p])
        assert np.array_equal(k[0], written[p])
    out = Q.window_attn_q8(state, [5], 2, 1, q_out, 1)
    ks, vs = Q.kv_frames(state, 0, [0, 4, 5])
    z = np.einsum("d,md->m", O.bf16_bits_to_f32(q_out)[0, 2, 1].astype(np.float64), ks[:, :, 1].reshape(-1, 128)) / math.sqrt(128)
    w = np.exp(z - z.max())
    assert np.allclose(out[0, 2, 1], (w @ vs[:, :, 1].reshape(-1, 128)) / w.sum(), rtol=1e-12)

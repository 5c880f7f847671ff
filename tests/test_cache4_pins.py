"""Pins of the 4-bit cache oracle: hand-worked groups, the scale rule against its
definition, the error of a rounding, and the attention against the bf16 cache's
oracle."""
import numpy as np
import pytest

import oracle
from paper_2502_12085_amd import inputs


def _bits(x):
    return inputs.f32_to_bf16_bits(np.asarray(x, dtype=np.float32))


def _group(*head):
    return _bits(np.array(list(head) + [0.0] * (32 - len(head)), dtype=np.float32))


def _codes(group):
    packed, scale = oracle.quantise4_ref(group)
    return [int(c) for b in packed for c in (b & 15, b >> 4)], int(scale[0])


@pytest.mark.parametrize("head,codes,b", [
    # the levels themselves, under a scale of 1
    ((0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0), [0, 1, 2, 3, 4, 5, 6, 7], 127),
    ((-0.5, -6.0, -0.0), [9, 15, 8], 127),
    # ties go to the even code: 0.25 -> 0, 0.75 -> 1, 1.25 -> 1, 1.75 -> 2, 2.5 -> 2,
    # 3.5 -> 4, 5 -> 4; 7 stays under this scale and becomes 6
    ((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0), [0, 2, 2, 4, 4, 6, 6, 7], 127),
    ((-0.25,), [14], 123),           # alone it is 4 / 16 (code 6): the scale follows it
    ((7.03125,), [6], 128),          # the next bf16 past 7: twice the scale, 3.52 -> 4
    ((3.5, 0.25), [7, 1], 126),      # 3.5 = 7 / 2; 0.25 = 0.5 / 2
    ((1.0,), [6], 125),              # 4 * 2^-2
    ((0.0,), [0], 7),                # nothing but zeros: the smallest scale
    ((2.0 ** -126,), [0], 7),        # 2^-6 of the smallest scale: zero
    ((2.0 ** -121,), [1], 7),        # half of it
    ((2.0 ** 127,), [6], 252),       # 4 * 2^125
    ((3.3895e38,), [7], 252),        # bf16's largest, 7.97 * 2^125: 6
    ((float("inf"), 1.0), [0, 0], 255),
    ((1.0, float("nan")), [0, 0], 255),
])
def test_groups_by_hand(head, codes, b):
    got, scale = _codes(_group(*head))
    assert scale == b
    assert got[:len(codes)] == codes
    assert not any(c & 7 for c in got[len(codes):])


def test_scale_is_the_smallest_that_holds():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((400, 32)) * np.exp2(rng.integers(-110, 110, (400, 1)))
    bits = _bits(x)
    top = np.abs(oracle.apb_oracle.bf16_to_f64(bits)).max(-1)
    _, b = oracle.quantise4_ref(bits)
    e = b[:, 0].astype(np.float64) - 127
    assert np.all(top <= 7 * np.exp2(e)) and np.all(top > 7 * np.exp2(e - 1))


def test_error_is_at_most_half_a_step():
    # of N(0, 1): between magnitudes m and the next the error is half their
    # distance; relative to the scale 0.25 below 2, 0.5 below 4, 1 up to 7
    bits = _bits(np.random.default_rng(4).standard_normal((2000, 64)))
    x = oracle.apb_oracle.bf16_to_f64(bits)
    codes, scales = oracle.quantise4_ref(bits)
    back = oracle.values4_ref(codes, scales)
    by = np.repeat(np.exp2(scales.astype(np.float64) - 127), 32, -1)
    half = np.where(np.abs(x) <= 2 * by, 0.25, np.where(np.abs(x) <= 4 * by, 0.5, 1.0)) * by
    assert np.all(np.abs(back - x) <= half)
    snr = 10 * np.log10((x ** 2).mean() / ((back - x) ** 2).mean())
    assert 18.5 < snr < 19.5
    # what was read back is held as it is
    again = oracle.quantise4_ref(_bits(back))
    assert np.array_equal(oracle.values4_ref(*again), back)


def test_values_by_hand():
    codes = np.zeros((1, 32), np.uint8)
    codes[0, 0], codes[0, 16] = 0x21, 0xF9  # elements 0, 1 = 0.5, 1; 32, 33 = -0.5, -6
    v = oracle.values4_ref(codes, np.array([[128, 126]], np.uint8))
    assert v[0, 0] == 1.0 and v[0, 1] == 2.0 and v[0, 32] == -0.25 and v[0, 33] == -3.0
    assert np.count_nonzero(v) == 4
    v = oracle.values4_ref(codes, np.array([[255, 126]], np.uint8))
    assert np.isnan(v[0, :32]).all() and v[0, 33] == -3.0


@pytest.mark.parametrize("causal", [0, 1])
def test_attention_is_that_of_the_values(causal):
    case = inputs.make_decode_case(8, 2, 64, [50], 5, seed=2)
    kc, vc = case["caches"][0]
    k = np.concatenate([kc, case["k_new"]], 1)
    v = np.concatenate([vc, case["v_new"]], 1)
    kv = oracle.values4_ref(*oracle.quantise4_ref(k))
    vv = oracle.values4_ref(*oracle.quantise4_ref(v))
    o, lse, pv, qk = oracle.decode4_ref(case["q"], kv, vv, causal=causal, bound=True)
    if causal:
        ro, rl = oracle.decode_attention_ref(case["q"], _bits(kv[:, :50]), _bits(vv[:, :50]),
                                             _bits(kv[:, 50:]), _bits(vv[:, 50:]))
    else:
        ro, rl = oracle.decode_attention_ref(case["q"], _bits(kv), _bits(vv))
    assert np.abs(o - ro).max() < 1e-12 and np.abs(lse - rl).max() < 1e-12
    assert np.all(pv >= np.abs(o) - 1e-12) and np.all(qk > 0)


def test_attention_without_keys():
    q = _bits(np.ones((2, 3, 64)))
    o, lse = oracle.decode4_ref(q, np.zeros((1, 0, 64)), np.zeros((1, 0, 64)), causal=0)
    assert not o.any() and np.all(lse == -np.inf)

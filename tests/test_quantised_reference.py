"""CPU pins of the 4-bit cache's reference: scales, codes and layout against the definition and by brute force."""
from fractions import Fraction

import numpy as np
import pytest

from oracle import quantised_cache_reference as qref
from paper_2403_02310_amd import workloads as wl

GRID = [Fraction(0), Fraction(1, 2), Fraction(1), Fraction(3, 2), Fraction(2), Fraction(3), Fraction(4), Fraction(6)]


def _rows(seed, shape, spread=0.0):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal(shape) * np.exp(spread * rng.standard_normal(shape))
    return wl.f32_to_bf16_bits(x.astype(np.float32))


def _fraction_code(x: Fraction, unit: Fraction) -> int:
    far = [abs(abs(x) - m * unit) for m in GRID]
    best = [i for i in range(8) if far[i] == min(far)]
    return next((i for i in best if i % 2 == 0), best[0])


@pytest.mark.parametrize("spread", [0.0, 3.0])
def test_codes_and_scales_against_exact_fractions(spread):
    bits = _rows(1, (6, 64), spread)
    x = qref._f64(bits)
    code, byte = qref.quantise_keys(bits)
    v_code, v_scale = qref.quantise_values(bits)
    for t in range(6):
        for b in range(2):
            top = max(abs(Fraction(float(v))) for v in x[t, 32 * b:32 * b + 32])
            e = int(byte[t, b]) - 127
            assert top <= 6 * Fraction(2) ** e and (e == qref.LOWEST or top > 6 * Fraction(2) ** (e - 1))
            for c in range(32 * b, 32 * b + 32):
                assert int(code[t, c]) & 7 == _fraction_code(Fraction(float(x[t, c])), Fraction(2) ** e)
        top, s = max(abs(Fraction(float(v))) for v in x[t]), Fraction(float(v_scale[t]))
        m = s
        while m >= 16:
            m /= 2
        while m < 8:
            m *= 2
        assert m.denominator == 1                                     # four significant bits
        below = s * (m - 1) / m if m > 8 else s * Fraction(15, 16)    # the next smaller scale
        assert top <= 6 * s and top > 6 * below
        for c in range(64):
            assert int(v_code[t, c]) & 7 == _fraction_code(Fraction(float(x[t, c])), s)


def test_ties_go_to_even_codes_and_large_numbers_to_six():
    x = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -0.25, -5.0, 6.0, 0.0, -0.0] + [0.0] * 20)
    code, byte = qref.quantise_keys(wl.f32_to_bf16_bits(x.astype(np.float32)[None]))
    assert byte[0, 0] == 127 and code[0, :12].tolist() == [0, 2, 2, 4, 4, 6, 6, 8, 14, 7, 0, 8]
    top = np.full((1, 32), 3.0e38, np.float32)
    code, byte = qref.quantise_keys(wl.f32_to_bf16_bits(top))
    assert byte[0, 0] == qref.HIGHEST + 127 and (code == 7).all()
    code, scale = qref.quantise_values(wl.f32_to_bf16_bits(top))
    assert scale[0] == np.float32(2.0 ** qref.HIGHEST) and (code == 7).all()
    code, scale = qref.quantise_values(np.zeros((1, 64), np.uint16))
    assert scale[0] == np.float32(2.0 ** qref.LOWEST) and (code == 0).all()


def test_infinities_and_nan_mark_their_block_and_their_position():
    k = _rows(2, (3, 2, 128))
    k[1, 0, 40] = 0x7F80
    k[2, 1, 127] = 0x7FC1
    got, _ = qref.stands_for(k, k)
    nan = np.isnan(qref._f64(got))
    assert nan[1, 0, 32:64].all() and nan[2, 1, 96:].all() and nan.sum() == 64
    _, got = qref.stands_for(k, k)
    nan = np.isnan(qref._f64(got))
    assert nan[1, 0].all() and nan[2, 1].all() and nan.sum() == 256


def test_no_value_is_further_than_half_its_step():
    """Steps are 1/2, 1 and 2 units below 2, below 4 and below 6 units: off by a quarter of a unit, a half and one at most."""
    bits = _rows(3, (200, 1, 128), 1.0)
    x = qref._f64(bits)
    k, v = (qref._f64(b) for b in qref.stands_for(bits, bits))
    unit = np.repeat(np.exp2(qref.quantise_keys(bits)[1].astype(float) - 127), 32, axis=-1)
    scale = qref.quantise_values(bits)[1].astype(float)[..., None]
    for y, u in ((k, unit), (v, np.broadcast_to(scale, x.shape))):
        a = np.abs(x) / u
        assert (np.abs(y - x) <= np.where(a <= 2, 0.25, np.where(a <= 4, 0.5, 1.0)) * u).all()


@pytest.mark.parametrize("d", [64, 128])
def test_places_cover_a_record_once_and_reading_undoes_appending(d):
    half = set()
    for at, shift in (qref.key_places(d), qref.value_places(d)):
        half |= set(zip(at.ravel().tolist(), shift.ravel().tolist()))
    assert half == {(b, s) for b in range(16 * d) for s in (0, 4)}
    rng = np.random.default_rng(4)
    pool = rng.integers(0, 256, (9, 2, qref.record_bytes(d)), dtype=np.uint8)
    before = pool.copy()
    table, q_len, ctx = [[3, 5, -1], [7, 0, 2], [8, -1, -1]], [20, 1, 3], [25, 33, 3]
    k, v = _rows(5, (24, 2, d)), _rows(6, (24, 2, d))
    qref.append(pool, k, v, table, [0, 20, 21], q_len, ctx)
    got = qref.read(pool, table, q_len, ctx, d)
    for a, b in zip(got, qref.stands_for(k, v)):
        assert (qref._f64(a) == qref._f64(b)).all()
    assert (pool[[0, 1, 4, 6, 7]] == before[[0, 1, 4, 6, 7]]).all()      # pages without a new position
    old, new = (qref.held_page(p[8], d) for p in (before, pool))
    for a, b in zip(old, new):
        np.testing.assert_array_equal(a[:, 3:], b[:, 3:])                # slots behind the last row


@pytest.mark.parametrize("mutant,fails", [
    ("truncate", True), ("odd_ties", True), ("double_scale", True), ("swapped_halves", True), ("none", False)])
def test_planted_mistakes_are_caught(mutant, fails, monkeypatch):
    """Mistakes in the reference itself trip the pins above."""
    if mutant == "truncate":
        monkeypatch.setattr(qref, "nearest_code", lambda x, s: (np.searchsorted(qref.MAGNITUDES, np.abs(x) / s, side="right") - 1 + 8 * np.signbit(x)).astype(np.uint8))
    elif mutant == "odd_ties":
        def odd(x, s):
            far = np.abs(np.abs(x)[..., None] - qref.MAGNITUDES * s[..., None])
            order = np.array([1, 3, 5, 7, 0, 2, 4, 6])
            return (order[np.argmin(far[..., order], axis=-1)] + 8 * np.signbit(x)).astype(np.uint8)
        monkeypatch.setattr(qref, "nearest_code", odd)
    elif mutant == "double_scale":
        plain = qref.smallest_scale
        monkeypatch.setattr(qref, "smallest_scale", lambda t, s: plain(2 * t, s))
    elif mutant == "swapped_halves":
        plain_places = qref.value_places
        monkeypatch.setattr(qref, "value_places", lambda d: (plain_places(d)[0], plain_places(d)[1] % 4))
    caught = False
    for check in (lambda: test_codes_and_scales_against_exact_fractions(0.0), test_ties_go_to_even_codes_and_large_numbers_to_six,
                  test_no_value_is_further_than_half_its_step, lambda: test_places_cover_a_record_once_and_reading_undoes_appending(64)):
        try:
            check()
        except AssertionError:
            caught = True
    assert caught == fails

"""The 4-bit format's oracle against its definition."""
import math

import numpy as np
import pytest

from oracle import fp4 as F


def test_values_of_the_codes():
    assert F.TABLE.tolist() == [0, .5, 1, 1.5, 2, 3, 4, 6, -0.0, -.5, -1, -1.5, -2, -3, -4, -6]
    assert math.isnan(F.scale_value(255)) and F.scale_value(127) == 1.0 and F.scale_value(0) == 2.0 ** -127


def test_every_stored_value_stores_itself():
    for byte in (2, 100, 127, 130, 252):
        block = np.tile(F.TABLE, 2) * F.scale_value(byte)
        codes, scales = F.encode(block)
        assert scales.tolist() == [byte]
        assert np.array_equal(F.decode(codes, scales), block)


def test_ties_go_to_the_even_code_and_nothing_is_off_by_more_than_half_a_step():
    block = np.zeros(32)
    block[:10] = [6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 7, -5]
    block[0] = 7.0                                  # exactly 1.75 * 4: scale 1
    codes, scales = F.encode(block)
    assert scales[0] == 127
    assert F.TABLE[codes[:10]].tolist() == [6, 0, 1, 1, 2, 2, 4, 4, 6, -4]
    block[0] = np.nextafter(7.0, 8.0)               # above: scale 2
    assert F.encode(block)[1][0] == 128
    rng = np.random.default_rng(0)
    x = rng.standard_normal((200, 32)) * np.exp2(rng.integers(-20, 20, (200, 1)))
    codes, scales = F.encode(x)
    step = np.array([F.scale_value(s) for s in scales[:, 0]])[:, None]
    y = F.decode(codes, scales)
    half = np.where(np.abs(y) >= 4 * step, step, np.where(np.abs(y) >= 2 * step, 0.5 * step, 0.25 * step))
    assert (np.abs(x - y) <= np.maximum(half, 0.25 * step)).all()
    assert (np.abs(x) <= 7.0 * step).all() and (np.abs(x).max(1) > 3.5 * step[:, 0] * 0.999).all()


def test_special_values():
    block = np.zeros(32)
    assert F.encode(block)[1][0] == 2
    block[3] = np.inf
    block[4] = -1e30
    codes, scales = F.encode(block)
    assert scales[0] == 252 and F.decode(codes, scales)[3] == 6 * 2.0 ** 125 and F.decode(codes, scales)[4] == 0.0
    block[5] = np.nan
    codes, scales = F.encode(block)
    assert scales[0] == 255 and np.isnan(F.decode(codes, scales)).all()


@pytest.mark.parametrize("bs,D", [(8, 64), (16, 128), (24, 64), (64, 128)])
@pytest.mark.parametrize("which", ["k", "v"])
def test_a_page_is_a_permutation_of_its_codes_and_scales(which, bs, D):
    places = {(F.code_byte(which, s, d, bs, D), d % 2) for s in range(bs) for d in range(D)}
    assert len(places) == bs * D and {p[0] for p in places} == set(range(bs * D // 2))
    scales = {F.scale_at(which, s, d, bs, D) for s in range(bs) for d in range(D)}
    assert scales == set(range(bs * D // 2, F.page_bytes(bs, D)))
    # two codes of a byte share a scale
    assert all(F.scale_at(which, s, d, bs, D) == F.scale_at(which, s, d + 1, bs, D) for s in range(bs) for d in range(0, D, 2))
    rng = np.random.default_rng(1)
    page = np.zeros(F.page_bytes(bs, D), np.uint8)
    codes, scales = F.encode(rng.standard_normal((bs, D)))
    for s in rng.permutation(bs):
        F.put_row(page, which, s, codes[s], scales[s], bs)
    assert np.array_equal(F.decode_pages(page[None, None], which, bs, D)[0, 0], F.decode(codes, scales))

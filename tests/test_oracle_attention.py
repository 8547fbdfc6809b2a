"""The oracle of the attention operators against definitions worked out another way."""
import itertools
import math

import numpy as np
import pytest

from oracle import attention as oa


def test_codes_are_the_nearest_with_ties_to_even():
    # every threshold between neighbours, hit exactly and from both sides
    expect = {0.25: 0, 0.75: 2, 1.25: 2, 1.75: 4, 2.5: 4, 3.5: 6, 5.0: 6}
    for mid, code in expect.items():
        x = np.zeros(32)
        x[0], x[1], x[2], x[3] = 6.0, mid, mid * (1 - 1e-9), mid * (1 + 1e-9)
        byte, c = oa.quantise_group(x)
        assert byte == 127 and c[0] == 7
        below = int(np.flatnonzero(oa.MAGNITUDES < mid)[-1])
        assert c[1] == code and c[2] == below and c[3] == below + 1


@pytest.mark.parametrize("top,e", [(6.0, 0), (7.0, 0), (np.nextafter(7.0, 8), 1), (3.5, -1), (3.6, 0), (14.0, 1), (1e-30, None)])
def test_scale_is_the_smallest_that_holds(top, e):
    x = np.zeros(32)
    x[5] = -top
    byte, c = oa.quantise_group(x)
    got = byte - 127
    assert top <= 7.0 * 2.0 ** got and top > 7.0 * 2.0 ** (got - 1)
    assert e is None or got == e
    assert c[5] >= 8 and (c[np.arange(32) != 5] == 0).all()


def test_scale_floor_and_non_finite():
    assert oa.quantise_group(np.zeros(32))[0] == 1
    assert oa.quantise_group(np.full(32, 1e-44))[0] == 1
    for bad in (np.nan, np.inf, -np.inf):
        x = np.ones(32)
        x[31] = bad
        byte, c = oa.quantise_group(x)
        assert byte == 255 and (c == 0).all()
        assert np.isnan(oa.value_of(byte, c)).all()


@pytest.mark.parametrize("D", [32, 64, 96, 128, 160, 256])
def test_tile_round_trip(D):
    rng = np.random.default_rng(D)
    tile = np.zeros(oa.tile_bytes(D), dtype=np.uint8)
    rows = {}
    for token, value in itertools.product((0, 1, 37, 63), (False, True)):
        x = rng.normal(size=D) * 10.0 ** rng.integers(-3, 4)
        oa.put(tile, D, value, token, x)
        rows[token, value] = x
    for (token, value), x in rows.items():
        y = oa.get(tile, D, value, token)
        for g in range(D // 32):
            part, held = x[32 * g:32 * g + 32], y[32 * g:32 * g + 32]
            unit = 2.0 ** (oa.quantise_group(part)[0] - 127)
            assert np.abs(part - held).max() <= 1.0 * unit          # half the widest gap, 4 to 6; 6 to 7
            byte, codes = oa.quantise_group(held)                    # a held value is its own nearest
            assert np.array_equal(oa.value_of(byte, codes), held)


def test_rotation_keeps_norms_and_turns_by_the_angle():
    rng = np.random.default_rng(1)
    x = rng.normal(size=96)
    a = rng.normal(size=32)
    for inter in (False, True):
        y = oa.norm_rope(x, None, 0.0, np.cos(a), np.sin(a), inter)
        z = oa.norm_rope(y, None, 0.0, np.cos(-a), np.sin(-a), inter)
        assert np.allclose(z, x) and np.allclose(y[64:], x[64:])
        i, j = (6, 7) if inter else (3, 35)
        assert np.allclose((y[i] + 1j * y[j]), (x[i] + 1j * x[j]) * np.exp(1j * a[3]))
    w = np.full(96, 2.0)
    assert math.isclose(np.mean(oa.norm_rope(x, w, 0.0, [], [], False) ** 2), 4.0)


def test_visible_keys():
    assert [oa.visible(p, 1, 5) for p in (-3, -1, 0, 3, 4, 9)] == [0, 0, 1, 4, 5, 5]
    assert [oa.visible(p, 4, 10) for p in (-4, -1, 0, 3, 4, 8)] == [0, 0, 4, 4, 8, 10]
    assert oa.visible(-7, 0, 6) == 6


def test_attend_against_a_double_loop():
    rng = np.random.default_rng(2)
    q, k, v = rng.normal(size=(5, 4, 8)), rng.normal(size=(7, 2, 8)), rng.normal(size=(7, 2, 8))
    out, lse, _, _ = oa.attend(q, k, v, 0.3, 1, -2)
    for i in range(5):
        seen = max(0, i - 2 + 1)
        for h in range(4):
            w = [math.exp(0.3 * float(np.dot(q[i, h], k[j, h // 2]))) for j in range(seen)]
            if not w:
                assert lse[i, h] == -np.inf and (out[i, h] == 0).all()
                continue
            assert math.isclose(lse[i, h], math.log(sum(w)))
            assert np.allclose(out[i, h], sum(wj * v[j, h // 2] for j, wj in enumerate(w)) / sum(w))

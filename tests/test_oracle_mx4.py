"""The 4-bit and distillation oracles against closed forms, brute force and differences."""

import numpy as np
import pytest

from oracle import distill, mx4


def test_every_tie_goes_to_the_even_code():
    x = np.array([[0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -0.25, -5.0, -0.75] + [0.0] * 21])
    codes, e, v = mx4.quantize(x)
    assert e[0, 0] == 0
    assert v[0, :11].tolist() == [0, 1, 1, 2, 2, 4, 4, 6, 0, -4, -1]


@pytest.mark.parametrize("top,e", [(6.0, 0), (np.nextafter(6.0, 7), 1), (3.0, -1), (12.0, 1), (12.1, 2), (0.0, -127),
                                   (2.0 ** -140, -127), (6 * 2.0 ** -127, -127), (6.1 * 2.0 ** -127, -126),
                                   (3.4e38, 126)])
def test_exponents(top, e):
    assert mx4.quantize(np.full((1, 3), top))[1][0, 0] == e


def test_no_code_is_further_than_half_a_step():
    x = np.random.default_rng(0).normal(size=(7, 75))
    codes, e, v = mx4.quantize(x)
    scale = np.repeat(2.0 ** e, 32, axis=1)[:, :75]
    m = np.abs(x) / scale
    half = np.where(m < 2, 0.25, np.where(m < 4, 0.5, 1.0))
    assert (np.abs(v - x) <= half * scale).all() and (m <= 6).all() and (np.abs(x).max() / scale[0, 0] > 0)


def test_layout_round_trip():
    x = np.random.default_rng(1).normal(size=(261, 300))
    codes, e, v = mx4.quantize(x)
    q, s = mx4.pack(codes, e)
    assert q.shape == (261, 160) and s.size == 3 * 3 * 512
    c2, e2 = mx4.unpack(q, s, 300)
    assert (mx4.value_of(c2, e2) == v).all()
    places = {mx4.scale_place(r, b, 300) for r in range(261) for b in range(10)}
    assert len(places) == 2610 and max(places) < s.size


def test_distill_gradient_against_differences():
    rng = np.random.default_rng(2)
    y = rng.normal(size=(4, 9))
    y[1, 3] = np.inf
    top, index = rng.normal(size=(4, 5)), rng.integers(-1, 11, size=(4, 5))
    index[0, :3] = 2
    index[3] = -1
    w = rng.random(4)
    kw = dict(factor=-1.7, silent=0.4, teacher_factor=0.8, weight=1.3, row_weight=w)
    loss, rows, g = distill.distill(y, top, index, **kw)
    assert np.isfinite(loss) and rows[3] == 0 and (g[3] == 0).all() and g[1, 3] == 0
    for r in range(4):
        for c in range(9):
            if not np.isfinite(y[r, c]):
                continue
            d = np.zeros_like(y)
            d[r, c] = 1e-5
            num = (distill.distill(y + d, top, index, **kw)[0] - distill.distill(y - d, top, index, **kw)[0]) / 2e-5
            assert abs(num - g[r, c]) < 1e-8


def test_distill_from_itself_is_zero():
    z = np.random.default_rng(3).normal(size=(3, 6))
    top, index = distill.top_logits(z, 6)
    loss, rows, g = distill.distill(z, top, index)
    assert abs(loss) < 1e-15 and np.abs(g).max() < 1e-16


def test_top_logits_orders_ties_and_nan():
    z = np.array([[1.0, 3.0, 3.0, np.nan, -np.inf, 3.0]])
    v, i = distill.top_logits(z, 5)
    assert i[0].tolist() == [3, 1, 2, 5, 0] and np.isnan(v[0, 0]) and v[0, 1:].tolist() == [3, 3, 3, 1]

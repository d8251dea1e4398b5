"""Where min-p ends a row in chunks: bins before it are kept whole and bins behind it dropped unseen, so no score of those may lie on the other side.
The rule on the host, against the whole-number weights; CPU only."""
import math

import numpy as np
import pytest

from tests import cut_util

f32 = np.float32
D0, DMAX, SHIFT, BINS = 0x35800000, 0x41B20000, 18, 800


def _bin(d):
    b = np.asarray(d, f32).view(np.uint32).astype(np.int64)
    return np.where(b < D0, 0, ((b - D0) >> SHIFT) + 1)


def _border(d):
    """The first and the last bin that are looked into around the distance d."""
    end = np.array(DMAX - 1, np.uint32).view(f32)
    near = lambda x: int(_bin(min(f32(max(x, 0.0)), end)))
    return max(near(d - 2e-6) - 1, 0), min(near(d + 2e-6) + 1, BINS - 1)


def _distances():
    grid = lambda a, b, n: np.unique(np.linspace(int(f32(a).view(np.uint32)), int(f32(b).view(np.uint32)), n).astype(np.uint32)).view(f32)
    return np.concatenate([grid(1e-9, 2e-5, 300000), grid(2e-5, 22.3, 400000)])


def _wrong(border):
    """How many of the settings put a score on the wrong side."""
    d = _distances()
    w, b = cut_util.weights(np.concatenate([[f32(0)], -d]).astype(f32))[1:], _bin(d)
    r, wrong = np.random.default_rng(2), 0
    for min_p in np.concatenate([1 - r.uniform(0, 2e-5, 250), 1 - r.uniform(0, 1e-6, 60), r.uniform(0.5, 1, 60), np.exp(r.uniform(-23, 0, 150)), [0.0, 1.0, 2.0 ** -32]]):
        least = max(math.ceil(float(f32(min_p)) * 2 ** 32), 1)
        b0, b1 = border(least)
        wrong += bool(((w < least) & (b < b0)).any() or ((w >= least) & (b > b1)).any())
    return wrong


def _near_one(least, units):
    """The distance by what the weight lacks of 2^32, in 32 bits, the logarithms `units` off."""
    if least > 1 << 31:
        d = f32(-math.log1p(-float(f32((1 << 32) - least) * f32(2.0 ** -32))))
        return float(d + units * np.spacing(d))
    x = f32(math.log2(float(f32(least))))
    return float(f32(f32(32) - (x + units * np.spacing(max(x, f32(1))))) * f32(0.693147181))


@pytest.mark.parametrize("units", [0, -3, 3])
def test_by_what_the_weight_lacks(units):
    assert _wrong(lambda least: _border(_near_one(least, units))) == 0


def test_a_logarithm_of_the_weight_would_have_to_be_rounded_right():
    """One unit of it near 32, in 32 bits, is wider than what is looked into."""
    low = lambda least: np.nextafter(f32(math.log2(least)), f32(-np.inf))
    assert _wrong(lambda least: _border(float(f32(f32(32) - low(least)) * f32(0.693147181)))) > 0


@pytest.mark.parametrize("from_,to,most", [(1e-9, 1e-3, 1e-6), (1e-3, 22.1, 1e-5)])
def test_how_far_the_weights_move_it(from_, to, most):
    d = _distances()
    d = d[(d >= from_) & (d < to)]
    w = cut_util.weights(np.concatenate([[f32(0)], -d]).astype(f32))[1:].astype(np.float64)
    # (a weight is cut to a whole number: the score's lies up to 1 above it)
    low, high = -np.log((w + 1) / 2 ** 32), -np.log(w / 2 ** 32)
    assert (low - d).max() < most and (d - high).max() < most

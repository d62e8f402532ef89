"""Frequencies of rotary positions (attention.py), every one of each scaling
against its definition in numpy, written apart from the package."""
import numpy as np
import pytest

import paper_2402_10076_amd as Q


def _plain(dim, base):
    return np.exp(-np.log(base) * np.arange(0, dim, 2) / dim)


def _keep(scaling, dim, base, original, low, high):
    """How much of its own frequency each pair keeps."""
    turns = original * _plain(dim, base) / (2 * np.pi)
    if scaling == "bands":
        return np.interp(turns, [low, high], [0, 1])
    # the whole numbers around the pairs that would turn `high` and `low` times: turns fall by the same factor a pair
    fall = np.log(base) * 2 / dim
    at = [np.log(turns[0] / t) / fall for t in (high, low)]
    first, last = max(np.floor(at[0]), 0), min(np.ceil(at[1]), dim - 1)
    i = np.arange(dim // 2)
    return np.where(i <= first, 1.0, np.where(i >= last, 0.0, (last - i) / max(last - first, 1)))


@pytest.mark.parametrize("dim", [2, 64, 96, 128, 250])
@pytest.mark.parametrize("base", [1e4, 5e5, 37.0])
@pytest.mark.parametrize("factor", [1.0, 4.0, 32.0, 0.5])
def test_every_frequency(dim, base, factor):
    plain = _plain(dim, base)

    def got(scaling, **kw):
        freqs, attention = Q.rotary_frequencies(dim, base, scaling=scaling, factor=factor, device="cpu", **kw)
        assert np.isclose(attention, 0.1 * np.log(factor) + 1 if scaling == "ramp" and factor > 1 else 1.0, rtol=1e-14)
        return freqs.numpy()
    assert np.allclose(got("none"), plain, rtol=1e-12, atol=0)
    assert np.allclose(got("linear"), plain / factor, rtol=1e-12, atol=0)
    # the slowest pair `factor` times slower, the fastest as before, and a constant ratio between
    assert np.allclose(got("base"), plain * factor ** (-np.arange(dim // 2) / max(dim // 2 - 1, 1)), rtol=1e-12, atol=0)
    for original in (64, 4096, 100000):
        for low, high in ((1.0, 32.0), (1.0, 4.0), (0.25, 8.0), (3.0, 3.5)):
            for scaling in ("ramp", "bands"):
                keep = _keep(scaling, dim, base, original, low, high)
                f = got(scaling, original=original, low=low, high=high)
                assert np.allclose(f, plain * keep + plain / factor * (1 - keep), rtol=1e-12, atol=0), (scaling, original, low, high)


def test_what_a_ramp_cannot_be_made_of():
    for base in (1.0, 0.5):
        with pytest.raises(Q.QuickError):
            Q.rotary_frequencies(64, base, scaling="ramp", factor=2.0, original=4096, device="cpu")
    for low, high in ((0.0, 4.0), (4.0, 4.0), (5.0, 4.0)):
        for scaling in ("ramp", "bands"):
            with pytest.raises(Q.QuickError):
                Q.rotary_frequencies(64, scaling=scaling, factor=2.0, original=4096, low=low, high=high, device="cpu")

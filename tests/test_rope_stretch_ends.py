"""The stretch by pair index where all pairs lie on one side of its ramp (no GPU): the library and the
oracle against the turns that the pairs make over the trained length."""
import numpy as np
import pytest

from oracle import sepllm_oracle as orc
from paper_2412_12094_b200 import api, build


@pytest.fixture(scope="module", autouse=True)
def _lib():
    build.build()


def _both(r, base, **kw):
    f, _ = api.sepllm_rope_frequencies(api.RopeDesc(1, 1, 1, 1, 128, rot_dim=r, scaling="yarn", base=base, **kw))
    ref = orc.rope_frequencies(r, base, "yarn", **kw)
    assert np.allclose(f, ref, rtol=1e-13, atol=0)
    return f, base ** (-2.0 * np.arange(r // 2) / r)


@pytest.mark.parametrize("r,base,N", [(64, 10.0, 1e6), (128, 2.0, 8192.0), (20, 10.0, 1e5), (4, 1.5, 2000.0),
                                      (64, 1e4, 1e12), (2, 10.0, 1e5)])
def test_pairs_that_all_turn_often_stay(r, base, N):
    f, plain = _both(r, base, factor=8.0, low=1.0, high=32.0, orig_len=N)
    assert (N * plain / (2 * np.pi) > 32.0).all()
    assert np.allclose(f, plain, rtol=1e-13, atol=0)


@pytest.mark.parametrize("r,base,N,low", [(64, 1e4, 2.0, 1.0), (128, 5e5, 16.0, 8.0), (20, 1e4, 1.0, 1.0),
                                          (64, 1e4, 100.0, 31.0)])
def test_pairs_that_all_turn_seldom_are_stretched_in_full(r, base, N, low):
    # (t(low) at most -1, so that its rounded-up place is before the first pair)
    assert r * np.log(N / (2 * np.pi * low)) / (2 * np.log(base)) <= -1.0
    f, plain = _both(r, base, factor=8.0, low=low, high=32.0, orig_len=N)
    assert (N * plain / (2 * np.pi) < low).all()
    assert np.allclose(f, plain / 8.0, rtol=1e-13, atol=0)


@pytest.mark.parametrize("r,base,N,low", [(4, 1e6, 0.01, 1.0)])
def test_a_ramp_that_rounds_to_the_first_pair_keeps_that_pair(r, base, N, low):
    """t(low) between -1 and 0 rounds up to 0 = lo: pair 0 is the formula's kept end, the others are stretched."""
    assert -1.0 < r * np.log(N / (2 * np.pi * low)) / (2 * np.log(base)) <= 0.0
    f, plain = _both(r, base, factor=8.0, low=low, high=32.0, orig_len=N)
    assert f[0] == plain[0] and np.allclose(f[1:], plain[1:] / 8.0, rtol=1e-13, atol=0)


@pytest.mark.parametrize("N", np.geomspace(0.1, 1e9, 60))
@pytest.mark.parametrize("r,base", [(64, 10.0), (64, 1e4), (20, 3.0)])
def test_a_longer_trained_length_never_stretches_a_pair_more(r, base, N):
    kw = dict(factor=4.0, low=1.0, high=32.0)
    a, plain = _both(r, base, orig_len=N, **kw)
    b, _ = _both(r, base, orig_len=1.5 * N, **kw)
    assert (b >= a * (1 - 1e-12)).all() and (a <= plain * (1 + 1e-12)).all() and (a >= plain / 4 * (1 - 1e-12)).all()

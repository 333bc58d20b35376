"""Frequencies of rotary positions are finite or refused."""
import numpy as np
import pytest


@pytest.mark.parametrize("rot, base, scaling, par", [(64, 1e4, 1, [1e-309]), (64, 1e4, 2, [1e-320]), (64, 1e4, 2, [5e-324]),
                                                     (4, 2.0, 2, [1e-300])])
def test_frequencies_that_are_not_finite_are_refused(rot, base, scaling, par):
    from paper_2602_11470_amd import binding as B
    with pytest.raises(B.CachemirError) as e:
        B.rotary_freqs(rot, base, scaling, par)
    assert e.value.status == -1


@pytest.mark.parametrize("rot, base, scaling, par", [(64, 1e4, 1, [1e-3]), (64, 1e4, 2, [0.5]), (64, 1e300, 2, [1e300]), (64, 1e4, 1, [1e300]), (2, 1e4, 2, [5e-324]),
                                                     (64, 1e4, 3, [0.5, 1.0, 4.0, 8192.0]),
                                                     # what the factor divides turns less than 4 times: 4 2 pi / 8192 / 1e-309 = 3e306
                                                     (64, 1e4, 3, [1e-309, 1.0, 4.0, 8192.0])])
def test_others_are_finite(rot, base, scaling, par):
    from paper_2602_11470_amd import binding as B
    assert np.isfinite(B.rotary_freqs(rot, base, scaling, par)).all()

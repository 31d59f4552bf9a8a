"""Frequencies that 64 bits do not hold are refused (CPU only)."""
import warnings

import numpy as np
import pytest

from paper_2609_28870_amd import pc

INF = float("inf")


@pytest.mark.parametrize("kw", [
    dict(rot_dim=4, scaling="base", factor=1e200),                               # the factor's power
    dict(rot_dim=8, base=1e308, scaling="base", factor=1e5),                     # the base's product with it
    dict(rot_dim=8, scaling="linear", factor=5e-324),
    dict(rot_dim=8, scaling="ramp", factor=5e-324, trained=1),
    dict(rot_dim=8, scaling="ramp", trained=10, slow=-INF, fast=INF),            # no ramp between them
], ids=str)
def test_refused(kw):
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        with pytest.raises(pc.PcError):
            pc.rope_frequencies(**kw)


def test_large_ones_are_taken():
    assert np.isclose(pc.rope_frequencies(64, 1e300, "base", 1e5)[-1], 1e300 ** (-62 / 64) / 1e5, rtol=1e-12, atol=0)
    assert np.array_equal(pc.rope_frequencies(64, 500.0, "ramp", 4.0, trained=100, fast=INF), pc.rope_frequencies(64, 500.0) / 4)

"""Rotary positions without a GPU: frequencies at the ends of their ranges."""
import math

import numpy as np
import pytest

pytest.importorskip("torch")
kmip = pytest.importorskip("paper_2604_03815_amd")


@pytest.mark.parametrize("factor", [1.0, 0.5, 1e-5, 1e-300])
def test_blend_of_shorter_contexts(factor):
    """The blend's magnitude makes up for longer contexts only: it neither falls below 1 nor changes its sign."""
    f, m = kmip.rotary_frequencies(64, scaling="blend", factor=factor, original_length=4096)
    plain, _ = kmip.rotary_frequencies(64)
    assert m == 1.0
    turns = 4096 * plain / (2 * math.pi)
    assert np.allclose(f[turns >= 32], plain[turns >= 32]) and np.allclose(f[turns <= 1], plain[turns <= 1] / factor)
    assert kmip.rotary_frequencies(64, scaling="blend", factor=4.0, original_length=4096)[1] == 0.1 * math.log(4.0) + 1.0

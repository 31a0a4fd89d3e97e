"""Frequencies that float32 cannot hold are refused (host)."""

import numpy as np
import pytest

import paper_2609_32197_amd as sp


def test_frequencies_are_finite():
    f, _ = sp.sparsp_rope_frequencies(256, 1e-30)  # 10^29.8 at most
    assert np.isfinite(f).all() and f[-1] > 1e29
    f, _ = sp.sparsp_rope_frequencies(256, 1e300)  # below the smallest number: 0
    assert f[0] == 1 and f[-1] == 0
    with pytest.raises(sp.SparspError, match="theta"):
        sp.sparsp_rope_frequencies(256, 1e-40)
    with pytest.raises(sp.SparspError, match="theta"):
        sp.sparsp_rope_frequencies(4, 5e-324)

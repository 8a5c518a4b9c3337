"""What the operators of a layer around the cached histories promise where a GPU is not needed to see it (the pointers are numbers
that are never followed)."""
from fractions import Fraction

import numpy as np
import pytest

from paper_2511_14881_amd import binding as st
from tests.test_layer_host import P, adapters, project


# ---------------------------------------------------------------- workspaces
@pytest.mark.parametrize("n", [16, 512, 1344, 5120, 65536])
@pytest.mark.parametrize("count,rank", [(1, 8), (4, 16), (8, 128), (300, 64)])
def test_workspace_for_more_rows_is_enough_for_fewer(n, count, rank):
    ad = adapters(n_adapters=count, rank=rank)
    rows = [0, 1, 2, 16, 63, 64, 65, 100, 128, 129, 191, 192, 193, 256, 320, 383, 384, 385, 500, 1025, 2048, 2049, 4000, 16384, 1 << 20]
    sizes = [st.lib().st_project_workspace_bytes(m, 4096, n, ad) for m in rows]
    assert sizes == sorted(sizes) and sizes[0] == 256
    # what a call asks for is found out with one byte less than all of it: refused for its workspace, or for what is checked behind that
    for m, size in zip(rows[1:], sizes[1:]):
        asked = [project(ad, rows=m, n=n, k=4096, stride=n, nbytes=b, work=P + 128) for b in (size, 255)]
        assert asked == [st.ST_EINVAL, st.ST_EWORKSPACE], (m, size)
    for larger in (len(rows) - 1, rows.index(2048), rows.index(385)):
        for m in rows[1:larger]:
            assert project(ad, rows=m, n=n, k=4096, stride=n, nbytes=sizes[larger], work=P + 128) == st.ST_EINVAL


# ---------------------------------------------------------------- angles
def test_angles_are_as_near_as_promised():
    """The turns that a rotation counts in fp64, position * (frequency * 1 / 2 pi), against exact ones: three roundings, 2.56 half steps in all, and more than two
    of them do come together."""
    pi = Fraction(314159265358979323846264338327950288419716939937510582097494459, 10 ** 62)
    inverse = 0.15915494309189533577
    rng = np.random.default_rng(5)
    positions, freqs = rng.integers(1, 2 ** 31, 4000).tolist(), np.exp(rng.uniform(np.log(1e-9), np.log(2 * np.pi), 4000)).tolist()
    off = []
    for p, f in zip(positions, freqs):
        turns = Fraction(p) * Fraction(f) / (2 * pi)
        off.append(float(abs(Fraction(p * (f * inverse)) / turns - 1) * 2 ** 52))
    assert max(off) <= (1 + 1 + 0.557) / 2 + 2.0 ** -50 < 1.3 and max(off) > 1.0

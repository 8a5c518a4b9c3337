"""What the operators of a layer around the cached histories promise where a GPU is not needed to see it (the pointers are numbers
that are never followed)."""
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

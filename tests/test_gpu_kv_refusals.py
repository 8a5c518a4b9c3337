"""A refused call on cached histories has written nothing."""
import pytest
import torch

from paper_2511_14881_amd import binding as st

pytestmark = pytest.mark.gpu


def test_weights_of_too_many_blocks_are_refused_before_anything_is_written():
    """4200 tables of 16384 blocks: the attention itself would fit a launch, summing the weights of 68.8 million blocks does not."""
    n_seq, group = 4200, 17
    cache = st.KvCache.empty(1, 1, 64)
    tables = torch.zeros((n_seq, st.ST_KV_MAX_BLOCKS), dtype=torch.int32, device="cuda")
    batch = st.KvBatch(tables, torch.ones(n_seq, dtype=torch.int32, device="cuda"), n_seq, max_len=1)
    q = torch.ones((n_seq, group, 64), dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(q, 7.0)
    mass = torch.full((n_seq, 1, st.ST_KV_MAX_BLOCKS), 7.0, device="cuda")
    with pytest.raises(st.StError) as refused:
        st.st_kv_attend(cache, batch, q, out=out, mass_out=mass)
    assert refused.value.code == st.ST_EINVAL
    torch.cuda.synchronize()
    assert (out == 7.0).all() and (mass == 7.0).all()
    st.st_kv_attend(cache, batch, q, out=out)  # without the weights it is a call like others
    assert (out == 0.0).all()

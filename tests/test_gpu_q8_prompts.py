"""Prompts that an 8-bit cache has no room for."""
import pytest
import torch

from paper_2512_00504_amd import make_config
from paper_2512_00504_amd.state import Q8DecodeState

pytestmark = pytest.mark.gpu


def test_a_prompt_beyond_the_capacity_is_refused_before_decoding():
    st = Q8DecodeState(make_config(1, 2, 2, 1, 64, 16, 4, 8, 32, "bf16"))
    k = torch.randn(33, 1, 2, 1, 64)
    st.load_prompt_rows(7, k, k, 40, [33, 32])             # the rows that fit are there
    with pytest.raises(ValueError, match="33 rows .* capacity of 32"):
        st.begin_decode(40, [33, 32])
    assert (st.d_state == 0).all() and st.len_host == 0
    st.begin_decode(40, [32, 32])
    assert st.len_host == 32 and st.d_state[0, :, 0].tolist() == [32, 32]

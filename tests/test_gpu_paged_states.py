"""Paged decode states where they refuse a call."""
import pytest
import torch

from paper_2512_00504_amd import Rotary, make_config
from paper_2512_00504_amd.state import PagedDecodeState

pytestmark = pytest.mark.gpu


def _states(n, **kw):
    cfg = make_config(2, 3, 4, 2, 64, 64, 8, 16, 96, "bf16")
    return [PagedDecodeState(cfg, **{**dict(max_rows=64, page_rows=16, rotary=Rotary(64)), **kw}) for _ in range(n)]


def _token(gen, n=3):
    return [torch.randn(2, n, h, 64, generator=gen).to(torch.bfloat16).cuda() for h in (4, 2, 2)]


def test_a_step_that_needs_pages_is_not_recorded():
    a, b = _states(2)
    gen = torch.Generator().manual_seed(0)
    q, k, v = _token(gen, 20)
    for st in (a, b):
        st.append(k, v, [16, 3, 1])
    ins = _token(gen)
    with pytest.raises(ValueError, match="record"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            a.attend_decode(*ins)
    for t in range(3):
        assert torch.equal(a.attend_decode(*ins), b.attend_decode(*ins))
        assert a.lengths == b.lengths == a.d_len.tolist() and torch.equal(a.page_table, b.page_table)


def test_queries_that_lie_apart_are_not_turned_in_place():
    a, = _states(1)
    q, k, v = _token(torch.Generator().manual_seed(1))
    both = torch.cat([q, q], dim=2)
    with pytest.raises(ValueError, match="place"):
        a.append(k, v, None, both[:, :, :4], None, both.view(-1)[:q.numel()].view(q.shape))
    assert a.lengths == a.d_len.tolist() == [0, 0, 0] and not any(a._pages)

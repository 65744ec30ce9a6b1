"""Buffers of a shared prefix that are too small: refused before anything is launched (no GPU needed)."""
import pytest
import torch

import paper_2512_00504_amd as P


def _ctx():
    return P.Context(P.make_config(n_layers=1, batch=4, n_q_heads=8, n_kv_heads=2, head_dim=64, budget=64, window=8, interval=16, capacity=96, dtype="bf16"))


def test_a_part_sized_for_fewer_rows_is_refused():
    # another buffer of the context was sized for these rows, so the C call alone would take them
    ctx = _ctx()
    short = torch.zeros(ctx.prefix_bytes(10), dtype=torch.uint8)
    long = torch.zeros(ctx.prefix_bytes(20000), dtype=torch.uint8)
    assert short.numel() < long.numel()
    q = torch.zeros(1, 4, 8, 64, dtype=torch.bfloat16)
    k = torch.zeros(1, 2, 1, 64, dtype=torch.bfloat16)
    for rows in (20000, 5000, 19999):                      # asked for, and between
        with pytest.raises(P.GkvError) as e:
            ctx.prefix_attend(q, k, k, rows, rows, 0, 4, short)
        assert e.value.status == 3
    with pytest.raises(P.GkvError):
        ctx.prefix_attend(q, k, k, 20000, 20000, 0, 4, long[:-1])
    # beyond what any buffer was sized for: the library's own refusal
    assert ctx.lib.gkv_prefix_attend(ctx.h, 4096, 4096, 4096, 20001, 20001, 0, 4, 4096, None) == 3
    ctx.close()

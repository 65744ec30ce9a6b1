"""Decode attention over pages stays inside the workspace that it asks for, and leaves its tickets at zero."""
import pytest
import torch

import paper_2512_00504_amd as P
from paper_2512_00504_amd import make_config

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d,g,hkv,params", [("bf16", 128, 7, 1, None), ("bf16", 128, 20, 1, None), ("bf16", 128, 33, 2, None), ("bf16", 256, 17, 1, None), ("bf16", 256, 4, 2, None),
                                                  ("bf16", 96, 5, 1, None), ("bf16", 64, 16, 1, None), ("f32", 64, 20, 1, None), ("f32", 128, 3, 2, None), ("bf16", 48, 5, 1, None),
                                                  ("f32", 20, 18, 1, None), ("bf16", 128, 18, 2, {"force_generic": 1})])
@pytest.mark.parametrize("lens,page_rows", [([33000], 16), ([33000], 12), ([4000, 1, 0, 9000, 700], 16)])
def test_nothing_behind_the_workspace_is_written(dtype, d, g, hkv, params, lens, page_rows):
    B = len(lens)
    ctx = P.Context(make_config(1, B, hkv * g, hkv, d, 64, 8, 16, 96, dtype))
    for name, value in (params or {}).items():
        ctx.set_param(name, value)
    gen, dt = torch.Generator(device="cuda").manual_seed(3), (torch.bfloat16 if dtype == "bf16" else torch.float32)
    n = [-(-x // page_rows) for x in lens]
    K, V = (torch.randn(1, sum(n), hkv, page_rows, d, generator=gen, device="cuda").to(dt) for _ in range(2))
    q = torch.randn(1, B, hkv * g, d, generator=gen, device="cuda").to(dt)
    table = torch.full((B, max(n)), -1, dtype=torch.int32)
    for i, m in enumerate(n):
        table[i, :m] = torch.arange(sum(n[:i]), sum(n[:i]) + m, dtype=torch.int32)
    table, d_len = table.cuda(), torch.tensor(lens, dtype=torch.int32).cuda()
    need = ctx.paged_workspace_bytes()
    buffer = torch.full((need + (1 << 20),), 0xA5, dtype=torch.uint8, device="cuda")
    workspace = buffer[:need]
    workspace.zero_()
    outs = []
    for _ in range(3):
        outs.append(torch.empty_like(q))
        ctx.paged_attend_decode(q, K, V, table, d_len, max(n) * page_rows, outs[-1], workspace)
    assert (buffer[need:] == 0xA5).all()
    tickets = 128 * 8 * B * hkv * -(-g // 16)
    assert (workspace[:tickets] == 0).all() and (workspace[tickets:] != 0).any()      # (units were cut)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])

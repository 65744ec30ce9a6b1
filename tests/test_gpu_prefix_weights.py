"""Shared prefixes: weights and their sum belong together."""
import math

import pytest
import torch

from paper_2512_00504_amd import make_config
from paper_2512_00504_amd.state import DecodeState, SharedPrefix

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("L,hkv,g,B", [(1, 2, 7, 4), (1, 2, 7, 9), (24, 32, 2, 33), (1, 1, 3, 1)])
def test_the_mean_of_equal_values_is_that_value(dtype, d, L, hkv, g, B):
    # Whatever the weights, sum w v / sum w is v where all v are the same: to the last bit in bf16, with 32-bit sums of 256 weights (256 * 2^-24, and
    # a few roundings of factors and quotient, far below the half step of 2^-8 that v is away from its neighbours).  Some keys weigh e^4.8555 = 128.45
    # of the first ones, where numbers of 8 bits lie 1 apart.
    rows, nats = 256, 4.8555
    st = DecodeState(make_config(L, B, hkv * g, hkv, d, 16, 4, 8, 64, dtype))
    q = torch.zeros(L, B, hkv * g, d)
    q[..., 0], q[..., 1] = 8.0, 0.125
    logit = torch.full((rows,), -50.0, dtype=torch.float64)
    logit[0:128:32] = 0.0
    logit[128::32] = nats
    k = torch.zeros(L, hkv, rows, d)
    first = (logit * math.sqrt(d) / 8).to(torch.bfloat16).double()
    k[..., 0], k[..., 1] = first.float(), ((logit * math.sqrt(d) - 8 * first) * 8).float()
    v = (torch.randint(128, 256, (L, hkv, 1, d), generator=torch.Generator().manual_seed(d)) / 128.0).expand(L, hkv, rows, d)
    prefix = SharedPrefix(st, k.cuda(), v.cuda())
    out = st.attend_decode(q.to(DT[dtype]).cuda(), None, None, 0, prefix=prefix).cpu().double()
    want = v[:, None, :, :1].expand(L, B, hkv, g, d).reshape(out.shape).double()
    assert ((out - want).abs() <= (0 if dtype == "bf16" else 300 * 2.0 ** -24) * want).all(), ((out - want) / want).abs().max().item()

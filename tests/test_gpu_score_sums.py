"""Window scores on 8-bit caches without recorded statistics: what the rows' sums lose to their offsets."""
import math

import pytest
import torch

from paper_2512_00504_amd import make_config
from paper_2512_00504_amd.state import Q8DecodeState

from planted import score
from q8_reference import values
from test_gpu_q8 import _fill

pytestmark = pytest.mark.gpu


def _pieces(x):
    """x >= 0, a multiple of 1/256 below 512, as four numbers of 4 bits each."""
    out = []
    for step in (16.0, 1.0, 2.0 ** -4, 2.0 ** -8):
        out.append(x // step * step if step > 2.0 ** -8 else x)
        x = x - out[-1]
    return out


@pytest.mark.parametrize("rise", [2.75, 2.8125, 5.0])
@pytest.mark.parametrize("dtype,g,w", [("bf16", 1, 8), ("bf16", 8, 16), ("bf16", 5, 32), ("bf16", 9, 16), ("f32", 2, 8)])
def test_sums_under_logits_that_rise_along_the_cache(dtype, g, w, rise):
    # Every eighth tile's first key is `rise` nats above the one before, from 140 on; the other tiles' first keys stay there, all others weigh
    # e^-40 of it.  q . k is exact, d^-1/2 is 1/8, log2(e) enters in two parts: what is left of a probability's error is
    #   the exponents' rounding in the sum: below 16 (2^8 before the offset rises, 7.3 for a rise of 5 nats in a tile) 2^-21 * ln 2 = 3.3e-7;
    #   the rounding of the score's own exponent, 2^(k - 24) * ln 2 from 2^k on (it has an 8 in it, the window's rows: 3 more), and of its second part: twice;
    #   two exponentials of 1.5 * 2^-23 each; 4 sums that matter within a lane, 3 over lanes and wavefronts, 5 over the window's rows: 12 * 2^-24.
    d, b, s, cap, B = 64, 2048, 64, 2112, 12
    st = Q8DecodeState(make_config(1, B, g, 1, d, b, w, s, cap, dtype))
    gen = torch.Generator().manual_seed(g)
    fine = torch.randint(0, 256, (B, cap), generator=gen).double() / 256
    logit = 100 + fine
    for tile in range(cap // 16):
        up = rise * (tile // 8) if tile % 8 == 0 else 0.0
        logit[:, 16 * tile] = 140 + up + fine[:, 16 * tile] / 4 // 2 ** -8 * 2 ** -8
    K = torch.zeros(1, B, 1, cap, d)
    for c, x in enumerate(_pieces(logit)):
        K[0, :, 0, :, c] = x.float()
    assert torch.equal(values(K), K.double()) and torch.equal(K[0, :, 0, :, :4].double().sum(dim=-1), logit)
    K = K.to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    q = torch.zeros(w, 1, B, g, d)
    q[..., :4] = 8.0                                       # 8 / sqrt(64): the logits are K's sums
    q[:, :, :, 1:, :4] = 4.0
    t = 2 * w + 3
    _fill(st, K, torch.zeros_like(K), [cap] * B, b, since=t - w + 1, decoded=w)
    st.qwin.copy_(q.roll(t - w + 1, 0))
    st.len_host = cap
    st.score_window(t)
    S = st.S[0, :, 0, :cap - w].cpu().double()
    for i in range(B):
        ref = score(q[:, 0, i].double(), K[0, i, 0].double(), 0.125)
        own = 2 * torch.exp2(torch.floor(torch.log2(3 - torch.log2(ref.clamp(min=2.0 ** -100)))) - 24) * math.log(2)
        err = ((S[i] - ref).abs() / ref - own)[ref > 2.0 ** -40]
        assert (err <= 3.3e-7 + 3.6e-7 + 7.2e-7).all(), (i, err.max().item())

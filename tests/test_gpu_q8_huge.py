"""8-bit caches under huge queries: a query times a code may pass 2^128 where the logit, with the row's scale, does not."""
import math

import pytest
import torch

from paper_2512_00504_amd import make_config
from paper_2512_00504_amd.state import Q8DecodeState

from planted import DT, rows, score
from q8_reference import values
from test_gpu_q8 import _fill

pytestmark = pytest.mark.gpu
FORMS = [("bf16", 128, 7, None), ("bf16", 64, 3, None), ("f32", 64, 4, None), ("f32", 128, 2, None), ("bf16", 48, 3, None), ("bf16", 128, 3, {"force_generic": 1}),
         ("f32", 64, 3, {"force_generic": 1}), ("bf16", 128, 9, None), ("bf16", 128, 4, {"attend_splits": 2})]


@pytest.mark.parametrize("dtype,d,g,params", FORMS)
@pytest.mark.parametrize("power", [100, 118, 121])
def test_the_largest_logit_takes_all(dtype, d, g, params, power):
    # logits of about 2^power apart by millions: the largest one's row is the result, to its rounding
    lens, cap = [40, 1, 200, 255], 256
    st = Q8DecodeState(make_config(1, 4, 2 * g, 2, d, 64, 8, 16, cap, dtype), params=params)
    gen = torch.Generator().manual_seed(power)
    K, V = rows(gen, dtype, 1, 4, 2, cap, d), rows(gen, dtype, 1, 4, 2, cap, d)
    q, kn, vn = rows(gen, dtype, 1, 4, 2 * g, d) * 2.0 ** power, rows(gen, dtype, 1, 4, 2, d), rows(gen, dtype, 1, 4, 2, d)
    _fill(st, K, V, lens, 48)
    out = st.attend_decode(q.cuda(), kn.cuda(), vn.cuda(), 5).cpu().double()
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -23
    for i, n in enumerate(lens):
        for j in range(2):
            k, v = (values(torch.cat([x[0, i, j, :n], y[0, i, j][None]])) for x, y in ((K, kn), (V, vn)))
            best = v[(q[0, i, j * g:(j + 1) * g].double() @ k.T).argmax(dim=-1)]
            assert ((out[0, i, j * g:(j + 1) * g] - best).abs() <= half * best.abs()).all(), (i, j)


def _score_case(dtype, d, g, params, power, decoded):
    """Every window row's probabilities are 1 and 0: S counts the rows that have their largest logit at a candidate."""
    b, w, s, lens, cap = 64, 8, 16, [80, 70], 96
    st = Q8DecodeState(make_config(1, 2, 2 * g, 2, d, b, w, s, cap, dtype), params=params)
    gen = torch.Generator().manual_seed(power + d)
    K, V = rows(gen, dtype, 1, 2, 2, cap, d), rows(gen, dtype, 1, 2, 2, cap, d)
    q = rows(gen, dtype, w, 1, 2, 2 * g, d) * 2.0 ** power
    t = 2 * w + 3
    if decoded:
        _fill(st, K, V, [n - w for n in lens], b, since=t - w + 1)
        for k in range(w):
            kn, vn = (torch.stack([x[:, i, :, n - w + k] for i, n in enumerate(lens)], dim=1) for x in (K, V))
            st.attend_decode(q[k].cuda(), kn.cuda().contiguous(), vn.cuda().contiguous(), t - w + 1 + k)
    else:
        _fill(st, K, V, lens, b, since=t - w + 1, decoded=w)
        st.qwin.copy_(q.roll(t - w + 1, 0))
        st.len_host = max(lens)
    st.score_window(t)
    for i, n in enumerate(lens):
        for j in range(2):
            ref = score(q[:, 0, i, j * g:(j + 1) * g].double(), values(K[0, i, j, :n]), 1 / math.sqrt(d))
            err = (st.S[0, i, j, :n - w].cpu().double() - ref).abs()
            assert (err <= 2.0 ** -20).all(), (i, j, err.max().item())


@pytest.mark.parametrize("dtype,d,g,params", FORMS[:8])
@pytest.mark.parametrize("power", [100, 118, 121])
def test_window_score_of_huge_queries(dtype, d, g, params, power):
    _score_case(dtype, d, g, params, power, False)


@pytest.mark.parametrize("dtype,d,g,params", [f for f in FORMS[:8] if f[0] == "bf16" or f[3]])
@pytest.mark.parametrize("power", [100, 118, 121])
def test_window_score_of_huge_queries_behind_decode_steps(dtype, d, g, params, power):
    _score_case(dtype, d, g, params, power, True)

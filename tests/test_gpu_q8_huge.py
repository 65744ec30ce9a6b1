"""8-bit caches under huge queries: a query times a code may pass 2^128 where the logit, with the row's scale, does not."""
import math

import pytest
import torch

from paper_2512_00504_amd import make_config
from paper_2512_00504_amd.state import DecodeState, Q8DecodeState, SharedPrefix

from planted import DT, rows, score
from q8_reference import values
from test_gpu_prefix import _own
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


@pytest.mark.parametrize("d,g", [(64, 4), (128, 2), (64, 9), (128, 16)])
@pytest.mark.parametrize("power", [5, 12, 21, 40, 100, 118, 121])
@pytest.mark.parametrize("w", [8, 40])
def test_fp32_window_score_takes_statistics_of_its_own_logits(d, g, power, w):
    # The decode step forms logits from bf16 parts of the queries, the score from 32-bit products: two roundings of a logit of 2^power.  Probabilities
    # are below 1 (and 2^-20) for every size all the same, and a row's sum over all of its keys is 1: with the w newest keys far below, over the
    # candidates (up to the logits' rounding, 2^(power - 20) and less where they are ordinary).
    b, s, n, cap = 64, 48, 112, 128
    st = Q8DecodeState(make_config(1, 1, g, 1, d, b, w, s, cap, "f32"))
    gen = torch.Generator().manual_seed(power + d)
    K, V = rows(gen, "f32", 1, 1, 1, cap, d), rows(gen, "f32", 1, 1, 1, cap, d)
    q = torch.randn(w, 1, 1, 1, d, generator=gen).expand(w, 1, 1, g, d).contiguous()   # one query for all heads: the largest of them is each of them
    K[..., 0], q[..., 0] = 1.0, 8.0
    K[0, 0, 0, n - w:, 0] = -1.0                           # the window's own keys: lower by 16 and more
    K[0, 0, 0, n - w:, 1:] = 0.0
    q = q * 2.0 ** power
    t = 2 * w + 3
    _fill(st, K, V, [n - w], b, since=t - w + 1)
    for k in range(w):
        kn, vn = K[:, :, :, n - w + k].contiguous(), V[:, :, :, n - w + k].contiguous()
        st.attend_decode(q[k].cuda(), kn.cuda(), vn.cuda(), t - w + 1 + k)
    st.score_window(t)
    S = st.S[0, 0, 0, :n - w].cpu().double()
    qw, kv = q[:, 0, 0].double(), values(K[0, 0, 0, :n])
    ref = score(qw, kv, 1 / math.sqrt(d))
    off = min(1.0, 2.0 ** (power + 6 - 20))                # logits of up to 2^(power + 6)
    assert (S <= 1 + 2.0 ** -20).all() and abs(S.sum().item() - ref.sum().item()) <= max(2.0 ** -18, off if power < 10 else 2.0 ** -18), (S.sum(), ref.sum())
    if power >= 40:
        assert ((S - ref).abs() <= 2.0 ** -20).all()


@pytest.mark.parametrize("dtype,d,g,params", [f for f in FORMS[:8] if f[0] == "f32" and not f[3]])
@pytest.mark.parametrize("power", [100, 118, 121])
def test_window_score_of_huge_fp32_queries_behind_decode_steps(dtype, d, g, params, power):
    _score_case(dtype, d, g, params, power, True)


@pytest.mark.parametrize("cls", [DecodeState, Q8DecodeState])
@pytest.mark.parametrize("dtype,d,g,params", FORMS)
@pytest.mark.parametrize("power", [100, 118, 121])
@pytest.mark.parametrize("P", [33, 3000])
def test_the_largest_logit_of_prefix_and_own_rows_takes_all(cls, dtype, d, g, params, power, P):
    lens, cap = [40, 0, 200, 255], 256
    st = cls(make_config(1, 4, 2 * g, 2, d, 64, 8, 16, cap, dtype), params=params)
    gen = torch.Generator().manual_seed(power + P)
    K, V = rows(gen, dtype, 1, 4, 2, cap, d), rows(gen, dtype, 1, 4, 2, cap, d)
    q = rows(gen, dtype, 1, 4, 2 * g, d) * 2.0 ** power
    pk, pv = rows(gen, dtype, 1, 2, P, d), rows(gen, dtype, 1, 2, P, d)
    pk[:, :, P - 1] *= 2                                   # (so that some heads have it in the last piece)
    _own(st, K, V, lens, 48)
    out = st.attend_decode(q.cuda(), None, None, 5, prefix=SharedPrefix(st, pk.cuda(), pv.cuda())).cpu().double()
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -23
    held = values if cls is Q8DecodeState else lambda x: x.double()
    for i, n in enumerate(lens):
        for j in range(2):
            k, v = torch.cat([held(K[0, i, j, :n]), pk[0, j].double()]), torch.cat([held(V[0, i, j, :n]), pv[0, j].double()])
            best = v[(q[0, i, j * g:(j + 1) * g].double() @ k.T).argmax(dim=-1)]
            assert ((out[0, i, j * g:(j + 1) * g] - best).abs() <= half * best.abs()).all(), (i, j)

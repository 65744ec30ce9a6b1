"""Attention over a prefix that sequences share, joined with their own caches, against 64 bits."""
import math

import pytest
import torch

import paper_2512_00504_amd as P
from paper_2512_00504_amd import make_config
from paper_2512_00504_amd.state import DecodeState, Q8DecodeState, SharedPrefix, k_rows_to_cache

from q8_reference import joint, rounding, values
from test_gpu_q8 import DT, _fill, _rows, _token

pytestmark = pytest.mark.gpu


def _make(cls, L=1, B=1, hkv=2, g=2, d=64, dtype="bf16", b=16, w=4, s=8, cap=64, params=None):
    return cls(make_config(L, B, hkv * g, hkv, d, b, w, s, cap, dtype), params=params)


def _own(st, K, V, lens, n_tiled):
    if isinstance(st, Q8DecodeState):
        _fill(st, K, V, lens, n_tiled)
        return
    for i, n in enumerate(lens):
        k, v = K[:, i].clone(), V[:, i].clone()
        k[:, :, n:] = float("nan"); v[:, :, n:] = float("nan")
        st.K[:, i] = k_rows_to_cache(k, min(n_tiled, n // 16 * 16)).cuda()
        st.V[:, i] = v.cuda()
    rec = torch.tensor([[n, 5, 0, min(n_tiled, n // 16 * 16)] for n in lens], dtype=torch.int32)
    st.d_state.copy_(rec.expand(st.cfg.n_layers, -1, -1))
    st._set_host(list(lens), [0] * len(lens))


def _check(st, out, K, V, q, kn, vn, lens, prefixes, append):
    """prefixes: (K [L,hkv,n,d], V, first, count) each."""
    cfg = st.cfg
    g, d, scale = cfg.n_q_heads // cfg.n_kv_heads, cfg.head_dim, 1 / math.sqrt(cfg.head_dim)
    dtype = "f32" if cfg.dtype == 0 else "bf16"
    own = values if isinstance(st, Q8DecodeState) else lambda x: x.double()
    out = out.cpu().double()
    for l in range(cfg.n_layers):
        for i, n in enumerate(lens):
            for j in range(cfg.n_kv_heads):
                parts = [(own(K[l, i, j, :n]), own(V[l, i, j, :n]))]
                if append:
                    parts.append((own(kn[l, i, j:j + 1]), own(vn[l, i, j:j + 1])))
                parts += [(k[l, j].double(), v[l, j].double()) for k, v, first, count in prefixes if first <= i < first + count]
                heads = slice(j * g, (j + 1) * g)
                ref, tol = joint(q[l, i, heads].double(), parts, scale)
                top = max([p[1].abs().max().item() for p in parts if len(p[1])], default=0.0)
                err = (out[l, i, heads] - ref).abs()
                assert (err <= tol + rounding(dtype, ref, top)).all(), (l, i, j, n, err.max().item(), tol)


def _case(cls, dtype, d, g, B, rows, lens=None, L=1, hkv=2, cap=64, append=True, params=None, seed=0, first=0, count=None):
    lens = lens or [(7 * i) % (cap - 1) for i in range(B)]
    st = _make(cls, L=L, B=B, hkv=hkv, g=g, d=d, dtype=dtype, cap=cap, params=params)
    gen = torch.Generator().manual_seed(seed + rows + d)
    K, V = _rows(gen, dtype, L, B, hkv, cap, d), _rows(gen, dtype, L, B, hkv, cap, d)
    _own(st, K, V, lens, 16)
    q, kn, vn = _token(gen, dtype, L, B, hkv, g, d)
    pk, pv = _rows(gen, dtype, L, hkv, rows, d), _rows(gen, dtype, L, hkv, rows, d)
    prefix = SharedPrefix(st, pk.cuda(), pv.cuda(), first, count)
    out = st.attend_decode(q.cuda(), kn.cuda() if append else None, vn.cuda() if append else None, 5, prefix=prefix)
    _check(st, out, K, V, q, kn, vn, lens, [(pk, pv, first, prefix.count)], append)
    return st, prefix


SHAPES = [("bf16", 128, 7), ("bf16", 128, 1), ("bf16", 64, 5), ("f32", 64, 4), ("f32", 128, 2), ("bf16", 48, 3), ("f32", 20, 2), ("bf16", 64, 17)]


@pytest.mark.parametrize("cls", [DecodeState, Q8DecodeState])
@pytest.mark.parametrize("dtype,d,g", SHAPES)
@pytest.mark.parametrize("rows", [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 255, 256, 257, 700])
def test_prefix_of_all_lengths(cls, dtype, d, g, rows):
    if cls is Q8DecodeState and d % 16:
        pytest.skip("rows of whole pieces only")
    _case(cls, dtype, d, g, 3, rows)


@pytest.mark.parametrize("dtype,d,g", [("bf16", 128, 7), ("bf16", 64, 3), ("f32", 64, 2)])
@pytest.mark.parametrize("B", [1, 2, 5, 9, 16, 33, 64, 150])
def test_prefix_of_batches(dtype, d, g, B):
    _case(DecodeState, dtype, d, g, B, 300)


@pytest.mark.parametrize("dtype,d,g,B,rows,L", [("bf16", 128, 7, 4, 5000, 1), ("bf16", 128, 5, 40, 3001, 2), ("f32", 64, 4, 3, 4999, 1), ("bf16", 64, 16, 20, 2500, 1),
                                                ("f32", 128, 7, 30, 1500, 1), ("bf16", 128, 8, 1, 20000, 1)])
def test_long_prefix(dtype, d, g, B, rows, L):
    _case(DecodeState, dtype, d, g, B, rows, L=L)


@pytest.mark.parametrize("cls", [DecodeState, Q8DecodeState])
def test_prefix_of_a_short_or_empty_cache_and_without_a_new_row(cls):
    for rows in (0, 40):
        _case(cls, "bf16", 128, 3, 4, rows, lens=[0, 0, 1, 40], append=False)
        _case(cls, "f32", 64, 3, 4, rows, lens=[0, 1, 2, 40], append=True)


@pytest.mark.parametrize("cls", [DecodeState, Q8DecodeState])
@pytest.mark.parametrize("params", [{"force_generic": 1}, {"attend_splits": 2}, {"attend_waves": 8}, {"attend_waves": 4}])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 128)])
def test_prefix_in_every_form(cls, params, dtype, d):
    _case(cls, dtype, d, 3, 4, 333, lens=[200, 17, 255, 0], cap=256, params=params)


@pytest.mark.parametrize("cls", [DecodeState, Q8DecodeState])
def test_prefix_with_own_units_cut_over_workgroups_and_many_units(cls):
    _case(cls, "bf16", 128, 7, 2, 1000, lens=[2000, 900], cap=2048)
    _case(cls, "bf16", 128, 2, 280, 70)


@pytest.mark.parametrize("cls", [DecodeState, Q8DecodeState])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64), ("bf16", 48)])
def test_prompts_of_a_batch_each_with_its_sequences(cls, dtype, d):
    # sequence 0 has no prefix, 1 .. 3 share one, 4 .. 5 another, 6 none
    B, hkv, g, lens = 7, 2, 3, [30, 0, 17, 40, 5, 33, 20]
    st = _make(cls, L=2, B=B, hkv=hkv, g=g, d=d, dtype=dtype)
    gen = torch.Generator().manual_seed(1)
    K, V = _rows(gen, dtype, 2, B, hkv, 64, d), _rows(gen, dtype, 2, B, hkv, 64, d)
    q, kn, vn = _token(gen, dtype, 2, B, hkv, g, d)
    a = [_rows(gen, dtype, 2, hkv, 900, d) for _ in range(2)]
    b = [_rows(gen, dtype, 2, hkv, 65, d) for _ in range(2)]
    first = SharedPrefix(st, a[0].cuda(), a[1].cuda(), 1, 3)
    second = SharedPrefix(st, b[0].cuda(), b[1].cuda(), 4, 2, part=first)
    with pytest.raises(ValueError):
        SharedPrefix(st, torch.zeros(2, hkv, 100000, d), torch.zeros(2, hkv, 100000, d), 4, 2, part=first)
    for _ in range(2):                                     # a second step finds what the first left
        _own(st, K, V, lens, 16)
        second.attend(q.cuda())
        out = st.attend_decode(q.cuda(), kn.cuda(), vn.cuda(), 5, prefix=first)
        _check(st, out, K, V, q, kn, vn, lens, [(a[0], a[1], 1, 3), (b[0], b[1], 4, 2)], True)


def test_prefix_capacity_beyond_32_bits_of_offset():
    # the last head's rows begin 4.4 GB into K and V; what lies behind the rows of each head is not read (NaN where a tile ends)
    d, hkv, g, B, rows, cap = 128, 8, 2, 2, 70, 2460000
    st = _make(DecodeState, B=B, hkv=hkv, g=g, d=d)
    gen = torch.Generator().manual_seed(4)
    K, V = _rows(gen, "bf16", 1, B, hkv, 64, d), _rows(gen, "bf16", 1, B, hkv, 64, d)
    _own(st, K, V, [20, 30], 16)
    q, kn, vn = _token(gen, "bf16", 1, B, hkv, g, d)
    pk, pv = _rows(gen, "bf16", 1, hkv, rows, d), _rows(gen, "bf16", 1, hkv, rows, d)
    Kp, Vp = (torch.empty(1, hkv, cap, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for x, y in ((Kp, pk), (Vp, pv)):
        x[:, :, :rows], x[:, :, rows:rows + 512] = y.cuda(), float("nan")
    part = torch.zeros(st.ctx.prefix_bytes(rows), dtype=torch.uint8, device="cuda")
    st.ctx.prefix_attend(q.cuda(), Kp, Vp, rows, cap, 0, B, part)
    st.ctx.attend_decode_prefix(q.cuda(), kn.cuda(), vn.cuda(), st.K, st.V, st.pos, 5, st.qwin, st.d_state, 30, part, st.out, st.workspace)
    _check(st, st.out, K, V, q, kn, vn, [20, 30], [(pk, pv, 0, B)], True)


@pytest.mark.parametrize("dtype,d,params", [("bf16", 128, None), ("f32", 64, None), ("bf16", 64, None), ("f32", 128, None), ("bf16", 128, {"force_generic": 1})])
def test_prefix_hard_logits(dtype, d, params):
    # huge logits in either part take all; a prefix whose logits are all -inf counts for nothing, +inf or NaN in it gives NaN
    B, g, lens = 6, 2, [40] * 6
    st = _make(DecodeState, B=B, hkv=1, g=g, d=d, dtype=dtype, params=params)
    gen = torch.Generator().manual_seed(9)
    K, V = (torch.randn(1, B, 1, 64, d, generator=gen).to(DT[dtype]) for _ in range(2))
    K[..., :4] = 0.0                                       # channels that only the prefix has
    q = torch.randn(1, B, g, d, generator=gen).to(DT[dtype])
    pk, pv = (torch.randn(1, 1, 100, d, generator=gen).to(DT[dtype]) for _ in range(2))
    pk[..., :4] = 0.0
    pk[0, 0, 77, 0] = 1.0                                  # row 77 answers channel 0, and so on
    pk[0, 0, :, 1] = 1.0
    pk[0, 0, 50, 2] = 1.0
    q[..., :4] = 0.0
    q[0, 0, :, 0] = 2.0 ** 40                              # one prefix row takes all
    q[0, 1, :, 1] = float("-inf")                          # the whole prefix: 0 * inf is NaN in the own rows, so -2^120 instead
    q[0, 1, :, 1] = -2.0 ** 120
    q[0, 2] *= 2.0 ** 40                                   # the largest of all
    q[0, 3, :, 2] = -2.0 ** 120                            # one row of it
    q[0, 4, :, 2] = float("nan")
    _own(st, K, V, lens, 16)
    prefix = SharedPrefix(st, pk.cuda(), pv.cuda())
    out = st.attend_decode(q.cuda(), None, None, 5, prefix=prefix).cpu().double()
    assert ((out[0, 0] - pv[0, 0, 77].double()).abs() <= 2.0 ** -8 * pv[0, 0, 77].double().abs()).all()
    scale = 1 / math.sqrt(d)
    allK = torch.cat([K[0, 2, 0, :40], pk[0, 0]]).double()
    allV = torch.cat([V[0, 2, 0, :40], pv[0, 0]]).double()
    best = (q[0, 2].double() @ allK.T).argmax(dim=-1)
    assert ((out[0, 2] - allV[best]).abs() <= 2.0 ** -8 * allV[best].abs()).all()
    assert torch.isnan(out[0, 4]).all()
    some = [x for x in range(100) if x != 50]
    for i, parts in ((1, [(K[0, 1, 0, :40].double()[:, 4:], V[0, 1, 0, :40].double())]),
                     (3, [(K[0, 3, 0, :40].double()[:, 4:], V[0, 3, 0, :40].double()), (pk[0, 0, some].double()[:, 4:], pv[0, 0, some].double())]),
                     (5, [(K[0, 5, 0, :40].double(), V[0, 5, 0, :40].double()), (pk[0, 0].double(), pv[0, 0].double())])):
        qi = q[0, i].double()[:, 4:] if i != 5 else q[0, i].double()
        ref, tol = joint(qi, parts, scale)
        assert ((out[0, i] - ref).abs() <= tol + rounding(dtype, ref, 5.0)).all(), i
    # all -inf, and nothing of its own: no number
    st2 = _make(DecodeState, B=1, hkv=1, g=g, d=d, dtype=dtype, params=params)
    _own(st2, K[:, :1], V[:, :1], [0], 0)
    pk2 = torch.ones(1, 1, 20, d).to(DT[dtype])
    q2 = torch.zeros(1, 1, g, d).to(DT[dtype])
    q2[..., 0] = float("-inf")
    out = st2.attend_decode(q2.cuda(), None, None, 5, prefix=SharedPrefix(st2, pk2.cuda(), pk2.cuda()))
    assert torch.isnan(out.float()).all()
    # and with rows of its own that are finite: those alone (the infinite query meets zeros nowhere: own keys are negative there)
    K3 = torch.randn(1, 1, 1, 64, d, generator=gen).to(DT[dtype])
    K3[..., 0] = -1.0
    _own(st2, K3, V[:, :1], [30], 16)
    out = st2.attend_decode(q2.cuda(), None, None, 5, prefix=SharedPrefix(st2, pk2.cuda(), pk2.cuda()))
    assert torch.isnan(out.float()).all()                  # +inf in the own rows: no number either


@pytest.mark.parametrize("cls", [DecodeState, Q8DecodeState])
def test_scores_are_those_of_the_own_rows(cls):
    # the same window, with and without a prefix: the local score does not see it
    L, B, hkv, g, d, b, w, s = 1, 2, 2, 4, 128, 32, 8, 16
    gen = torch.Generator().manual_seed(6)
    toks = [[x.cuda() for x in _token(gen, "bf16", L, B, hkv, g, d)] for _ in range(b + s)]
    pk, pv = _rows(gen, "bf16", L, hkv, 200, d).cuda(), _rows(gen, "bf16", L, hkv, 200, d).cuda()
    got = []
    for shared in (False, True):
        st = _make(cls, L=L, B=B, hkv=hkv, g=g, d=d, b=b, w=w, s=s)
        prefix = SharedPrefix(st, pk, pv) if shared else None
        for t, tok in enumerate(toks):
            st.attend_decode(*tok, t, prefix=prefix)
        st.score_window(b + s - 1)
        got.append(st.S.clone())
    assert torch.equal(*got)


@pytest.mark.parametrize("cls,dtype,d,g,B,rows", [(DecodeState, "bf16", 128, 7, 4, 3000), (Q8DecodeState, "bf16", 128, 5, 16, 500), (DecodeState, "f32", 64, 2, 3, 900)])
def test_recorded_steps_replay_as_eager_ones(cls, dtype, d, g, B, rows):
    st = _make(cls, B=B, hkv=2, g=g, d=d, dtype=dtype)
    gen = torch.Generator().manual_seed(8)
    K, V = _rows(gen, dtype, 1, B, 2, 64, d), _rows(gen, dtype, 1, B, 2, 64, d)
    lens = [10 + i for i in range(B)]
    prefix = SharedPrefix(st, _rows(gen, dtype, 1, 2, rows, d).cuda(), _rows(gen, dtype, 1, 2, rows, d).cuda())
    toks = [[x.cuda() for x in _token(gen, dtype, 1, B, 2, g, d)] for _ in range(3)]
    want = []
    for tok in toks:
        _own(st, K, V, lens, 16)
        want.append(st.attend_decode(*tok, 5, prefix=prefix).clone())
    ins = [x.clone() for x in toks[0]]
    _own(st, K, V, lens, 16)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        st.attend_decode(*ins, 5, prefix=prefix)
    for i in (0, 1, 2, 1):
        for x, y in zip(ins, toks[i]):
            x.copy_(y)
        prefix.part.fill_(255)                             # (NaN: everything that counts is written again)
        st.out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(st.out.view(torch.uint8), want[i].view(torch.uint8)), i


@pytest.mark.parametrize("cls", [DecodeState, Q8DecodeState])
def test_prefix_of_another_shape_or_state_is_refused(cls):
    st, other = (cls(make_config(1, 2, 4, 2, 64, 16, 4, 8, 64, "bf16")) for _ in range(2))
    k = torch.zeros(1, 2, 40, 64)
    for bad in ((k[0], k[0]), (k[:, :1], k[:, :1]), (k[..., :32], k[..., :32]), (k, k[:, :, :39]), (torch.cat([k, k]), torch.cat([k, k]))):
        with pytest.raises(ValueError):
            SharedPrefix(st, *bad)
    short, long = SharedPrefix(st, k[:, :, :1], k[:, :, :1], count=1), torch.zeros(1, 2, 9000, 64)
    with pytest.raises(ValueError):
        SharedPrefix(st, long, long, first=1, part=short)
    with pytest.raises(ValueError):
        SharedPrefix(other, k, k, part=short)
    q, kn, vn = (torch.zeros(1, 2, n, 64, dtype=torch.bfloat16, device="cuda") for n in (4, 2, 2))
    with pytest.raises(ValueError):
        other.attend_decode(q, kn, vn, 0, prefix=short)
    with pytest.raises(P.GkvError):
        SharedPrefix(st, k, k, first=1, count=2).attend(q)

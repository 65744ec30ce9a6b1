"""Decode, shared prefixes and window scores on inputs whose result shows every edge row, see planted.py."""
import math

import pytest
import torch

from paper_2512_00504_amd import make_config
from paper_2512_00504_amd.state import DecodeState, Q8DecodeState, SharedPrefix, k_cache_to_rows, k_rows_to_cache

from planted import DT, attend, bound, direction, height, plant, queries, rows, score, score_bound
from q8_reference import F8, held as codes, values
from test_gpu_prefix import _own
from test_gpu_q8 import _fill

pytestmark = pytest.mark.gpu


def _make(cls, L, B, hkv, g, d, dtype, cap, b=16, w=4, s=8, params=None):
    return cls(make_config(L, B, hkv * g, hkv, d, b, w, s, cap, dtype), params=params)


def _case(cls, dtype, d, g, lens, prefix, cap=64, L=1, hkv=2, n_tiled=16, append=True, params=None, seed=0, check=None):
    """One decode step of sequences with `lens` rows and a shared prefix of `prefix` rows (None: no prefix) against 64 bits."""
    gen = torch.Generator().manual_seed(seed + d + g + (prefix or 0) + sum(lens))
    B, scale = len(lens), 1 / math.sqrt(d)
    st = _make(cls, L, B, hkv, g, d, dtype, cap, params=params)
    u = direction(gen, d)
    K, V = rows(gen, dtype, L, B, hkv, cap, d), rows(gen, dtype, L, B, hkv, cap, d)
    q = queries(gen, u, dtype, L, B, hkv * g)
    kn, vn = rows(gen, dtype, L, B, hkv, d), rows(gen, dtype, L, B, hkv, d)
    P = prefix or 0
    pk, pv = rows(gen, dtype, L, hkv, P, d), rows(gen, dtype, L, hkv, P, d)
    for i, n in enumerate(lens):
        for at in {0, n - 1} if n else ():
            plant(K[:, i], u, at, height(n + P))
        kn[:, i] = (u * height(n + P) / math.sqrt(d)).to(DT[dtype])
    for at in {0, P - 1} if P else ():
        plant(pk, u, at, height(P + sum(lens) // B))
    _own(st, K, V, lens, n_tiled)
    shared = None if prefix is None else SharedPrefix(st, pk.cuda(), pv.cuda())
    out = st.attend_decode(q.cuda(), kn.cuda() if append else None, vn.cuda() if append else None, 5, prefix=shared).cpu().double()
    held = values if cls is Q8DecodeState else lambda x: x.double()
    for l, i, j in check or [(l, i, j) for l in range(L) for i in range(B) for j in range(hkv)]:
        n, heads = lens[i], slice(j * g, (j + 1) * g)
        parts = [(held(K[l, i, j, :n]), held(V[l, i, j, :n])), (pk[l, j].double(), pv[l, j].double())]
        if append:
            parts.append((held(kn[l, i, j:j + 1]), held(vn[l, i, j:j + 1])))
        k, v = (torch.cat([x[y] for x in parts]) for y in (0, 1))
        if not len(k):
            assert (out[l, i, heads] == 0).all()
            continue
        ref = attend(q[l, i, heads].double(), k, v, scale)
        tol = bound(q[l, i, heads].double(), k, v, ref, scale, dtype)
        err = (out[l, i, heads] - ref).abs()
        assert (err <= tol).all(), (l, i, j, n, P, (err / tol).max().item())


SHAPES = [("bf16", 128, 7), ("bf16", 128, 16), ("bf16", 64, 5), ("f32", 64, 4), ("f32", 128, 3), ("bf16", 48, 3), ("f32", 32, 2), ("bf16", 64, 17)]


@pytest.mark.parametrize("cls", [DecodeState, Q8DecodeState])
@pytest.mark.parametrize("dtype,d,g", SHAPES)
def test_prefix_ends(cls, dtype, d, g):
    for P in (0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 700):
        _case(cls, dtype, d, g, [20, 0, 33, 1], P, append=P % 3 != 0)


@pytest.mark.parametrize("dtype,d,g,B,P,L", [("bf16", 128, 7, 4, 5000, 1), ("bf16", 128, 5, 40, 3001, 2), ("f32", 64, 4, 3, 4999, 1), ("bf16", 64, 16, 20, 2500, 1),
                                             ("f32", 128, 7, 30, 1500, 1), ("bf16", 128, 8, 1, 20000, 1), ("bf16", 128, 7, 8, 3003, 1), ("f32", 64, 2, 64, 1033, 1)])
def test_long_prefix_ends(dtype, d, g, B, P, L):
    _case(DecodeState, dtype, d, g, [(7 * i + 3) % 63 for i in range(B)], P, L=L)
    _case(Q8DecodeState, dtype, d, g, [(11 * i) % 63 for i in range(B)], P, L=L, append=False)


@pytest.mark.parametrize("cls", [DecodeState, Q8DecodeState])
@pytest.mark.parametrize("params", [{"force_generic": 1}, {"attend_splits": 2}, {"attend_splits": 64}, {"attend_waves": 8}, {"attend_waves": 4}])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 128)])
def test_ends_in_every_form(cls, params, dtype, d):
    for P in (None, 333):
        _case(cls, dtype, d, 3, [200, 17, 255, 0, 32, 1], P, cap=256, n_tiled=4096, params=params)


@pytest.mark.parametrize("dtype,d,g", SHAPES[:7])
@pytest.mark.parametrize("n_tiled", [0, 48, 4096])
def test_decode_ends_on_8_bit_caches(dtype, d, g, n_tiled):
    if d % 16 == 0:
        for append in (True, False):
            _case(Q8DecodeState, dtype, d, g, [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 250, 255], None, cap=256, n_tiled=n_tiled, append=append)


@pytest.mark.parametrize("cls", [DecodeState, Q8DecodeState])
@pytest.mark.parametrize("dtype,d,g", [("bf16", 128, 7), ("f32", 64, 4), ("bf16", 64, 2), ("f32", 128, 2)])
def test_decode_ends_of_long_and_of_many_units(cls, dtype, d, g):
    _case(cls, dtype, d, g, [3000, 17, 1999, 0, 3001], None, cap=3008, n_tiled=1024)
    _case(cls, dtype, d, g, [700 + 13 * i for i in range(70)], None, cap=1664, n_tiled=512, check=[(0, i, i % 2) for i in range(0, 70, 7)])
    for B in (85, 87, 173):                                # 255, 261, 519 units
        _case(cls, dtype, d, g, [i % 96 for i in range(B)], None, cap=96, hkv=3)


@pytest.mark.parametrize("cls", [DecodeState, Q8DecodeState])
@pytest.mark.parametrize("params", [{"attend_tile": 32}, {"attend_waves": 16}, {"attend_tile": 32, "attend_splits": 3}])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64), ("f32", 128)])
def test_ends_with_the_other_knobs(cls, params, dtype, d):
    for P in (None, 1, 777):
        _case(cls, dtype, d, 2, [200, 17, 1000, 0, 32, 1], P, cap=1024, n_tiled=512, params=params)


@pytest.mark.parametrize("cls", [DecodeState, Q8DecodeState])
@pytest.mark.parametrize("dtype,d,g", [("bf16", 128, 7), ("f32", 64, 2), ("bf16", 64, 3)])
def test_cut_units_joined_with_many_pieces(cls, dtype, d, g):
    for P in (2049, 20000):
        _case(cls, dtype, d, g, [3000, 900], P, cap=3008, n_tiled=1024)
        _case(cls, dtype, d, g, [2000], P, cap=3008, n_tiled=0, hkv=1, append=False)


# ---- larger than the memory-side cache: what is read once is asked for in another way ----------------
@pytest.mark.parametrize("dtype,d,g,B,P", [("bf16", 128, 7, 4, 33000), ("bf16", 128, 7, 8, 33001), ("bf16", 128, 7, 16, 32999), ("bf16", 64, 3, 10, 65999),
                                           ("bf16", 64, 4, 16, 66000), ("bf16", 64, 4, 32, 65970), ("f32", 128, 5, 2, 16500), ("f32", 128, 5, 12, 16501),
                                           ("f32", 128, 4, 32, 16499), ("f32", 64, 8, 4, 33003), ("f32", 64, 8, 8, 33007), ("f32", 64, 8, 16, 32993)])
def test_prefix_beyond_the_memory_side_cache(dtype, d, g, B, P):
    # 16 units of K and V above 256 MiB; one, two and up to four blocks of 32 query rows
    L, hkv, scale = 2, 8, 1 / math.sqrt(d)
    assert L * hkv * P * 2 * d * (4 if dtype == "f32" else 2) > 256 << 20 and B * g <= 128
    gen, dev = torch.Generator().manual_seed(P), torch.Generator("cuda").manual_seed(P)
    st = _make(DecodeState, L, B, hkv, g, d, dtype, 64)
    u = direction(gen, d)
    q = queries(gen, u, dtype, L, B, hkv * g)
    pk, pv = (torch.randn(L, hkv, P, d, generator=dev, device="cuda").to(DT[dtype]) for _ in range(2))
    for at in (0, P // 2, P - 1):
        plant(pk, u.cuda(), at, height(P))
    K, V = rows(gen, dtype, L, B, hkv, 64, d), rows(gen, dtype, L, B, hkv, 64, d)
    lens = [20 + i for i in range(B)]
    for i, n in enumerate(lens):
        plant(K[:, i], u, n - 1, height(P))
    _own(st, K, V, lens, 16)
    out = st.attend_decode(q.cuda(), None, None, 5, prefix=SharedPrefix(st, pk, pv)).cpu().double()
    for l, j in ((0, 0), (1, hkv - 1)):
        heads = slice(j * g, (j + 1) * g)
        for i in sorted({0, B // 2, B - 1}):
            k, v = (torch.cat([x[l, i, j, :lens[i]].double(), y[l, j].cpu().double()]) for x, y in ((K, pk), (V, pv)))
            ref = attend(q[l, i, heads].double(), k, v, scale)
            err, tol = (out[l, i, heads] - ref).abs(), bound(q[l, i, heads].double(), k, v, ref, scale, dtype)
            assert (err <= tol).all(), (l, j, i, (err / tol).max().item())


@pytest.mark.parametrize("dtype,d,g,w,B", [("bf16", 128, 8, 16, 250), ("bf16", 128, 5, 32, 250), ("bf16", 128, 4, 8, 250), ("bf16", 64, 7, 16, 490), ("bf16", 64, 2, 32, 490),
                                           ("f32", 128, 3, 8, 250), ("f32", 64, 4, 16, 490)])
def test_codes_beyond_the_memory_side_cache(dtype, d, g, w, B):
    # w decode steps and the window score behind them (with the steps' statistics, and without) on more than 256 MiB of K's codes
    hkv, b, s, cap, scale = 8, 1024, 64, 1088, 1 / math.sqrt(d)
    assert B * hkv * cap * d > 256 << 20
    gen, dev = torch.Generator().manual_seed(d + g), torch.Generator("cuda").manual_seed(d + g)
    st = _make(Q8DecodeState, 1, B, hkv, g, d, dtype, cap, b=b, w=w, s=s)
    n0, t0, u = cap - w, 7, direction(gen, d)
    for cache, which in ((st.K8, 0), (st.V8, 1)):
        x = torch.randint(2, 7, (1, B, hkv, cap, 1), generator=dev, device="cuda")
        for i in range(0, B, 50):
            y = torch.randn(1, min(50, B - i), hkv, cap, d, generator=dev, device="cuda")
            cache.view(torch.uint8)[:, i:i + 50] = torch.ldexp(y, x[:, i:i + 50]).to(F8).view(torch.uint8)
        st.scales[..., which] = torch.ldexp(torch.ones((), device="cuda"), -x[..., 0]).to(torch.bfloat16)
    units = [(0, 0), (1, 7), (B // 2, 3), (B - 1, 7)]
    held = {}
    for i, j in units:                                     # the first tiles as after a compaction; planted rows at both ends
        raw = st.K8[0, i, j].cpu().view(torch.uint8)
        k = k_cache_to_rows(raw, b).view(F8).double() * st.scales[0, i, j, :, :1].cpu().double()
        c = k_cache_to_rows(raw, b)
        for at in (0, n0 // 2, n0 - 1):
            one = (u * height(cap) / math.sqrt(d)).to(torch.bfloat16)[None]
            y, e = codes(one)
            c[at] = y[0].to(F8).view(torch.uint8)
            st.scales[0, i, j, at, 0] = 2.0 ** e.item()
            k[at] = torch.ldexp(y[0], e[0].double())
        st.K8.view(torch.uint8)[0, i, j] = k_rows_to_cache(c, b).cuda()
        held[i, j] = [k[:n0], (st.V8[0, i, j].cpu().double() * st.scales[0, i, j, :, 1:].cpu().double())[:n0]]
    st.d_state.copy_(torch.tensor([n0, t0, 0, b], dtype=torch.int32))
    st._set_host([n0] * B, [0] * B)
    window = []
    for t in range(t0, t0 + w):
        q = queries(gen, u, dtype, 1, B, hkv * g)
        kn, vn = rows(gen, dtype, 1, B, hkv, d), rows(gen, dtype, 1, B, hkv, d)
        if t in (t0, t0 + w - 1):
            kn[:] = (u * height(cap) / math.sqrt(d)).to(DT[dtype])
        window.append(q[0].double())
        out = st.attend_decode(q.cuda(), kn.cuda(), vn.cuda(), t)
        for i, j in units:
            held[i, j] = [torch.cat([x, values(y[0, i, j][None])]) for x, y in zip(held[i, j], (kn, vn))]
            if t in (t0, t0 + w - 1):
                k, v = held[i, j]
                qh = q[0, i, j * g:(j + 1) * g].double()
                ref = attend(qh, k, v, scale)
                err, tol = (out[0, i, j * g:(j + 1) * g].cpu().double() - ref).abs(), bound(qh, k, v, ref, scale, dtype)
                assert (err <= tol).all(), (t, i, j, (err / tol).max().item())
    for reuse in (1, 0):
        st.ctx.set_param("score_reuse_stats", reuse)
        st.S.fill_(-7.0)
        st.score_window(t0 + w - 1)
        for i, j in units:
            qw = torch.stack([x[i, j * g:(j + 1) * g] for x in window])
            ref, tol = score(qw, held[i, j][0], scale), score_bound(qw, held[i, j][0], scale)
            err = ((st.S[0, i, j, :n0].cpu().double() - ref) / ref).abs()
            assert (err <= tol).all(), (reuse, i, j, (err / tol).max().item())
            assert (st.S[0, i, j, n0:] == -7).all()


# ---- window scores -----------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,d,g,w", [("bf16", 128, 7, 16), ("bf16", 64, 5, 32), ("f32", 64, 4, 8), ("f32", 128, 2, 16), ("bf16", 128, 5, 32), ("bf16", 128, 16, 7),
                                         ("bf16", 64, 1, 1), ("bf16", 48, 3, 5), ("bf16", 128, 9, 16)])
def test_window_score_ends_on_8_bit_caches(dtype, d, g, w):
    b, s, scale = 64, max(w, 16), 1 / math.sqrt(d)
    lens = [64, 65, 70, 79, 64 + s, 100]
    cap = -(-max(max(lens), b + s) // 32) * 32 + 32
    st = _make(Q8DecodeState, 1, len(lens), 2, g, d, dtype, cap, b=b, w=w, s=s)
    gen = torch.Generator().manual_seed(d + g + w)
    u = direction(gen, d)
    K, V = rows(gen, dtype, 1, len(lens), 2, cap, d), rows(gen, dtype, 1, len(lens), 2, cap, d)
    q = queries(gen, u, dtype, w, 1, len(lens), 2 * g)
    for i, n in enumerate(lens):
        for at in {0, n - w - 1, n - w, n - 1}:
            plant(K[:, i], u, at, height(n))
    t = 2 * w + 3
    _fill(st, K, V, lens, b, since=t - w + 1, decoded=w)
    for k in range(w):
        st.qwin[(t - w + 1 + k) % w] = q[k].cuda()
    st.len_host = max(lens)
    st.S.fill_(-7.0)
    st.score_window(t)
    for i, n in enumerate(lens):
        for j in range(2):
            if n <= b:
                assert (st.S[0, i, j] == -7).all()
                continue
            qw, k = q[:, 0, i, j * g:(j + 1) * g].double(), values(K[0, i, j, :n])
            ref, tol = score(qw, k, scale), score_bound(qw, k, scale)
            err = ((st.S[0, i, j, :n - w].cpu().double() - ref) / ref).abs()
            assert (err <= tol).all(), (i, j, n, (err / tol).max().item())
            assert (st.S[0, i, j, n - w:] == -7).all()


# ---- a prefix that weighs nothing ---------------------------------------------------------------------
@pytest.mark.parametrize("cls", [DecodeState, Q8DecodeState])
@pytest.mark.parametrize("params", [None, {"force_generic": 1}, {"attend_splits": 2}])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("P", [20, 700])
def test_prefix_whose_logits_are_all_minus_infinity_counts_for_nothing(cls, params, dtype, d, P):
    # -2^120 * 2^20 is -inf in 32 bits; the own rows have zeros in that channel
    B, hkv, g, lens, scale = 3, 1, 3, [200, 1, 40], 1 / math.sqrt(d)
    st = _make(cls, 1, B, hkv, g, d, dtype, 256, params=params)
    gen = torch.Generator().manual_seed(P)
    K, V = rows(gen, dtype, 1, B, hkv, 256, d), rows(gen, dtype, 1, B, hkv, 256, d)
    K[..., 0] = 0
    q = rows(gen, dtype, 1, B, g, d)
    pk, pv = rows(gen, dtype, 1, hkv, P, d), rows(gen, dtype, 1, hkv, P, d)
    pk[..., 0], q[..., 0] = 2.0 ** 20, -2.0 ** 120
    q[0, 2, :, 0] = 0                                      # a sequence that does see the prefix
    _own(st, K, V, lens, 16)
    out = st.attend_decode(q.cuda(), None, None, 5, prefix=SharedPrefix(st, pk.cuda(), pv.cuda())).cpu().double()
    held = values if cls is Q8DecodeState else lambda x: x.double()
    for i, n in enumerate(lens):
        k, v = held(K[0, i, 0, :n])[:, 1:], held(V[0, i, 0, :n])
        if i == 2:
            k, v = torch.cat([k, pk[0, 0].double()[:, 1:]]), torch.cat([v, pv[0, 0].double()])
        qi = q[0, i].double()[:, 1:]
        ref = attend(qi, k, v, scale)
        err, tol = (out[0, i] - ref).abs(), bound(qi, k, v, ref, scale, dtype)
        assert (err <= tol).all(), (i, (err / tol).max().item())

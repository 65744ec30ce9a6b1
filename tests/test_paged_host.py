"""What the calls on rotary positions and paged caches refuse, their sizes and frequencies: host code only."""
import math

import pytest
import torch

import paper_2512_00504_amd as P
from paper_2512_00504_amd.state import PagedDecodeState

LIB = P.load_library()
AT = 1 << 20                                  # an aligned address that is never dereferenced: every call here fails on the host
INVALID, SHAPE, WORKSPACE, OVERFLOW = 1, 2, 3, 6


def _ctx(**kw):
    base = dict(n_layers=2, batch=3, n_q_heads=8, n_kv_heads=2, head_dim=64, budget=64, window=8, interval=16, capacity=96, dtype="bf16")
    base.update(kw)
    return P.Context(P.make_config(**base))


# good arguments of each call, without context and stream; a refusal differs in one place
GOOD = {
    # q, q_stride, k, k_stride, tokens, positions, step, freq, dim, layout, amplitude, transposed, q_out, k_out
    "gkv_rotate": [AT, 0, AT, 0, 5, AT, 0, AT, 64, 0, 1.0, 0, 2 * AT, 2 * AT],
    "gkv_paged_advance": [AT, AT],
    # q, q_stride, k, k_stride, v, v_stride, tokens, d_start, d_len, positions, freq, dim, layout, amplitude, table, width, page_rows, n_pages, K, V, q_out
    "gkv_paged_append": [AT, 0, AT, 0, AT, 0, 5, AT, AT, AT, AT, 64, 0, 1.0, AT, 4, 16, 9, AT, AT, 2 * AT],
    # q, K, V, table, width, page_rows, n_pages, d_len, len_max, out, workspace
    "gkv_paged_attend_decode": [AT, AT, AT, AT, 4, 16, 9, AT, 64, AT, AT],
}
REFUSED = [
    *[("gkv_rotate", at, v, INVALID) for at, v in [(0, None), (2, None), (7, None), (12, None), (13, None), (1, 511), (1, -512), (3, 127), (4, -1), (6, -1),
                                                   (7, AT + 4), (8, 0), (8, 63), (8, 66), (8, -2), (9, 2), (9, -1),
                                                   (10, float("nan")), (10, float("inf")), (0, AT + 1), (2, AT + 3), (12, AT + 1), (13, AT + 1)]],
    ("gkv_rotate", 4, 2 ** 23, SHAPE),
    ("gkv_paged_advance", 0, None, INVALID),
    *[("gkv_paged_append", at, v, INVALID) for at, v in [(i, None) for i in (0, 2, 4, 7, 8, 10, 14, 18, 19, 20)]
      + [(1, 511), (3, 127), (5, 127), (6, -1), (10, AT + 4), (11, 0), (11, 63), (11, 66), (12, 2), (13, float("nan")), (15, 0), (16, 0), (17, 0), (15, -4), (0, AT + 1), (2, AT + 1), (4, AT + 1), (18, AT + 1), (19, AT + 1), (20, AT + 1)]],
    ("gkv_paged_append", 6, 2 ** 23, SHAPE), ("gkv_paged_append", 15, 2 ** 26 + 1, SHAPE),
    *[("gkv_paged_attend_decode", at, v, INVALID) for at, v in [(i, None) for i in (0, 1, 2, 3, 7, 9)] + [(4, 0), (5, 0), (6, 0), (8, -1), (0, AT + 1), (1, AT + 1), (2, AT + 1), (9, AT + 1)]],
    ("gkv_paged_attend_decode", 4, 2 ** 26 + 1, SHAPE), ("gkv_paged_attend_decode", 8, 65, OVERFLOW),
    ("gkv_paged_attend_decode", 10, None, WORKSPACE), ("gkv_paged_attend_decode", 10, AT + 8, WORKSPACE),
]


@pytest.mark.parametrize("name,at,value,status", REFUSED)
def test_arguments_are_refused_on_the_host(name, at, value, status):
    ctx = _ctx()
    args = list(GOOD[name])
    args[at] = value
    assert getattr(LIB, name)(ctx.h, *args, None) == status
    assert getattr(LIB, name)(None, *args, None) in (INVALID, status)
    ctx.close()


@pytest.mark.parametrize("name,q_out,stride", [("gkv_rotate", 12, 1), ("gkv_rotate", 13, 3), ("gkv_paged_append", 20, 1)])
def test_rows_apart_are_not_turned_in_place(name, q_out, stride):
    ctx = _ctx()
    args = list(GOOD[name])
    args[q_out], args[stride] = AT, 1024
    assert getattr(LIB, name)(ctx.h, *args, None) == INVALID
    ctx.close()


def test_nothing_to_turn_and_queries_without_frequencies_are_refused():
    ctx = _ctx()
    args = list(GOOD["gkv_rotate"])
    args[0] = args[2] = args[12] = args[13] = None
    assert LIB.gkv_rotate(ctx.h, *args, None) == INVALID
    args = list(GOOD["gkv_paged_append"])
    args[7] = None                                                # one token each: not five of three sequences
    assert LIB.gkv_paged_append(ctx.h, *args, None) == INVALID
    ctx.close()


def test_more_units_than_a_launch_has_room_for_are_refused():
    ctx = _ctx(n_layers=1, batch=1 << 22)
    assert LIB.gkv_paged_attend_decode(ctx.h, *GOOD["gkv_paged_attend_decode"], None) == SHAPE
    ctx.close()


def test_workspace_covers_the_pieces_of_every_unit():
    for kw in (dict(), dict(batch=64, n_layers=1), dict(n_layers=36, batch=64, n_q_heads=40, n_kv_heads=8, head_dim=128), dict(batch=1, n_layers=1, head_dim=72)):
        ctx = _ctx(**kw)
        c = ctx.cfg
        n = ctx.paged_workspace_bytes()
        assert 256 <= n < 1 << 30
        assert LIB.gkv_paged_workspace_bytes(ctx.h, None) == INVALID
        ctx.close()


@pytest.mark.parametrize("dim", [2, 4, 20, 64, 96, 128])
@pytest.mark.parametrize("base", [10000.0, 5.0e5])
def test_frequencies(dim, base):
    f = [base ** (-2 * p / dim) for p in range(dim // 2)]
    close = lambda a, b: all(abs(x - y) <= 1e-13 * abs(y) for x, y in zip(a, b)) and len(a) == len(b)
    got, m = P.rotary_frequencies(dim, base)
    assert close(got, f) and m == 1.0
    got, m = P.rotary_frequencies(dim, base, "linear", 4.0)
    assert close(got, [x / 4 for x in f]) and m == 1.0
    got, m = P.rotary_frequencies(dim, base, "base", 4.0)
    assert close(got, [x * 4.0 ** (-2 * p / (dim - 2)) if dim > 2 else x for p, x in enumerate(f)]) and m == 1.0
    if dim > 2:
        assert abs(got[-1] * 4 / f[-1] - 1) < 1e-12 and got[0] == f[0]
    trained = 4096.0
    got, m = P.rotary_frequencies(dim, base, "smooth", 8.0, trained, 1.0, 4.0)
    turns = [trained * x / (2 * math.pi) for x in f]
    share = [min(1.0, max(0.0, (t - 1.0) / 3.0)) for t in turns]
    assert close(got, [x / 8 * (1 - s) + x * s for x, s in zip(f, share)]) and m == 1.0
    assert all(g == x for g, x, t in zip(got, f, turns) if t >= 4)
    assert all(abs(g * 8 / x - 1) < 1e-12 for g, x, t in zip(got, f, turns) if t <= 1)
    got, m = P.rotary_frequencies(dim, base, "by_parts", 8.0, trained, 1.0, 32.0)
    at = [dim / 2 * math.log(trained / (2 * math.pi * t), base) for t in (32.0, 1.0)]
    lo, hi = max(math.floor(at[0]), 0), min(math.ceil(at[1]), dim - 1)
    ramp = [min(1.0, max(0.0, (p - lo) / max(hi - lo, 0.001))) for p in range(dim // 2)]
    assert close(got, [x * (1 - r) + x / 8 * r for x, r in zip(f, ramp)])
    assert abs(m - (0.1 * math.log(8.0) + 1)) < 1e-6
    assert P.rotary_frequencies(dim, base, "by_parts", 0.5, trained, 1.0, 32.0)[1] == 1.0


@pytest.mark.parametrize("kw", [dict(dim=0), dict(dim=3), dict(dim=-2), dict(base=1.0), dict(base=float("nan")), dict(base=float("inf")), dict(scaling=5),
                                dict(scaling=-1), dict(factor=0.0), dict(factor=float("inf")), dict(scaling="smooth", trained_length=0.0),
                                dict(scaling="by_parts", trained_length=4096.0, low=0.0), dict(scaling="smooth", trained_length=4096.0, low=4.0, high=4.0)])
def test_frequencies_refuse(kw):
    with pytest.raises(P.GkvError):
        P.rotary_frequencies(**{**dict(dim=64), **kw})


def _tensors(ctx, tokens=3):
    c = ctx.cfg
    dt = (torch.float32, torch.bfloat16)[c.dtype]
    z = lambda *s, dtype=dt: torch.zeros(*s, dtype=dtype)
    return dict(q=z(c.n_layers, tokens, c.n_q_heads, c.head_dim), k=z(c.n_layers, tokens, c.n_kv_heads, c.head_dim),
                v=z(c.n_layers, tokens, c.n_kv_heads, c.head_dim), K=z(c.n_layers, 9, c.n_kv_heads, 16, c.head_dim),
                V=z(c.n_layers, 9, c.n_kv_heads, 16, c.head_dim), table=z(c.batch, 4, dtype=torch.int32), d_len=z(c.batch, dtype=torch.int32),
                q_out=z(c.n_layers, tokens, c.n_q_heads, c.head_dim), k_out=z(c.n_layers, tokens, c.n_kv_heads, c.head_dim),
                positions=z(tokens, dtype=torch.int32), d_start=z(c.batch + 1, dtype=torch.int32),
                workspace=z(ctx.paged_workspace_bytes(), dtype=torch.uint8))


WRONG = [("q", lambda t: t[:, :, :4]), ("k", lambda t: t[..., :32]), ("q", lambda t: t.half()), ("k", lambda t: t.float()), ("q_out", lambda t: t[:1]),
         ("q", lambda t: t.transpose(2, 3).contiguous().transpose(2, 3)), ("q", lambda t: t.expand(-1, -1, -1, -1).flip(0)[:, :2]),
         ("positions", lambda t: t.long()), ("positions", lambda t: t[:2]), ("d_start", lambda t: t[:3]), ("d_len", lambda t: t.float()), ("table", lambda t: t[:2]),
         ("table", lambda t: t.long()), ("table", lambda t: t[0]), ("K", lambda t: t[..., :32]), ("V", lambda t: t[:, :4]), ("V", lambda t: t.float()), ("K", lambda t: t[0])]


@pytest.mark.parametrize("name,wrong", WRONG)
def test_python_refuses_other_shapes_and_types(name, wrong):
    ctx = _ctx()
    a = _tensors(ctx)
    a[name] = wrong(a[name])
    rotary = P.Rotary(64, device="cpu")
    calls = [("rotate", lambda: ctx.rotate(a["q"], a["k"], a["positions"], 0, rotary, a["q_out"], a["k_out"]), ("q", "k", "positions", "q_out")),
             ("append", lambda: ctx.paged_append(a["q"], a["k"], a["v"], a["d_start"], a["d_len"], a["positions"], rotary, a["table"], a["K"], a["V"], a["q_out"]),
              ("q", "k", "positions", "d_start", "d_len", "table", "K", "V", "q_out")),
             ("attend", lambda: ctx.paged_attend_decode(a["q"], a["K"], a["V"], a["table"], a["d_len"], 64, a["q_out"], a["workspace"]),
              ("q", "d_len", "table", "K", "V", "q_out")),
             ("advance", lambda: ctx.paged_advance(a["d_len"], a["d_start"]), ("d_len", "d_start"))]
    for what, call, takes in calls:
        if name in takes:
            with pytest.raises(ValueError):
                call()
    ctx.close()


def test_python_refuses_tensors_that_are_not_on_the_current_gpu():
    ctx = _ctx()
    a = _tensors(ctx)
    rotary = P.Rotary(64, device="cpu")
    for call in (lambda: ctx.rotate(a["q"], a["k"], a["positions"], 0, rotary, a["q_out"], a["k_out"]),
                 lambda: ctx.paged_append(a["q"], a["k"], a["v"], a["d_start"], a["d_len"], None, rotary, a["table"], a["K"], a["V"], a["q_out"]),
                 lambda: ctx.paged_attend_decode(a["q"], a["K"], a["V"], a["table"], a["d_len"], 64, a["q_out"], a["workspace"]),
                 lambda: ctx.paged_advance(a["d_len"], None)):
        with pytest.raises((ValueError, RuntimeError)):
            call()
    ctx.close()


def test_python_refuses_a_small_workspace_and_wrong_frequencies():
    ctx = _ctx()
    a = _tensors(ctx)
    with pytest.raises(P.GkvError):
        ctx.paged_attend_decode(a["q"], a["K"], a["V"], a["table"], a["d_len"], 64, a["q_out"], a["workspace"][:-1])
    with pytest.raises(ValueError):
        P.Rotary(64, device="cpu", freq=torch.ones(31))
    with pytest.raises(KeyError):
        P.Rotary(64, device="cpu", layout="other")
    ctx.close()


def test_state_refuses_what_its_pages_have_no_room_for():
    cfg = P.make_config(1, 2, 4, 2, 64, 64, 8, 16, 96, "f32")
    st = PagedDecodeState(cfg, max_rows=40, page_rows=16, n_pages=4, device="cpu")
    with pytest.raises(ValueError, match="longer"):
        st.reserve([49, 0])
    with pytest.raises(ValueError, match="free"):
        st.reserve([40, 40])
    with pytest.raises(ValueError):
        st.reserve([1])
    st.reserve([33, 16])
    assert sorted(st.page_table[0, :3].tolist() + st.page_table[1, :1].tolist()) == [0, 1, 2, 3] and not st._free
    with pytest.raises(ValueError):
        st.reserve([33, 17])
    st.release(0)
    assert (st.page_table[0] == -1).all() and int(st.d_len[0]) == -1
    st.reserve([0, 40])
    assert len(set(st.page_table[1].tolist())) == 3
    k = torch.zeros(1, 3, 2, 64)
    for counts in ([1], [1, -1], [2, 2]):
        with pytest.raises(ValueError):
            st.append(k, k, counts)
    with pytest.raises(ValueError):
        st.append(k, k)
    with pytest.raises(ValueError, match="rotary"):
        st.append(k[:, :2], k[:, :2], None, torch.zeros(1, 2, 4, 64))
    for i in (-1, 2):
        with pytest.raises(ValueError):
            st.release(i)


def test_a_refused_call_leaves_the_state_as_it_was():
    cfg = P.make_config(1, 2, 4, 2, 64, 64, 8, 16, 96, "f32")
    st = PagedDecodeState(cfg, max_rows=40, page_rows=16, rotary=P.Rotary(64, device="cpu"), device="cpu")
    q, k = torch.zeros(1, 2, 4, 64), torch.zeros(1, 2, 2, 64)
    before = (st._len, list(st._pages), len(st._free), st.d_len.clone())
    for call in (lambda: st.append(k[..., :32], k), lambda: st.append(k, k[:, :1]), lambda: st.append(k.half(), k.half()), lambda: st.append(k, k, [40, 2]),
                 lambda: st.append(k, k, None, q[:, :, :3]), lambda: st.append(k, k, None, q, torch.zeros(2)), lambda: st.append(k, k, None, q, None, q[:, :1]),
                 lambda: st.append(k, k.to("meta")), lambda: st.attend_decode(q[:, :1], k, k), lambda: st.append(k, k, None, q, torch.zeros(3, dtype=torch.int32))):
        with pytest.raises(ValueError):
            call()
        assert (st._len, list(st._pages), len(st._free)) == before[:3] and torch.equal(st.d_len, before[3])


def test_a_state_refuses_what_no_call_could_take():
    make = lambda **kw: PagedDecodeState(P.make_config(1, 2, 4, 2, 64, 64, 8, 16, 96, "f32"), **{**dict(max_rows=40, page_rows=16, device="cpu"), **kw})
    for kw in (dict(max_rows=0), dict(page_rows=0), dict(n_pages=0), dict(max_rows=(1 << 30) + 1, page_rows=1 << 29, n_pages=1), dict(rotary=P.Rotary(66, device="cpu"))):
        with pytest.raises(ValueError):
            make(**kw)
    # more tokens than a call takes: refused before the sequences grow
    st = PagedDecodeState(P.make_config(1, 2, 1, 1, 4, 64, 8, 16, 96, "f32"), max_rows=1 << 24, page_rows=1 << 20, n_pages=1, device="cpu")
    k = torch.zeros(1, 1 << 24, 1, 4)
    with pytest.raises(ValueError, match="too many"):
        st.append(k, k, [5, 5])
    assert st._len == [0, 0] and st._pages == [0, 0]

"""What the calls on caches in 8 bits and on shared prefixes refuse, and their sizes: host code only."""
import ctypes

import pytest
import torch

import paper_2512_00504_amd as P

from q8_reference import F8, held, same, values

LIB = P.load_library()
AT = 1 << 20                                  # an aligned address that is never dereferenced: every call here fails on the host


def _ctx(**kw):
    base = dict(n_layers=2, batch=3, n_q_heads=8, n_kv_heads=2, head_dim=64, budget=64, window=8, interval=16, capacity=96,
                dtype="bf16")
    base.update(kw)
    return P.Context(P.make_config(**base))


# good arguments of each call, without context and stream; a refusal differs in one place
GOOD = {
    "gkv_q8_store_prompt": [AT, AT, 5, 0, 5, AT, AT, AT, AT, AT],
    "gkv_q8_read": [AT, AT, AT, AT, 0, AT, AT],
    "gkv_q8_attend_decode": [AT] * 7 + [0, AT, AT, 3, None, AT, AT],
    "gkv_q8_score_window": [AT, AT, AT, AT, 0, 3, AT, AT],
    "gkv_q8_compact": [AT, 2 * AT, AT, AT, AT, AT, AT, AT, 0, AT],
    "gkv_q8_evict": [AT, AT, AT, AT, AT, AT, AT, 0, 3, AT, 2 * AT, AT, AT],
    "gkv_prefix_attend": [AT, AT, AT, 5, 7, 0, 3, AT],
    "gkv_attend_decode_prefix": [AT] * 6 + [0, AT, AT, 3, AT, AT, AT],
}
INVALID, SHAPE, WORKSPACE, OVERFLOW = 1, 2, 3, 6
REFUSED = [
    *[("gkv_q8_store_prompt", at, v, INVALID) for at, v in [(i, None) for i in (0, 1, 5, 6, 7, 8, 9)] + [(2, 0), (3, -1), (4, -1)]
      + [(i, AT + 8) for i in (0, 1, 6, 7, 8)]],
    *[("gkv_q8_read", at, v, INVALID) for at, v in [(0, None), (1, None), (2, None), (3, None), (4, -1)] + [(i, AT + 8) for i in (0, 1, 2, 5, 6)]],
    *[("gkv_q8_attend_decode", at, v, INVALID) for at, v in [(i, None) for i in (0, 1, 2, 3, 4, 5, 6, 8, 9, 12)] + [(7, -1), (10, -1)]
      + [(i, AT + 4) for i in (3, 4, 5, 11)]],
    ("gkv_q8_attend_decode", 13, None, WORKSPACE), ("gkv_q8_attend_decode", 10, 96, OVERFLOW),
    *[("gkv_q8_score_window", at, v, INVALID) for at, v in [(i, None) for i in (0, 1, 2, 3, 6)] + [(4, -1), (5, -1), (1, AT + 8), (2, AT + 4)]],
    ("gkv_q8_score_window", 5, 97, OVERFLOW),
    *[("gkv_q8_compact", at, v, INVALID) for at, v in [(i, None) for i in range(8)] + [(8, -1), (1, AT)] + [(i, AT + 8) for i in (2, 3, 4)]],
    *[("gkv_q8_evict", at, v, INVALID) for at, v in [(i, None) for i in (0, 1, 2, 3, 4, 5, 6, 9, 10, 11)] + [(7, -1), (8, -1), (10, AT), (2, AT + 8)]],
    ("gkv_q8_evict", 8, 97, OVERFLOW),
    *[("gkv_prefix_attend", at, v, INVALID) for at, v in [(i, None) for i in (0, 1, 2, 7)] + [(3, -1), (3, 8), (5, -1), (5, 1), (6, 0), (6, 4),
                                                                                               (6, 2 ** 31 - 1), (7, AT + 8)]],
    *[("gkv_attend_decode_prefix", at, v, INVALID) for at, v in [(i, None) for i in (0, 1, 2, 3, 4, 5, 7, 8, 10, 11)] + [(6, -1), (9, -1), (10, AT + 8)]],
    ("gkv_attend_decode_prefix", 12, None, WORKSPACE), ("gkv_attend_decode_prefix", 9, 96, OVERFLOW),
]


@pytest.mark.parametrize("name,at,value,status", REFUSED)
def test_arguments_are_refused_on_the_host(name, at, value, status):
    ctx = _ctx()
    ctx.prefix_bytes(7)
    args = list(GOOD[name])
    args[at] = value
    assert getattr(LIB, name)(ctx.h, *args, None) == status
    assert getattr(LIB, name)(None, *args, None) in (INVALID, status)
    ctx.close()


@pytest.mark.parametrize("name", [n for n in GOOD if "q8" in n])
def test_rows_that_are_not_whole_pieces_are_refused(name):
    ctx = _ctx(head_dim=72)
    assert getattr(LIB, name)(ctx.h, *GOOD[name], None) == SHAPE
    ctx.close()


def test_a_prefix_longer_than_the_buffer_was_sized_for_is_refused():
    ctx = _ctx()
    assert LIB.gkv_prefix_attend(ctx.h, *GOOD["gkv_prefix_attend"], None) == WORKSPACE      # never sized
    ctx.prefix_bytes(4)
    assert LIB.gkv_prefix_attend(ctx.h, *GOOD["gkv_prefix_attend"], None) == WORKSPACE
    with pytest.raises(P.GkvError):
        ctx.prefix_bytes(-1)
    assert LIB.gkv_prefix_bytes(ctx.h, 5, None) == INVALID
    ctx.close()


def test_more_rows_than_indices_have_room_for_are_refused():
    ctx = _ctx()
    ctx.prefix_bytes(2 ** 31 - 1)
    args = list(GOOD["gkv_prefix_attend"])
    args[3] = args[4] = 2 ** 30 + 1
    assert LIB.gkv_prefix_attend(ctx.h, *args, None) == SHAPE
    args = list(GOOD["gkv_q8_store_prompt"])
    args[2] = 2 ** 30 + 1
    assert LIB.gkv_q8_store_prompt(ctx.h, *args, None) == SHAPE
    ctx.close()


@pytest.mark.parametrize("batch", [1, 3, 64])
def test_prefix_buffer_never_shrinks_with_more_rows(batch):
    ctx = _ctx(batch=batch)
    sizes = [ctx.prefix_bytes(n) for n in (0, 1, 63, 64, 255, 256, 257, 1000, 4096, 65536, 1 << 20, 2 ** 31 - 1)]
    assert sizes == sorted(sizes)
    heads = 2 * batch * 8
    assert sizes[0] >= heads * (64 * 4 + 8)
    ctx.close()


@pytest.mark.parametrize("name,at,value", [(n, i, v) for n, i, v, _ in REFUSED if n not in ("gkv_q8_store_prompt", "gkv_q8_read")
                                           and not isinstance(v, int)])
def test_the_python_calls_raise(name, at, value):
    if not torch.cuda.is_available():
        pytest.skip("the stream's handle needs a GPU")
    ctx = _ctx()
    ctx.prefix_bytes(7)
    args = [None if v is None else v if isinstance(v, int) and v < AT else torch.zeros(64, device="cuda") for v in GOOD[name]]
    args[at] = value
    with pytest.raises(P.GkvError):
        getattr(ctx, name.removeprefix("gkv_"))(*args)
    ctx.close()


def test_reference_agrees_with_torchs_e4m3():
    g = torch.Generator().manual_seed(0)
    x = torch.randn(300, 64, generator=g, dtype=torch.float64).to(torch.bfloat16).double() * torch.logspace(-30, 30, 300).double()[:, None]
    c, e = held(x)
    y = torch.ldexp(x, -e.double())
    assert (y.abs().amax(dim=-1) <= 448).all() and (y.abs().amax(dim=-1) > 224).all()
    assert same(y.float().to(F8), c)
    assert ((values(x) - x).abs() <= torch.maximum(2.0 ** -4 * x.abs(), torch.ldexp(torch.ones_like(x), e.double() - 10))).all()
    for row, exponent in (([448.0, 1], 0), ([449.0, 1], 1), ([0.0, 0], 0), ([float("inf"), 2.0 ** -8], -16), ([2.0 ** -130, 0], -126)):
        assert held(torch.tensor([row]))[1].item() == exponent

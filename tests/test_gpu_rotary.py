"""Queries and keys turned by their positions, against 64 bits."""
import pytest
import torch

import paper_2512_00504_amd as P
from paper_2512_00504_amd import Rotary, make_config
from paper_2512_00504_amd.state import DecodeState, Q8DecodeState, SharedPrefix

from paged_reference import DT, turned

pytestmark = pytest.mark.gpu


def _ctx(L=1, B=1, hq=4, hkv=2, d=64, dtype="bf16"):
    return P.Context(make_config(L, B, hq, hkv, d, 64, 8, 16, 96, dtype))


def _inputs(L, n, hq, hkv, d, dtype, apart, seed=0):
    g = torch.Generator().manual_seed(seed + n + d)
    x = (torch.randn(L, n, hq + 2 * hkv, d, generator=g) * 3).to(DT[dtype])
    if apart == "fused":                                     # slices of one projection's output
        x = x.cuda()
        return x[:, :, :hq], x[:, :, hq:hq + hkv]
    if apart == "odd":                                       # tokens an odd number of elements apart, the first one not on 16 bytes
        q = torch.zeros(L, n, hq * d + 3, dtype=DT[dtype]).cuda()[..., 1:1 + hq * d].view(L, n, hq, d) if n * L else x[:, :, :hq].cuda()
        k = torch.zeros(L, n, hkv * d + 1, dtype=DT[dtype]).cuda()[..., :hkv * d].view(L, n, hkv, d)
        q.copy_(x[:, :, :hq]); k.copy_(x[:, :, hq:hq + hkv])
        return q, k
    return x[:, :, :hq].contiguous().cuda(), x[:, :, hq:hq + hkv].contiguous().cuda()


def _check(got, x, positions, rotary, layout, dtype, transposed=False):
    ref, tol = turned(x.cpu(), positions.cpu(), rotary.freq.cpu(), layout, rotary.amplitude, transposed, dtype)
    err = (got.cpu().double() - ref).abs()
    assert (err <= tol).all(), (err - tol).max().item()


SHAPES = [("bf16", 128, 128), ("bf16", 128, 96), ("bf16", 128, 32), ("bf16", 64, 64), ("f32", 64, 64), ("f32", 64, 48), ("f32", 20, 20), ("bf16", 72, 40), ("bf16", 72, 72),
          ("f32", 36, 6), ("bf16", 64, 2), ("bf16", 64, 50), ("f32", 128, 126), ("bf16", 512, 512), ("f32", 256, 256), ("bf16", 24, 16)]


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype,d,dim", SHAPES)
@pytest.mark.parametrize("n,apart", [(1, "no"), (3, "fused"), (9, "odd"), (70, "fused")])
def test_every_shape(layout, dtype, d, dim, n, apart):
    L, hq, hkv = 2, 6, 2
    ctx = _ctx(L, 1, hq, hkv, d, dtype)
    q, k = _inputs(L, n, hq, hkv, d, dtype, apart)
    rotary = Rotary(dim, 10000.0, layout, "by_parts", 8.0, 4096.0)
    positions = (torch.arange(n, dtype=torch.int32) * 977 + 5).cuda()
    q_out, k_out = (torch.full(x.shape, float("nan"), dtype=x.dtype, device="cuda") for x in (q, k))
    for transposed in (False, True):
        ctx.rotate(q, k, positions, 0, rotary, q_out, k_out, transposed)
        _check(q_out, q, positions, rotary, layout, dtype, transposed)
        _check(k_out, k, positions, rotary, layout, dtype, transposed)


@pytest.mark.parametrize("n,L", [(1500, 1), (3000, 2), (20000, 1), (700, 28)])
def test_many_tokens(n, L):
    ctx = _ctx(L, 1, 7, 1, 128)
    q, k = _inputs(L, n, 7, 1, 128, "bf16", "fused")
    rotary = Rotary(128)
    positions = torch.arange(n, dtype=torch.int32).cuda()
    q_out, k_out = (torch.empty(x.shape, dtype=x.dtype, device="cuda") for x in (q, k))
    ctx.rotate(q, k, positions, 0, rotary, q_out, k_out)
    _check(q_out, q, positions, rotary, "half", "bf16")
    _check(k_out, k, positions, rotary, "half", "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_and_negative_positions(dtype):
    at = [0, 1, -1, -7, 1 << 20, (1 << 22) + 3, (1 << 24) + 1, -(1 << 26) - 5, 2 ** 31 - 1, -(2 ** 31)]
    ctx = _ctx(1, 1, 2, 1, 64, dtype)
    q, k = _inputs(1, len(at), 2, 1, 64, dtype, "no")
    rotary = Rotary(64, 500000.0, amplitude=0.75)
    positions = torch.tensor(at, dtype=torch.int32).cuda()
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    ctx.rotate(q, k, positions, 0, rotary, q_out, k_out)
    _check(q_out, q, positions, rotary, "half", dtype)
    _check(k_out, k, positions, rotary, "half", dtype)
    assert torch.equal(q_out[0, 0], (q[0, 0].float() * 0.75).to(q.dtype))       # position 0: the amplitude alone


def test_angles_next_to_quarter_turns():
    # frequencies that make the angle a multiple of pi/4 up to a rounding, on either side
    n, dim = 64, 64
    ctx = _ctx(1, 1, 1, 1, dim, "f32")
    freq = torch.pi / 4 * (1 + (torch.arange(dim // 2, dtype=torch.float64) - 16) * 2.0 ** -52)
    rotary = Rotary(dim, freq=freq)
    q, k = _inputs(1, n, 1, 1, dim, "f32", "no")
    positions = torch.arange(n, dtype=torch.int32).cuda()
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    ctx.rotate(q, k, positions, 0, rotary, q_out, k_out)
    _check(q_out, q, positions, rotary, "half", "f32")


def test_frequencies_rewritten_between_calls():
    ctx = _ctx(1, 1, 2, 1, 64, "f32")
    q, _ = _inputs(1, 5, 2, 1, 64, "f32", "no")
    rotary = Rotary(64)
    positions = torch.arange(5, dtype=torch.int32).cuda()
    out = torch.empty_like(q)
    for factor in (1.0, 4.0):
        rotary.freq.copy_(torch.tensor(P.rotary_frequencies(64, scaling="linear", factor=factor)[0], dtype=torch.float64))
        ctx.rotate(q, None, positions, 0, rotary, out, None)
        _check(out, q, positions, rotary, "half", "f32")


@pytest.mark.parametrize("dim,layout", [(64, "half"), (32, "interleaved"), (50, "half"), (10, "interleaved")])
def test_in_place_and_one_of_both(dim, layout):
    ctx = _ctx(2, 1, 4, 2, 64)
    q, k = _inputs(2, 33, 4, 2, 64, "bf16", "no")
    rotary = Rotary(dim, layout=layout)
    positions = torch.arange(33, dtype=torch.int32).cuda()
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    ctx.rotate(q, None, positions, 0, rotary, q_out, None)
    ctx.rotate(None, k, positions, 0, rotary, None, k_out)
    ctx.rotate(q, k, positions, 0, rotary, q, k)
    assert torch.equal(q, q_out) and torch.equal(k, k_out)
    ctx.rotate(q[:, :0], k[:, :0], positions[:0], 0, rotary, q_out[:, :0], k_out[:, :0])


def test_channels_that_stay_keep_their_bits_and_others_turn_into_no_number_alone():
    ctx = _ctx(1, 1, 2, 1, 64)
    q, _ = _inputs(1, 4, 2, 1, 64, "bf16", "no")
    q[..., 48:] = torch.tensor([float("inf"), float("nan"), float("-inf"), 0.0] * 4, dtype=q.dtype)
    q[0, 1, 0, 3] = float("nan")
    positions = torch.arange(4, dtype=torch.int32).cuda() + 1
    for dim, layout, hit in ((48, "half", (3, 27)), (48, "interleaved", (2, 3)), (46, "half", (3, 26))):
        out = torch.empty_like(q)
        ctx.rotate(q, None, positions, 0, Rotary(dim, layout=layout), out, None)
        assert torch.equal(out[..., dim:].view(torch.int16), q[..., dim:].view(torch.int16))
        nan = torch.isnan(out[..., :dim]).nonzero().cpu().tolist()
        assert nan == [[0, 1, 0, c] for c in hit]


def test_step_for_every_token_and_step_base():
    ctx = _ctx(1, 3, 2, 1, 64, "f32")
    q, k = _inputs(1, 3, 2, 1, 64, "f32", "no")
    rotary = Rotary(64)
    out, ref = torch.empty_like(q), torch.empty_like(q)
    at = lambda n: torch.full((3,), n, dtype=torch.int32).cuda()
    ctx.rotate(q, None, at(1000), 0, rotary, ref, None)
    ctx.rotate(q, None, None, 1000, rotary, out, None)
    assert torch.equal(out, ref)
    base = torch.tensor([992], dtype=torch.int32).cuda()
    ctx.set_step_base(base)
    ctx.rotate(q, None, None, 8, rotary, out, None)
    assert torch.equal(out, ref)
    ctx.advance_step_base(16)
    ctx.rotate(q, None, None, 8, rotary, out, None)
    ctx.rotate(q, None, at(1016), 0, rotary, ref, None)
    assert torch.equal(out, ref)
    ctx.set_step_base(None)


@pytest.mark.parametrize("layout,dim", [("half", 64), ("interleaved", 40)])
def test_transposed_is_the_gradient(layout, dim):
    # of sum(w * y): by the formula's own derivative in 64 bits, and by differences of the kernel's outputs (32 bits, linear: a step of 1
    # in one channel changes y by a column, each output off by its bound twice)
    ctx = _ctx(1, 1, 2, 1, 64, "f32")
    q, _ = _inputs(1, 6, 2, 1, 64, "f32", "no")
    rotary = Rotary(dim, layout=layout, amplitude=1.25)
    positions = (torch.arange(6, dtype=torch.int32) * 31).cuda()
    w = torch.randn(q.shape, generator=torch.Generator().manual_seed(3)).cuda()
    grad = torch.empty_like(q)
    ctx.rotate(w, None, positions, 0, rotary, grad, None, transposed=True)
    x = q.cpu().double().requires_grad_()
    y, _ = turned(x, positions.cpu(), rotary.freq.cpu(), layout, 1.25, dtype="f32")
    (y * w.cpu().double()).sum().backward()
    _, tol = turned(w.cpu(), positions.cpu(), rotary.freq.cpu(), layout, 1.25, True, "f32")
    assert ((grad.cpu().double() - x.grad).abs() <= tol).all()
    out, more = torch.empty_like(q), torch.empty_like(q)
    ctx.rotate(q, None, positions, 0, rotary, out, None)
    for c in (0, 1, dim // 2, dim - 1, 63):
        q2 = q.clone()
        q2[..., c] += 1.0
        step = q2[..., c].double() - q[..., c].double()
        ctx.rotate(q2, None, positions, 0, rotary, more, None)
        change = ((more.double() - out.double()) * w.double()).sum(dim=-1) / step
        _, t1 = turned(q2.cpu(), positions.cpu(), rotary.freq.cpu(), layout, 1.25, dtype="f32")
        _, t0 = turned(q.cpu(), positions.cpu(), rotary.freq.cpu(), layout, 1.25, dtype="f32")
        bound = ((t0 + t1) * w.cpu().double().abs()).sum(dim=-1) / step.cpu().abs() + tol[..., c]
        assert ((change - grad[..., c].double()).abs().cpu() <= bound).all(), c


@pytest.mark.parametrize("cls", [DecodeState, Q8DecodeState])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_steps_with_a_rotary_are_those_of_turned_inputs(cls, dtype):
    cfg = lambda: make_config(2, 3, 4, 2, 64, 16, 4, 8, 32, dtype)
    a, b = cls(cfg()), cls(cfg())
    rotary = Rotary(64, scaling="linear", factor=2.0)
    g = torch.Generator().manual_seed(0)
    for t in range(40):
        q, k, v = (torch.randn(2, 3, h, 64, generator=g).to(DT[dtype]).cuda() for h in (4, 2, 2))
        qt, kt = torch.empty_like(q), torch.empty_like(k)
        b.ctx.rotate(q, k, torch.full((3,), t, dtype=torch.int32).cuda(), 0, rotary, qt, kt)
        out = a.attend_decode(q, k, v, t, rotary=rotary).clone()
        assert torch.equal(out, b.attend_decode(qt, kt, v, t))
        assert torch.equal(a.qwin[t % 4], qt)
        if a.is_trigger(t):
            a.evict(t); b.evict(t)
    assert torch.equal(a.pos, b.pos) and torch.equal(a.d_state, b.d_state) and torch.equal(a.F_hist, b.F_hist)


@pytest.mark.parametrize("cls", [DecodeState, Q8DecodeState])
def test_decode_steps_with_a_rotary_and_a_shared_prefix(cls):
    # the prompt's keys at the positions before the first step's
    cfg, rows = make_config(2, 3, 4, 2, 64, 16, 4, 8, 32, "bf16"), 21
    a, b = cls(cfg), cls(cfg)
    rotary, g = Rotary(64), torch.Generator().manual_seed(1)
    pk, pv = (torch.randn(2, 2, rows, 64, generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    ctx, turned_pk = _ctx(2, 1, 4, 2), torch.empty(2, rows, 2, 64, dtype=torch.bfloat16, device="cuda")
    ctx.rotate(None, pk.transpose(1, 2).contiguous(), torch.arange(rows, dtype=torch.int32).cuda(), 0, rotary, None, turned_pk)
    prompts = [SharedPrefix(st, turned_pk.transpose(1, 2), pv) for st in (a, b)]
    a.set_state(0, rows, 0, 0); b.set_state(0, rows, 0, 0)
    for t in range(rows, rows + 10):
        q, k, v = (torch.randn(2, 3, h, 64, generator=g).to(torch.bfloat16).cuda() for h in (4, 2, 2))
        qt, kt = torch.empty_like(q), torch.empty_like(k)
        b.ctx.rotate(q, k, torch.full((3,), t, dtype=torch.int32).cuda(), 0, rotary, qt, kt)
        out = a.attend_decode(q, k, v, t, prefix=prompts[0], rotary=rotary).clone()
        assert torch.equal(out, b.attend_decode(qt, kt, v, t, prefix=prompts[1]))


def test_recorded_calls_replay():
    ctx = _ctx(2, 1, 4, 2, 128)
    q, k = _inputs(2, 50, 4, 2, 128, "bf16", "fused")
    rotary = Rotary(128)
    positions = torch.arange(50, dtype=torch.int32).cuda()
    q_out, k_out = (torch.zeros(x.shape, dtype=x.dtype, device="cuda") for x in (q, k))
    ctx.rotate(q, k, positions, 0, rotary, q_out, k_out)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.rotate(q, k, positions, 0, rotary, q_out, k_out)
    ref_q, ref_k = torch.empty_like(q_out), torch.empty_like(k_out)
    for i in range(3):
        positions += 100
        q.mul_(-1)
        ctx.rotate(q, k, positions, 0, rotary, ref_q, ref_k)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(q_out, ref_q) and torch.equal(k_out, ref_k)

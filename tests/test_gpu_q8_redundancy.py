"""The redundancy term on a cache in 8 bits, part by part."""
import pytest
import torch

from paper_2512_00504_amd import make_config
from paper_2512_00504_amd.state import DecodeState, Q8DecodeState, k_rows_to_cache

from q8_reference import values
from test_gpu_q8 import _fill, _rows

pytestmark = pytest.mark.gpu


def _pair(L, B, hkv, g, d, dtype, b, w, s, cap, seed=0, params=None):
    """The same rows in 8 bits and as a cache of the type that holds the same values; lengths of up to the capacity."""
    cfg = make_config(L, B, hkv * g, hkv, d, b, w, s, cap, dtype)
    st, ref = Q8DecodeState(cfg, params=params), DecodeState(cfg, params=params)
    gen = torch.Generator().manual_seed(seed)
    K, V = _rows(gen, dtype, L, B, hkv, cap, d), _rows(gen, dtype, L, B, hkv, cap, d)
    lens = [cap - 3 * (i % 5) if i % 4 else b for i in range(B)]
    _fill(st, K, V, lens, b, since=20, decoded=w)
    ref.d_state.copy_(st.d_state)
    F = torch.rand(L, B, hkv, cap, generator=gen)
    for i in range(B):
        ref.K[:, i] = k_rows_to_cache(values(K[:, i]).to(K.dtype), min(b, (lens[i] - w) // 16 * 16)).cuda()
    for x in (st, ref):
        x.F.copy_(F)
        x.R.fill_(-7.0); x.F_sel.fill_(-7.0)
        x.len_host = max(lens)
    return st, ref


@pytest.mark.parametrize("L,B,hkv,g,d,dtype", [(4, 40, 4, 2, 128, "bf16"), (3, 100, 2, 1, 64, "f32"), (1, 131, 4, 1, 128, "f32"), (2, 37, 8, 2, 64, "bf16"),
                                               (2, 2, 2, 2, 128, "bf16"), (5, 60, 1, 3, 48, "bf16")])
def test_parts_give_what_the_whole_gives(L, B, hkv, g, d, dtype):
    b, w, s = 40, 8, 16
    st, ref = _pair(L, B, hkv, g, d, dtype, b, w, s, 64)
    for step in (20 + w - 1, 20 + w - 1):
        for x in (st, ref):
            x.redundancy_combine(step, 0.7, 0.3, w)
        assert torch.equal(st.R, ref.R) and torch.equal(st.F_sel, ref.F_sel)
        st._K_part.fill_(float("nan"))                     # what is behind the rows does not count
        st.R.fill_(-7.0); st.F_sel.fill_(-7.0)
    units = L * B * hkv
    assert st._K_part.numel() <= (st.K8.numel() if units < 512 else 384 * 64 * d) and st.K is None


def test_params_and_step_base_reach_the_parts():
    st, ref = _pair(2, 80, 4, 1, 128, "bf16", 40, 8, 16, 64)
    st.redundancy_combine(27, 0.7, 0.3, 8)
    for x in (st, ref):
        x.ctx.set_param("force_generic", 1)
        x.ctx.set_step_base(torch.tensor([20], dtype=torch.int32, device="cuda"))
        x.redundancy_combine(7, 0.7, 0.3, 8)
    assert torch.equal(st.R, ref.R) and torch.equal(st.F_sel, ref.F_sel)
    for x in (st, ref):
        x.ctx.set_step_base(None)
        x.ctx.set_param("force_generic", 0)
        x.redundancy_combine(27, 0.7, 0.3, 8)
    assert torch.equal(st.R, ref.R) and torch.equal(st.F_sel, ref.F_sel)


def test_the_full_method_takes_less_memory_than_a_cache_of_the_type():
    cfg = make_config(4, 64, 28, 4, 128, 512, 16, 128, 640, "bf16")
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    st = Q8DecodeState(cfg)
    held = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    st.set_state(640 - 16, 20, 0, 512)
    st.len_host = 640
    st.redundancy_combine(35, 0.7, 0.3, 16)
    codes = st.K8.numel() + st.V8.numel() + 2 * st.scales.numel()
    more = torch.cuda.max_memory_allocated() - held
    assert more <= codes // 4, (more, codes)               # of 1024 units a quarter of K, twice the size of its codes


def test_a_recorded_redundancy_term_replays_as_an_eager_one():
    st, ref = _pair(2, 80, 4, 1, 128, "bf16", 40, 8, 16, 64)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    st._parts()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        st.redundancy_combine(27, 0.7, 0.3, 8)
    for k in range(3):
        for x in (st, ref):
            x.F.mul_(0.75)
        ref.redundancy_combine(27, 0.7, 0.3, 8)
        st.R.fill_(-7.0); st.F_sel.fill_(-7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(st.R, ref.R) and torch.equal(st.F_sel, ref.F_sel), k
        st.redundancy_combine(27, 0.7, 0.3, 8)             # an eager call in between


def test_profile_counts_the_parts():
    st, _ = _pair(2, 80, 4, 1, 128, "bf16", 40, 8, 16, 64)
    st.ctx.profile_enable(True)
    for _ in range(2):
        st.redundancy_combine(27, 0.7, 0.3, 8)
    ms, calls = st.ctx.profile_read("redundancy")
    assert ms > 0 and calls == 2 * len(st._parts()) == 6
    st.ctx.profile_reset()
    assert st.ctx.profile_read("redundancy") == (0.0, 0)


def test_a_first_call_that_is_recorded():
    st, ref = _pair(2, 80, 4, 1, 128, "bf16", 40, 8, 16, 64)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        st.redundancy_combine(27, 0.7, 0.3, 8)
    ref.redundancy_combine(27, 0.7, 0.3, 8)
    for _ in range(3):
        for f in (graph.replay, lambda: st.redundancy_combine(27, 0.7, 0.3, 8)):
            st.R.fill_(-7.0); st.F_sel.fill_(-7.0)
            torch.cuda.synchronize()
            f()
            torch.cuda.synchronize()
            assert torch.equal(st.R, ref.R) and torch.equal(st.F_sel, ref.F_sel)

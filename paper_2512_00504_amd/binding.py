"""ctypes binding of libgkv.so: argument marshalling only.

Every step of the path runs in the HIP kernels behind the C ABI declared in
include/gkv.h; the functions here have the same names and pass device
pointers of torch tensors and the current torch stream straight through.
The calls a program makes per decode step or compression are marshalled by
_gkv_call (csrc/call.cpp); what it does not take, ctypes converts or refuses,
and all of it (1 to 2 us more a call) where only libgkv.so is built, with a warning.
There is no other way to the kernels: if libgkv.so is missing, loading raises.
"""
from __future__ import annotations

import ctypes
import os
import warnings
from ctypes import POINTER, byref, c_char_p, c_double, c_float, c_int32, c_int64, c_size_t, c_void_p

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("GKV_LIB_PATH") or os.path.join(_HERE, "libgkv.so")

GKV_F32, GKV_BF16 = 0, 1
GKV_COMBINE = {"max": 0, "avg": 1, "sum": 2}
GKV_ERR_WORKSPACE = 3
ST_LEN, ST_LEN_STEP, ST_N_HIST, ST_N_TILED = 0, 1, 2, 3     # fields of a d_state record
KERNEL_IDS = {"attend": 0, "score": 1, "global": 2, "topk": 3, "compact": 4, "redundancy": 5}

EXPORTS = [
    "gkv_create", "gkv_destroy", "gkv_status_string", "gkv_workspace_bytes", "gkv_workspace_init",
    "gkv_cache_bytes", "gkv_k_offset", "gkv_set_param", "gkv_attend_decode", "gkv_score_window",
    "gkv_global_update", "gkv_select_topk", "gkv_compact", "gkv_evict", "gkv_profile_enable",
    "gkv_profile_read", "gkv_profile_reset", "gkv_probe_attend_read", "gkv_redundancy_combine", "gkv_evicted_positions", "gkv_pool_scores",
    "gkv_evict_static", "gkv_set_step_base", "gkv_advance_step_base",
    "gkv_q8_store_prompt", "gkv_q8_read", "gkv_q8_attend_decode", "gkv_q8_score_window", "gkv_q8_compact", "gkv_q8_evict",
    "gkv_prefix_bytes", "gkv_prefix_attend", "gkv_attend_decode_prefix",
    "gkv_rotary_frequencies", "gkv_rotate", "gkv_paged_append", "gkv_paged_advance", "gkv_paged_workspace_bytes", "gkv_paged_attend_decode",
]
MOST_F32 = 2.0 ** 128 - 2.0 ** 104
ROTARY_LAYOUT = {"half": 0, "interleaved": 1}
ROTARY_SCALING = {"none": 0, "linear": 1, "base": 2, "by_parts": 3, "smooth": 4}


class GkvConfig(ctypes.Structure):
    _fields_ = [
        ("n_layers", c_int32), ("batch", c_int32), ("n_q_heads", c_int32), ("n_kv_heads", c_int32),
        ("head_dim", c_int32), ("budget", c_int32), ("window", c_int32), ("interval", c_int32),
        ("capacity", c_int32), ("dtype", c_int32), ("combine", c_int32), ("alpha", c_float),
        ("softmax_scale", c_float),
    ]


class GkvError(RuntimeError):
    def __init__(self, status, what):
        self.status = status
        super().__init__(f"{what}: gkv status {status}")


_lib = None


def load_library():
    """Load libgkv.so (built in-tree by __graft_entry__.build()).  Raises if it is absent."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            f"{LIB_PATH} is missing: build it with `python -c 'import __graft_entry__ as g; g.build()'`")
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32 = c_void_p, c_int32
    lib.gkv_create.argtypes = [POINTER(GkvConfig), POINTER(vp)]
    lib.gkv_destroy.argtypes = [vp]; lib.gkv_destroy.restype = None
    lib.gkv_status_string.argtypes = [i32]; lib.gkv_status_string.restype = c_char_p
    lib.gkv_workspace_bytes.argtypes = [vp, POINTER(c_size_t)]
    lib.gkv_workspace_init.argtypes = [vp, vp, vp]
    lib.gkv_cache_bytes.argtypes = [POINTER(GkvConfig), i32, i32, POINTER(c_size_t), POINTER(c_size_t)]
    lib.gkv_k_offset.argtypes = [POINTER(GkvConfig), i32, i32, i32]; lib.gkv_k_offset.restype = c_int64
    lib.gkv_set_param.argtypes = [vp, c_char_p, i32]
    lib.gkv_attend_decode.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, vp, vp, i32, vp, vp, vp]
    lib.gkv_score_window.argtypes = [vp, vp, vp, vp, i32, i32, vp, vp, vp]
    lib.gkv_global_update.argtypes = [vp, vp, vp, vp, i32, i32, vp, vp]
    lib.gkv_select_topk.argtypes = [vp, vp, vp, i32, i32, vp, vp, vp]
    lib.gkv_compact.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, vp]
    lib.gkv_evict.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, i32, vp, vp, vp, vp, vp]
    lib.gkv_set_step_base.argtypes = [vp, vp]
    lib.gkv_advance_step_base.argtypes = [vp, i32, vp]
    lib.gkv_evict_static.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, i32, vp, vp]
    lib.gkv_redundancy_combine.argtypes = [vp, vp, vp, i32, i32, vp, c_float, c_float, c_float, i32, vp, vp, vp, vp]
    lib.gkv_pool_scores.argtypes = [vp, vp, vp, i32, i32, vp, vp]
    lib.gkv_evicted_positions.argtypes = [vp, vp, vp, vp, i32, vp, vp]
    lib.gkv_q8_store_prompt.argtypes = [vp, vp, vp, i32, i32, i32, vp, vp, vp, vp, vp, vp]
    lib.gkv_q8_read.argtypes = [vp, vp, vp, vp, vp, i32, vp, vp, vp]
    lib.gkv_q8_attend_decode.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, vp, i32, vp, vp, vp, vp]
    lib.gkv_q8_score_window.argtypes = [vp, vp, vp, vp, vp, i32, i32, vp, vp, vp]
    lib.gkv_q8_compact.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, vp, i32, vp, vp]
    lib.gkv_q8_evict.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, i32, i32, vp, vp, vp, vp, vp]
    lib.gkv_prefix_bytes.argtypes = [vp, i32, POINTER(c_size_t)]
    lib.gkv_prefix_attend.argtypes = [vp, vp, vp, vp, i32, i32, i32, i32, vp, vp]
    lib.gkv_attend_decode_prefix.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, vp, vp, i32, vp, vp, vp, vp]
    lib.gkv_rotary_frequencies.argtypes = [i32, c_double, i32, c_double, c_double, c_double, c_double, vp, POINTER(c_float)]
    lib.gkv_rotate.argtypes = [vp, vp, i32, vp, i32, i32, vp, i32, vp, i32, i32, c_float, i32, vp, vp, vp]
    lib.gkv_paged_advance.argtypes = [vp, vp, vp, vp]
    lib.gkv_paged_append.argtypes = [vp, vp, i32, vp, i32, vp, i32, i32, vp, vp, vp, vp, i32, i32, c_float, vp, i32, i32, i32, vp, vp, vp, vp]
    lib.gkv_paged_workspace_bytes.argtypes = [vp, POINTER(c_size_t)]
    lib.gkv_paged_attend_decode.argtypes = [vp, vp, vp, vp, vp, i32, i32, i32, vp, i32, vp, vp, vp]
    lib.gkv_profile_enable.argtypes = [vp, i32]
    lib.gkv_profile_read.argtypes = [vp, i32, POINTER(c_double), POINTER(c_int64)]
    lib.gkv_profile_reset.argtypes = [vp]
    lib.gkv_probe_attend_read.argtypes = [vp, vp, i32, i32, i32, vp, vp]
    for name in EXPORTS:
        fn = getattr(lib, name)
        if name not in ("gkv_destroy", "gkv_status_string", "gkv_k_offset"):
            fn.restype = c_int32
    _lib = lib
    return lib


def make_config(n_layers, batch, n_q_heads, n_kv_heads, head_dim, budget, window, interval,
                capacity, dtype, combine="max", alpha=0.8, softmax_scale=0.0) -> GkvConfig:
    dt = {"f32": GKV_F32, "bf16": GKV_BF16}[dtype] if isinstance(dtype, str) else int(dtype)
    cb = GKV_COMBINE[combine] if isinstance(combine, str) else int(combine)
    return GkvConfig(n_layers, batch, n_q_heads, n_kv_heads, head_dim, budget, window, interval,
                     capacity, dt, cb, alpha, softmax_scale)


def _ptr(t):
    """Device pointer of a torch tensor (or None), as the integer the argument types convert."""
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("gkv: tensors must be contiguous")
    return t.data_ptr()


def _ptr_here(t, contiguous=True):
    """The same, of the current device; an address stays one."""
    if t is None or isinstance(t, int):
        return t
    import torch
    if not t.is_cuda or t.device.index != torch.cuda.current_device():
        raise ValueError(f"gkv: a tensor is on {t.device}, which is not the current GPU")
    return _ptr(t) if contiguous else t.data_ptr()


def _stream():
    """The raw handle of the current device's current stream.  A decode step is one call of a few
    microseconds of GPU time: building a torch.cuda.Stream object only to read its handle, and a
    c_void_p per argument, cost about a third of the call."""
    import torch
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def rotary_frequencies(dim, base=10000.0, scaling="none", factor=1.0, trained_length=0.0, low=1.0, high=32.0):
    """Radians a position of each pair of channels, and what cosines and sines are multiplied by (gkv_rotary_frequencies)."""
    lib = load_library()
    if not 2 <= dim < 1 << 16:
        raise GkvError(1, "gkv_rotary_frequencies")
    freq, amplitude = (c_double * (dim // 2))(), c_float()
    st = lib.gkv_rotary_frequencies(dim, base, ROTARY_SCALING[scaling] if isinstance(scaling, str) else int(scaling), factor,
                                    trained_length, low, high, freq, byref(amplitude))
    if st != 0:
        raise GkvError(st, "gkv_rotary_frequencies")
    return list(freq), amplitude.value


class Rotary:
    """Rotary positions of heads' first `dim` channels: frequencies on the device, layout ("half" or "interleaved") and amplitude.
    freq (float64 [dim/2]) may be rewritten in place, or given instead of what base and scaling say."""

    def __init__(self, dim, base=10000.0, layout="half", scaling="none", factor=1.0, trained_length=0.0, low=1.0, high=32.0,
                 device="cuda:0", freq=None, amplitude=None):
        import torch
        values, own = rotary_frequencies(dim, base, scaling, factor, trained_length, low, high)
        self.dim, self.layout = dim, ROTARY_LAYOUT[layout] if isinstance(layout, str) else int(layout)
        self.amplitude = own if amplitude is None else float(amplitude)
        if not 0 <= self.layout <= 1 or not abs(self.amplitude) <= MOST_F32:
            raise ValueError(f"gkv: a rotary's layout is one of {list(ROTARY_LAYOUT)}, its amplitude a finite number of 32 bits")
        self.freq = torch.tensor(values, dtype=torch.float64).to(device) if freq is None else freq.to(device, torch.float64).contiguous()
        if self.freq.shape != (dim // 2,):
            raise ValueError(f"gkv: freq has to be [{dim // 2}]")


_call = None


class _LeavesAllToCtypes:
    def __getattr__(self, name):
        return lambda *args: None


def _load_call():
    """The native marshalling, bound to the entry points of the library that ctypes loaded."""
    global _call
    if _call is None:
        lib = load_library()
        import torch  # noqa: F401  (the extension's libraries)
        try:
            from . import _gkv_call
        except ImportError as e:
            warnings.warn(f"gkv: calls go through ctypes, the native binding is not there ({e}): build it with "
                          "`python -c 'import __graft_entry__ as g; g.build()'`", RuntimeWarning, stacklevel=3)
            _call = _LeavesAllToCtypes()
            return _call
        for name in [*dir(_gkv_call), "gkv_rotate", "gkv_paged_append", "gkv_paged_attend_decode", "gkv_paged_advance"]:
            if name.startswith("gkv_"):
                _gkv_call.bind(name, ctypes.cast(getattr(lib, name), c_void_p).value)
        _call = _gkv_call
    return _call


class Context:
    """Owns a gkv_ctx.  Methods mirror the C entry points one to one."""

    def __init__(self, cfg: GkvConfig):
        self.lib = load_library()
        self.cfg = cfg
        h = c_void_p()
        st = self.lib.gkv_create(byref(cfg), byref(h))
        if st != 0:
            raise GkvError(st, "gkv_create")
        self.h = h
        self._handle = h.value
        self._call = _load_call()
        self._params, self._step_base, self._profiled, self._parts = {}, None, False, {}
        import torch
        self._spec = GkvConfig.from_buffer_copy(cfg)           # as the library has it
        self._spec_at, self._dtype, self._paged_bytes = ctypes.addressof(self._spec), (torch.float32, torch.bfloat16)[cfg.dtype], None
        self._double = torch.float64
        self._prefix_bytes, self._prefix_rows = {}, -1       # rows -> size of a buffer for them; the most rows asked for

    def part(self, sequences: int) -> "Context":
        """A context of so many (layer, sequence)s, for calls on slices of this one's buffers.  It is set as this one is, now and later, and
        the time and calls of its kernels count here."""
        if sequences not in self._parts:
            cfg = GkvConfig.from_buffer_copy(self.cfg)
            cfg.n_layers, cfg.batch = 1, sequences
            part = Context(cfg)
            for name, value in self._params.items():
                part.set_param(name, value)
            part.set_step_base(self._step_base)
            part.profile_enable(self._profiled)
            self._parts[sequences] = part
        return self._parts[sequences]

    def close(self):
        for part in getattr(self, "_parts", {}).values():
            part.close()
        if getattr(self, "h", None):
            self.lib.gkv_destroy(self.h)
            self.h = self._handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, st, what):
        if st != 0:
            raise GkvError(st, what)

    def set_param(self, name: str, value: int):
        self._check(self.lib.gkv_set_param(self.h, name.encode(), value), "gkv_set_param")
        self._params[name] = value
        for part in self._parts.values():
            part.set_param(name, value)

    def workspace_bytes(self) -> int:
        n = c_size_t()
        self._check(self.lib.gkv_workspace_bytes(self.h, byref(n)), "gkv_workspace_bytes")
        return n.value

    def set_step_base(self, d_step_base):
        """d_step_base: int32 device tensor of one element (or None for absolute steps)."""
        self._check(self.lib.gkv_set_step_base(self.h, _ptr(d_step_base)), "gkv_set_step_base")
        self._step_base = d_step_base
        for part in self._parts.values():
            part.set_step_base(d_step_base)

    def advance_step_base(self, delta: int):
        self._check(self.lib.gkv_advance_step_base(self.h, delta, _stream()), "gkv_advance_step_base")

    def workspace_init(self, workspace):
        self._check(self.lib.gkv_workspace_init(self.h, _ptr(workspace), _stream()), "gkv_workspace_init")

    def attend_decode(self, q, k_new, v_new, K, V, pos, step, qwin, d_state, len_max_host, out, workspace):
        st = self._call.gkv_attend_decode(self._handle, q, k_new, v_new, K, V, pos, step, qwin, d_state, len_max_host, out, workspace)
        if st is None:
            st = self.lib.gkv_attend_decode(self.h, _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(K), _ptr(V),
                                            _ptr(pos), step, _ptr(qwin), _ptr(d_state), len_max_host,
                                            _ptr(out), _ptr(workspace), _stream())
        if st:
            raise GkvError(st, "gkv_attend_decode")

    def score_window(self, qwin, K, d_state, step, len_max_host, S, workspace):
        st = self._call.gkv_score_window(self._handle, qwin, K, d_state, step, len_max_host, S, workspace)
        if st is None:
            st = self.lib.gkv_score_window(self.h, _ptr(qwin), _ptr(K), _ptr(d_state), step, len_max_host,
                                           _ptr(S), _ptr(workspace), _stream())
        if st:
            raise GkvError(st, "gkv_score_window")

    def global_update(self, S, F_hist, d_state, step, len_max_host, F_out):
        st = self._call.gkv_global_update(self._handle, S, F_hist, d_state, step, len_max_host, F_out)
        if st is None:
            st = self.lib.gkv_global_update(self.h, _ptr(S), _ptr(F_hist), _ptr(d_state), step,
                                            len_max_host, _ptr(F_out), _stream())
        if st:
            raise GkvError(st, "gkv_global_update")

    def select_topk(self, F, d_state, step, len_max_host, keep_idx, workspace):
        st = self._call.gkv_select_topk(self._handle, F, d_state, step, len_max_host, keep_idx, workspace)
        if st is None:
            st = self.lib.gkv_select_topk(self.h, _ptr(F), _ptr(d_state), step, len_max_host, _ptr(keep_idx),
                                          _ptr(workspace), _stream())
        if st:
            raise GkvError(st, "gkv_select_topk")

    def compact(self, keep_idx, F, K, V, F_hist, pos, d_state, step, workspace):
        st = self._call.gkv_compact(self._handle, keep_idx, F, K, V, F_hist, pos, d_state, step, workspace)
        if st is None:
            st = self.lib.gkv_compact(self.h, _ptr(keep_idx), _ptr(F), _ptr(K), _ptr(V), _ptr(F_hist),
                                      _ptr(pos), _ptr(d_state), step, _ptr(workspace), _stream())
        if st:
            raise GkvError(st, "gkv_compact")

    def evict(self, qwin, K, V, F_hist, pos, d_state, step, len_max_host, S, F, keep_idx, workspace):
        st = self._call.gkv_evict(self._handle, qwin, K, V, F_hist, pos, d_state, step, len_max_host, S, F, keep_idx, workspace)
        if st is None:
            st = self.lib.gkv_evict(self.h, _ptr(qwin), _ptr(K), _ptr(V), _ptr(F_hist), _ptr(pos),
                                    _ptr(d_state), step, len_max_host, _ptr(S), _ptr(F),
                                    _ptr(keep_idx), _ptr(workspace), _stream())
        if st:
            raise GkvError(st, "gkv_evict")

    def evict_static(self, qwin, K, V, F_hist, pos, d_state, step, len_max_host, workspace):
        self._check(self.lib.gkv_evict_static(self.h, _ptr(qwin), _ptr(K), _ptr(V), _ptr(F_hist), _ptr(pos),
                                              _ptr(d_state), step, len_max_host, _ptr(workspace), _stream()),
                    "gkv_evict_static")

    def redundancy_combine(self, K, d_state, step, len_max_host, F, lam, tau, eps, n_recent, R_norm, F_sel, workspace):
        st = self._call.gkv_redundancy_combine(self._handle, K, d_state, step, len_max_host, F, lam, tau, eps, n_recent, R_norm, F_sel, workspace)
        if st is None:
            st = self.lib.gkv_redundancy_combine(self.h, _ptr(K), _ptr(d_state), step, len_max_host, _ptr(F),
                                                 lam, tau, eps, n_recent, _ptr(R_norm), _ptr(F_sel),
                                                 _ptr(workspace), _stream())
        if st:
            raise GkvError(st, "gkv_redundancy_combine")

    def pool_scores(self, F, d_state, step, kernel, F_out):
        self._check(self.lib.gkv_pool_scores(self.h, _ptr(F), _ptr(d_state), step, kernel, _ptr(F_out), _stream()),
                    "gkv_pool_scores")

    def evicted_positions(self, keep_idx, pos, d_state, step, evicted):
        st = self._call.gkv_evicted_positions(self._handle, keep_idx, pos, d_state, step, evicted)
        if st is None:
            st = self.lib.gkv_evicted_positions(self.h, _ptr(keep_idx), _ptr(pos), _ptr(d_state), step,
                                                _ptr(evicted), _stream())
        if st:
            raise GkvError(st, "gkv_evicted_positions")

    # cache in 8 bits: K8, V8 torch.float8_e4m3fn [L,B,h_kv,capacity,d], scales bfloat16 [L,B,h_kv,capacity,2]
    def q8_store_prompt(self, k, v, n, t_first, t0, d_prompt_len, K8, V8, scales, pos):
        self._check(self.lib.gkv_q8_store_prompt(self.h, _ptr(k), _ptr(v), n, t_first, t0, _ptr(d_prompt_len), _ptr(K8),
                                                 _ptr(V8), _ptr(scales), _ptr(pos), _stream()), "gkv_q8_store_prompt")

    def q8_read(self, K8, V8, scales, d_state, step, K, V):
        self._check(self.lib.gkv_q8_read(self.h, _ptr(K8), _ptr(V8), _ptr(scales), _ptr(d_state), step, _ptr(K), _ptr(V),
                                         _stream()), "gkv_q8_read")

    def q8_attend_decode(self, q, k_new, v_new, K8, V8, scales, pos, step, qwin, d_state, len_max_host, part, out, workspace):
        st = self._call.gkv_q8_attend_decode(self._handle, q, k_new, v_new, K8, V8, scales, pos, step, qwin, d_state, len_max_host, part, out, workspace)
        if st is None:
            st = self.lib.gkv_q8_attend_decode(self.h, _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(K8), _ptr(V8), _ptr(scales),
                                               _ptr(pos), step, _ptr(qwin), _ptr(d_state), len_max_host, _ptr(part),
                                               _ptr(out), _ptr(workspace), _stream())
        if st:
            raise GkvError(st, "gkv_q8_attend_decode")

    def q8_score_window(self, qwin, K8, scales, d_state, step, len_max_host, S, workspace):
        st = self._call.gkv_q8_score_window(self._handle, qwin, K8, scales, d_state, step, len_max_host, S, workspace)
        if st is None:
            st = self.lib.gkv_q8_score_window(self.h, _ptr(qwin), _ptr(K8), _ptr(scales), _ptr(d_state), step, len_max_host,
                                              _ptr(S), _ptr(workspace), _stream())
        if st:
            raise GkvError(st, "gkv_q8_score_window")

    def q8_compact(self, keep_idx, F, K8, V8, scales, F_hist, pos, d_state, step, workspace):
        st = self._call.gkv_q8_compact(self._handle, keep_idx, F, K8, V8, scales, F_hist, pos, d_state, step, workspace)
        if st is None:
            st = self.lib.gkv_q8_compact(self.h, _ptr(keep_idx), _ptr(F), _ptr(K8), _ptr(V8), _ptr(scales), _ptr(F_hist),
                                         _ptr(pos), _ptr(d_state), step, _ptr(workspace), _stream())
        if st:
            raise GkvError(st, "gkv_q8_compact")

    def q8_evict(self, qwin, K8, V8, scales, F_hist, pos, d_state, step, len_max_host, S, F, keep_idx, workspace):
        st = self._call.gkv_q8_evict(self._handle, qwin, K8, V8, scales, F_hist, pos, d_state, step, len_max_host, S, F, keep_idx, workspace)
        if st is None:
            st = self.lib.gkv_q8_evict(self.h, _ptr(qwin), _ptr(K8), _ptr(V8), _ptr(scales), _ptr(F_hist), _ptr(pos),
                                       _ptr(d_state), step, len_max_host, _ptr(S), _ptr(F), _ptr(keep_idx),
                                       _ptr(workspace), _stream())
        if st:
            raise GkvError(st, "gkv_q8_evict")

    # prefix that sequences share: Kp, Vp [L,h_kv,prefix_capacity,d]; part: prefix_bytes(rows) bytes, zeroed once
    def prefix_bytes(self, rows: int) -> int:
        n = c_size_t()
        self._check(self.lib.gkv_prefix_bytes(self.h, rows, byref(n)), "gkv_prefix_bytes")
        self._prefix_bytes[rows], self._prefix_rows = n.value, max(rows, self._prefix_rows)
        return n.value

    def prefix_attend(self, q, Kp, Vp, rows, prefix_capacity, first, count, part):
        """Refuses a part that is too small for rows, which the C call cannot tell; rows beyond all that prefix_bytes() was asked for are its to refuse."""
        if part is not None and 0 <= rows <= self._prefix_rows:
            need = self._prefix_bytes.get(rows)
            if part.numel() * part.element_size() < (self.prefix_bytes(rows) if need is None else need):
                raise GkvError(GKV_ERR_WORKSPACE, "gkv_prefix_attend")
        st = self._call.gkv_prefix_attend(self._handle, q, Kp, Vp, rows, prefix_capacity, first, count, part)
        if st is None:
            st = self.lib.gkv_prefix_attend(self.h, _ptr(q), _ptr(Kp), _ptr(Vp), rows, prefix_capacity, first, count,
                                            _ptr(part), _stream())
        if st:
            raise GkvError(st, "gkv_prefix_attend")

    def attend_decode_prefix(self, q, k_new, v_new, K, V, pos, step, qwin, d_state, len_max_host, part, out, workspace):
        st = self._call.gkv_attend_decode_prefix(self._handle, q, k_new, v_new, K, V, pos, step, qwin, d_state, len_max_host, part, out, workspace)
        if st is None:
            st = self.lib.gkv_attend_decode_prefix(self.h, _ptr(q), _ptr(k_new), _ptr(v_new), _ptr(K), _ptr(V), _ptr(pos),
                                                   step, _ptr(qwin), _ptr(d_state), len_max_host, _ptr(part), _ptr(out),
                                                   _ptr(workspace), _stream())
        if st:
            raise GkvError(st, "gkv_attend_decode_prefix")

    def _heads(self, t, tokens, heads, what, apart=True):
        """A tensor [L, tokens, heads, d] as the calls take it: itself and 0, or, where tokens lie apart, its address and the elements between them."""
        if t is None:
            return None, 0
        L, d = self._spec.n_layers, self._spec.head_dim
        if t.shape != (L, tokens, heads, d) or t.dtype is not self._dtype:
            raise ValueError(f"gkv: {what} has to be [{L}, {tokens}, {heads}, {d}] of {self._dtype}, not {list(t.shape)} of {t.dtype}")
        if t.is_contiguous():
            return t, 0
        sl, st, sh, sd = t.stride()
        stride = st if tokens > 1 else sl
        if (not apart or (sd != 1 and d > 1) or (sh != d and heads > 1) or (L > 1 and sl != stride * tokens)
                or not heads * d <= stride < 1 << 31):
            raise ValueError(f"gkv: {what}'s heads have to lie side by side and its layers one behind the other" if apart
                             else f"gkv: {what} must be contiguous")
        return _ptr_here(t, False), stride

    def _pages(self, page_table, d_len, K, V):
        """Shapes of a paged cache: pages of a sequence, rows of a page, pages."""
        cfg = self._spec
        if K.dim() != 5 or (K.shape[0], K.shape[2], K.shape[4]) != (cfg.n_layers, cfg.n_kv_heads, cfg.head_dim) or V.shape != K.shape:
            raise ValueError(f"gkv: K and V have to be [{cfg.n_layers}, pages, {cfg.n_kv_heads}, rows, {cfg.head_dim}]")
        if K.dtype is not self._dtype or V.dtype is not self._dtype:
            raise ValueError(f"gkv: K and V have to be {self._dtype}")
        if page_table.dim() != 2:
            raise ValueError("gkv: page_table has to be [B, pages of a sequence]")
        self._ints(page_table, (cfg.batch, page_table.shape[1]), "page_table")
        self._ints(d_len, (cfg.batch,), "d_len")
        return page_table.shape[1], K.shape[3], K.shape[1]

    def _ints(self, t, shape, what, may_be_none=False):
        import torch
        if t is None and may_be_none:
            return
        if t.shape != shape or t.dtype is not torch.int32:
            raise ValueError(f"gkv: {what} has to be int32 {list(shape)}, not {t.dtype} {list(t.shape)}")

    def _freq(self, rotary):
        import torch
        if rotary.freq.dtype is not torch.float64 or rotary.freq.numel() < rotary.dim // 2:
            raise ValueError(f"gkv: frequencies have to be float64 [{rotary.dim // 2}]")

    def _turns(self, rotary, device):
        """Refuses a rotary that no call takes."""
        d, dim, f = self._spec.head_dim, rotary.dim, rotary.freq
        if (dim < 2 or dim % 2 or dim > d or not 0 <= rotary.layout <= 1 or not abs(rotary.amplitude) <= MOST_F32 or f.dtype is not self._double
                or f.numel() < dim // 2 or f.device != device or not f.is_contiguous()):
            raise ValueError(f"gkv: the rotary does not turn {dim} of {d} channels on {device}: layout {rotary.layout}, amplitude {rotary.amplitude}, "
                             f"frequencies {list(f.shape)} of {f.dtype} on {f.device}")

    # Rotary positions: q, k [L, tokens, heads, d], slices of one projection's output too; rotary: a Rotary.
    # Paged cache: K, V [L, n_pages, h_kv, page_rows, d], page_table int32 [B, table_width], d_len int32 [B].
    # The native half takes what has the right shapes, types and device; the rest is refused here, or goes through ctypes.
    def rotate(self, q, k, positions, step, rotary, q_out, k_out, transposed=False):
        r = rotary
        st = self._call.rotate(self._handle, self._spec_at, q, k, positions, step, r.freq, r.dim, r.layout, r.amplitude, int(transposed), q_out, k_out)
        if st is None:
            st = self._rotate(q, k, positions, step, r, q_out, k_out, transposed)
        if st:
            raise GkvError(st, "gkv_rotate")

    def _rotate(self, q, k, positions, step, r, q_out, k_out, transposed):
        cfg = self._spec
        if q is None and k is None:
            raise GkvError(1, "gkv_rotate")
        tokens = (k if q is None else q).shape[1]
        (q, qs), (k, ks) = self._heads(q, tokens, cfg.n_q_heads, "q"), self._heads(k, tokens, cfg.n_kv_heads, "k")
        q_out, _ = self._heads(q_out, tokens, cfg.n_q_heads, "q_out", False)
        k_out, _ = self._heads(k_out, tokens, cfg.n_kv_heads, "k_out", False)
        self._ints(positions, (tokens,), "positions", True)
        self._freq(r)
        if tokens == 0:
            return 0
        return self.lib.gkv_rotate(self.h, _ptr_here(q), qs, _ptr_here(k), ks, tokens, _ptr_here(positions), step, _ptr_here(r.freq), r.dim, r.layout,
                                   r.amplitude, int(transposed), _ptr_here(q_out), _ptr_here(k_out), _stream())

    def paged_advance(self, d_len, d_start):
        st = self._call.paged_advance(self._handle, self._spec_at, d_len, d_start)
        if st is None:
            self._ints(d_len, (self._spec.batch,), "d_len")
            self._ints(d_start, (self._spec.batch + 1,), "d_start", True)
            st = self.lib.gkv_paged_advance(self.h, _ptr_here(d_len), _ptr_here(d_start), _stream())
        if st:
            raise GkvError(st, "gkv_paged_advance")

    def paged_append(self, q, k, v, d_start, d_len, positions, rotary, page_table, K, V, q_out):
        """rotary: a Rotary, or None where keys are turned already (q and q_out are None then)."""
        freq, dim, layout, amplitude = (None, 0, 0, 1.0) if rotary is None else (rotary.freq, rotary.dim, rotary.layout, rotary.amplitude)
        st = self._call.paged_append(self._handle, self._spec_at, q, k, v, d_start, positions, freq, dim, layout, amplitude, d_len, page_table, K, V, q_out)
        if st is None:
            st = self._paged_append(q, k, v, d_start, d_len, positions, rotary, freq, dim, layout, amplitude, page_table, K, V, q_out)
        if st:
            raise GkvError(st, "gkv_paged_append")

    def _paged_append(self, q, k, v, d_start, d_len, positions, rotary, freq, dim, layout, amplitude, page_table, K, V, q_out):
        cfg = self._spec
        if k is None or v is None:
            raise GkvError(1, "gkv_paged_append")
        tokens = k.shape[1]
        (q, qs), (k, ks), (v, vs) = (self._heads(q, tokens, cfg.n_q_heads, "q"), self._heads(k, tokens, cfg.n_kv_heads, "k"),
                                     self._heads(v, tokens, cfg.n_kv_heads, "v"))
        q_out, _ = self._heads(q_out, tokens, cfg.n_q_heads, "q_out", False)
        self._ints(d_start, (cfg.batch + 1,), "d_start", True)
        self._ints(positions, (tokens,), "positions", True)
        if rotary is not None:
            self._freq(rotary)
        width, rows, pages = self._pages(page_table, d_len, K, V)
        if tokens == 0:
            return 0
        return self.lib.gkv_paged_append(self.h, _ptr_here(q), qs, _ptr_here(k), ks, _ptr_here(v), vs, tokens, _ptr_here(d_start), _ptr_here(d_len),
                                         _ptr_here(positions), _ptr_here(freq), dim, layout, amplitude, _ptr_here(page_table), width, rows, pages,
                                         _ptr_here(K), _ptr_here(V), _ptr_here(q_out), _stream())

    def paged_workspace_bytes(self) -> int:
        if self._paged_bytes is None:
            n = c_size_t()
            self._check(self.lib.gkv_paged_workspace_bytes(self.h, byref(n)), "gkv_paged_workspace_bytes")
            self._paged_bytes = n.value
        return self._paged_bytes

    def paged_attend_decode(self, q, K, V, page_table, d_len, len_max_host, out, workspace):
        """Refuses a workspace that is too small, which the C call cannot tell."""
        need = self._paged_bytes or self.paged_workspace_bytes()
        st = self._call.paged_attend_decode(self._handle, self._spec_at, q, d_len, page_table, K, V, len_max_host, out, workspace, need)
        if st is None:
            st = self._paged_attend_decode(q, K, V, page_table, d_len, len_max_host, out, workspace, need)
        if st:
            raise GkvError(st, "gkv_paged_attend_decode")

    def _paged_attend_decode(self, q, K, V, page_table, d_len, len_max_host, out, workspace, need):
        cfg = self._spec
        if workspace is not None and workspace.numel() * workspace.element_size() < need:
            return GKV_ERR_WORKSPACE
        q, _ = self._heads(q, cfg.batch, cfg.n_q_heads, "q", False)
        out, _ = self._heads(out, cfg.batch, cfg.n_q_heads, "out", False)
        width, rows, pages = self._pages(page_table, d_len, K, V)
        return self.lib.gkv_paged_attend_decode(self.h, _ptr_here(q), _ptr_here(K), _ptr_here(V), _ptr_here(page_table), width, rows, pages,
                                                _ptr_here(d_len), len_max_host, _ptr_here(out), _ptr_here(workspace), _stream())

    def profile_enable(self, on: bool):
        self._check(self.lib.gkv_profile_enable(self.h, int(on)), "gkv_profile_enable")
        self._profiled = bool(on)
        for part in self._parts.values():
            part.profile_enable(on)

    def profile_reset(self):
        self._check(self.lib.gkv_profile_reset(self.h), "gkv_profile_reset")
        for part in self._parts.values():
            part.profile_reset()

    def profile_read(self, kernel: str):
        ms, n = c_double(), c_int64()
        self._check(self.lib.gkv_profile_read(self.h, KERNEL_IDS[kernel], byref(ms), byref(n)), "gkv_profile_read")
        of_parts = [part.profile_read(kernel) for part in self._parts.values()]
        return ms.value + sum(x for x, _ in of_parts), n.value + sum(x for _, x in of_parts)


def probe_attend_read(K, V, rows, sink):
    """Enqueue one pass of the decode kernel's read pattern over rows [0, rows) of every unit of the
    bf16, d = 128 caches K, V [..., capacity, 128] (measurement aid)."""
    lib = load_library()
    cap = K.shape[-2]
    units = K.numel() // (cap * K.shape[-1])
    st = lib.gkv_probe_attend_read(_ptr(K), _ptr(V), units, cap, rows, _ptr(sink), _stream())
    if st != 0:
        raise GkvError(st, "gkv_probe_attend_read")


def cache_bytes(cfg: GkvConfig, rows: int, score_elem_bytes: int = 4):
    lib = load_library()
    kv, sc = c_size_t(), c_size_t()
    st = lib.gkv_cache_bytes(byref(cfg), rows, score_elem_bytes, byref(kv), byref(sc))
    if st != 0:
        raise GkvError(st, "gkv_cache_bytes")
    return kv.value, sc.value


def k_offset(cfg: GkvConfig, row: int, channel: int, n_tiled: int) -> int:
    return load_library().gkv_k_offset(byref(cfg), row, channel, n_tiled)

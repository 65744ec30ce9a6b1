"""Device buffers for one decode job, allocated through torch, plus the K-layout
permutations.  No arithmetic of the method lives here: each method below is one
call into the C ABI."""
from __future__ import annotations

import torch

from .binding import ST_LEN, ST_LEN_STEP, ST_N_HIST, ST_N_TILED, Context, GkvConfig, make_config

_TORCH_DTYPE = {0: torch.float32, 1: torch.bfloat16}


def k_rows_to_cache(K_rows: torch.Tensor, n_tiled: int) -> torch.Tensor:
    """[..., cap, d] row-major -> the library's K layout with the first n_tiled rows tiled."""
    n_tiled = n_tiled // 16 * 16
    out = K_rows.clone()
    if n_tiled:
        *lead, cap, d = K_rows.shape
        epc = 16 // K_rows.element_size()
        t = K_rows[..., :n_tiled, :].reshape(*lead, n_tiled // 16, 16, d // epc, epc)
        n = len(lead)
        t = t.permute(*range(n), n, n + 2, n + 1, n + 3).contiguous()
        out[..., :n_tiled, :] = t.reshape(*lead, n_tiled, d)
    return out


def k_cache_to_rows(K_cache: torch.Tensor, n_tiled: int) -> torch.Tensor:
    """Inverse of k_rows_to_cache."""
    n_tiled = n_tiled // 16 * 16
    out = K_cache.clone()
    if n_tiled:
        *lead, cap, d = K_cache.shape
        epc = 16 // K_cache.element_size()
        t = K_cache[..., :n_tiled, :].reshape(*lead, n_tiled // 16, d // epc, 16, epc)
        n = len(lead)
        t = t.permute(*range(n), n, n + 2, n + 1, n + 3).contiguous()
        out[..., :n_tiled, :] = t.reshape(*lead, n_tiled, d)
    return out


class DecodeState:
    """All device state of the path for L layers x B sequences."""

    def __init__(self, cfg: GkvConfig, device="cuda:0", params=None):
        self.cfg = cfg
        self.ctx = Context(cfg)
        for name, val in (params or {}).items():
            self.ctx.set_param(name, val)
        L, B, Hq, Hkv, d = cfg.n_layers, cfg.batch, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim
        cap, w, b = cfg.capacity, cfg.window, cfg.budget
        dt = _TORCH_DTYPE[cfg.dtype]
        dev = torch.device(device)
        self.device = dev
        z = lambda *s, dtype: torch.zeros(*s, dtype=dtype, device=dev)
        # the newest queries and keys, where they come not turned by their positions
        self._q_turned, self._k_turned = z(L, B, Hq, d, dtype=dt), z(L, B, Hkv, d, dtype=dt)
        self._allocate_cache()
        self.pos = torch.full((L, B, Hkv, cap), -1, dtype=torch.int32, device=dev)
        self.qwin = z(w, L, B, Hq, d, dtype=dt)          # ring of the last w q tensors
        self.d_state = z(L, B, 4, dtype=torch.int32)     # {len, len_step, n_hist, n_tiled}
        self.F_hist = z(L, B, Hkv, cap, dtype=torch.float32)
        self.S = z(L, B, Hkv, cap, dtype=torch.float32)
        self.F = z(L, B, Hkv, cap, dtype=torch.float32)
        self.R = z(L, B, Hkv, cap, dtype=torch.float32)      # normalised redundancy score
        self.F_sel = z(L, B, Hkv, cap, dtype=torch.float32)  # lambda*F - (1-lambda)*R'
        self.keep_idx = z(L, B, Hkv, b - w, dtype=torch.int32)
        self.evicted = torch.full((L, B, Hkv, cap - b), -1, dtype=torch.int32, device=dev)
        self.out = z(L, B, Hq, d, dtype=dt)
        self.workspace = torch.zeros(self.ctx.workspace_bytes(), dtype=torch.uint8, device=dev)
        self.ctx.workspace_init(self.workspace)
        # host mirror of the device records, for launch sizing and the trigger only: per sequence,
        # the cache length and the steps decoded since the cache was loaded or last compacted, both as
        # of the last time they were set apart; _grown rows and _stepped steps later for all of them
        self._set_host([0] * B, [0] * B)

    def _allocate_cache(self):
        cfg = self.cfg
        shape = (cfg.n_layers, cfg.batch, cfg.n_kv_heads, cfg.capacity, cfg.head_dim)
        # rows of K below N_TILED tiled, the rest row-major
        self.K, self.V = (torch.zeros(shape, dtype=_TORCH_DTYPE[cfg.dtype], device=self.device) for _ in range(2))

    @classmethod
    def from_workload(cls, wl, device="cuda:0", params=None, **over):
        kw = dict(n_layers=wl.n_layers, batch=wl.batch, n_q_heads=wl.n_q_heads, n_kv_heads=wl.n_kv_heads,
                  head_dim=wl.head_dim, budget=wl.budget, window=wl.window, interval=wl.interval,
                  capacity=wl.capacity, dtype=wl.dtype, combine=wl.combine, alpha=wl.alpha)
        kw.update(over)
        return cls(make_config(**kw), device=device, params=params)

    def _set_host(self, lengths, since):
        self._len0, self._since0, self._max0 = lengths, since, max(lengths)
        self._grown = self._stepped = 0

    @property
    def _len(self):
        return [x + self._grown for x in self._len0]

    @property
    def _since(self):
        return [x + self._stepped for x in self._since0]

    @property
    def len_host(self) -> int:
        """Upper bound of every sequence's length, as the calls' len_max_host wants it."""
        return self._max0 + self._grown

    @len_host.setter
    def len_host(self, value: int):
        """Declare every sequence `value` rows long with a full observation window."""
        self._set_host([int(value)] * self.cfg.batch, [self.cfg.window] * self.cfg.batch)

    # lengths as the kernels see them ---------------------------------------------------------
    def lengths(self, next_step: int) -> torch.Tensor:
        """[L,B] cache lengths before decode step `next_step` (LEN + next_step - LEN_STEP)."""
        return self.d_state[..., ST_LEN] + (next_step - self.d_state[..., ST_LEN_STEP])

    def set_state(self, length, len_step, n_hist, n_tiled):
        """Fill every (layer, sequence) record with the same values."""
        self.d_state[..., ST_LEN] = length
        self.d_state[..., ST_LEN_STEP] = len_step
        self.d_state[..., ST_N_HIST] = n_hist
        self.d_state[..., ST_N_TILED] = n_tiled
        self._set_host([int(length)] * self.cfg.batch, [0] * self.cfg.batch)

    def load_prefix(self, k, v, t0=0):
        """Place tokens t0..t0+n-1 (k, v: [n, L, B, h_kv, d]) as cache rows 0..n-1 with positions
        t0..t0+n-1, K row-major (N_TILED = 0).  For n <= budget this is exactly the state n
        appending decode steps leave behind (nothing is evicted before the cache exceeds the
        budget); pure data placement."""
        n = k.shape[0]
        assert n <= self.cfg.budget
        self.K.zero_(); self.V.zero_()
        self.K[..., :n, :] = k.to(self.V.dtype).permute(1, 2, 3, 0, 4)
        self.V[..., :n, :] = v.to(self.V.dtype).permute(1, 2, 3, 0, 4)
        self.pos.fill_(-1)
        self.pos[..., :n] = torch.arange(t0, t0 + n, dtype=torch.int32, device=self.device)
        self.set_state(n, t0 + n, 0, 0)

    def load_prompt_rows(self, t_first, k, v, t0, prompt_lens):
        """Place prompt tokens.  k, v [n, L, B, h_kv, d] hold positions t_first .. t_first+n-1 of
        every sequence's token stream; sequence i's prompt is the positions [t0 - P_i, t0) (a
        left-padded batch: decoding starts at step t0 for everyone) and goes to cache rows
        [0, P_i), K row-major.  May be called chunk by chunk; finish with begin_decode().
        Pure data placement."""
        n = k.shape[0]
        for i, P in enumerate(prompt_lens):
            lo = max(t_first, t0 - P)
            hi = min(t_first + n, t0)
            if hi <= lo:
                continue
            r0 = lo - (t0 - P)
            src = slice(lo - t_first, hi - t_first)
            self.K[:, i, :, r0:r0 + hi - lo] = k[src, :, i].to(self.K.dtype).permute(1, 2, 0, 3)
            self.V[:, i, :, r0:r0 + hi - lo] = v[src, :, i].to(self.V.dtype).permute(1, 2, 0, 3)
            self.pos[:, i, :, r0:r0 + hi - lo] = torch.arange(lo, hi, dtype=torch.int32, device=self.device)

    def begin_decode(self, t0, prompt_lens):
        """Records {P_i, t0, 0, 0}: sequence i holds P_i prompt rows before decode step t0."""
        rec = torch.tensor([[P, t0, 0, 0] for P in prompt_lens], dtype=torch.int32)
        self.d_state.copy_(rec.to(self.device).expand(self.cfg.n_layers, -1, -1))
        self._set_host([int(P) for P in prompt_lens], [0] * len(prompt_lens))

    def _after_compression(self):
        """Host mirror of what the compression kernels decide per sequence."""
        b, w = self.cfg.budget, self.cfg.window
        done = [n > b and k >= w for n, k in zip(self._len, self._since)]
        self._set_host([b if x else n for x, n in zip(done, self._len)], [0 if x else k for x, k in zip(done, self._since)])

    # one call each -------------------------------------------------------------------------
    def _turned(self, q, k_new, step, rotary):
        """q and k_new turned by the step.  Not in the step's slot of the window ring, whose query the next compression still needs where the
        decode call is refused: that call puts q there."""
        k_turned = None if k_new is None else self._k_turned
        self.ctx.rotate(q, k_new, None, step, rotary, self._q_turned, k_turned)
        return self._q_turned, k_turned

    def attend_decode(self, q, k_new, v_new, step, prefix=None, rotary=None):
        """prefix: a SharedPrefix, attended to together with the sequences' own rows.  rotary: a Rotary; q and k_new are not turned yet, `step` is
        their position, in every sequence, and the rows that the cache and prefixes hold are turned by theirs: row r of a prompt of n rows before the
        first step t by t - n + r.  With another prefix of the step, its attend() takes the same step and rotary."""
        if rotary is not None:
            q, k_new = self._turned(q, k_new, step, rotary)
        if prefix is None:
            self.ctx.attend_decode(q, k_new, v_new, self.K, self.V, self.pos, step, self.qwin, self.d_state,
                                   self.len_host, self.out, self.workspace)
        else:
            prefix.attend(q, self)
            self.ctx.attend_decode_prefix(q, k_new, v_new, self.K, self.V, self.pos, step, self.qwin, self.d_state,
                                          self.len_host, prefix.part, self.out, self.workspace)
        return self._stepped_on(k_new)

    def _stepped_on(self, k_new):
        if k_new is not None:
            self._grown += 1
        self._stepped += 1
        return self.out

    def score_window(self, step):
        self.ctx.score_window(self.qwin, self.K, self.d_state, step, self.len_host, self.S, self.workspace)

    def global_update(self, step):
        self.ctx.global_update(self.S, self.F_hist, self.d_state, step, self.len_host, self.F)

    def redundancy_combine(self, step, lam, tau, n_recent, eps=1e-8):
        self.ctx.redundancy_combine(self.K, self.d_state, step, self.len_host, self.F, lam, tau, eps, n_recent,
                                    self.R, self.F_sel, self.workspace)

    def select_topk(self, step, on_combined=False):
        self.ctx.select_topk(self.F_sel if on_combined else self.F, self.d_state, step, self.len_host,
                             self.keep_idx, self.workspace)

    def evicted_positions(self, step):
        """Eviction log of this compression; call between select_topk and compact."""
        self.ctx.evicted_positions(self.keep_idx, self.pos, self.d_state, step, self.evicted)

    def compact(self, step):
        self.ctx.compact(self.keep_idx, self.F, self.K, self.V, self.F_hist, self.pos, self.d_state, step,
                         self.workspace)
        self._after_compression()

    def evict(self, step):
        self.ctx.evict(self.qwin, self.K, self.V, self.F_hist, self.pos, self.d_state, step,
                       self.len_host, self.S, self.F, self.keep_idx, self.workspace)
        self._after_compression()

    def is_trigger(self, step) -> bool:
        """Host-side trigger: compression after every s generated tokens, if some sequence is above
        the budget with a full observation window (the kernels skip the others)."""
        b, w = self.cfg.budget, self.cfg.window
        return (step + 1) % self.cfg.interval == 0 and any(
            n > b and k >= w for n, k in zip(self._len, self._since))


class Q8DecodeState(DecodeState):
    """The same with K and V held in 8 bits: K8, V8 (codes) and scales (of a row of K and of V) in place of K and V.

    The redundancy term needs K in the configuration's type: redundancy_combine() reads it back part by part, into a buffer
    for one part that is made at its first call."""

    def _allocate_cache(self):
        cfg = self.cfg
        shape = (cfg.n_layers, cfg.batch, cfg.n_kv_heads, cfg.capacity)
        self.K8, self.V8 = (torch.zeros(*shape, cfg.head_dim, dtype=torch.uint8, device=self.device).view(torch.float8_e4m3fn)
                            for _ in range(2))
        self.scales = torch.ones(*shape, 2, dtype=torch.bfloat16, device=self.device)
        self.K = self.V = None
        self._part_ctx = self._K_part = None

    def load_prompt_rows(self, t_first, k, v, t0, prompt_lens):
        """As DecodeState's, quantised on the way.  Rows that would lie at or beyond the capacity are left out; begin_decode() refuses such prompts."""
        cfg, n, lens = self.cfg, k.shape[0], [int(P) for P in prompt_lens]
        row = (cfg.n_layers, cfg.batch, cfg.n_kv_heads, cfg.head_dim)
        if k.shape[1:] != row or v.shape != k.shape:
            raise ValueError(f"gkv: k and v have to be [n, {', '.join(map(str, row))}]")
        if len(lens) > cfg.batch:
            raise ValueError("gkv: more prompts than sequences")
        if n == 0:
            return
        k, v = (x.to(self.device, self.qwin.dtype).contiguous() for x in (k, v))
        lens = torch.tensor(lens + [0] * (cfg.batch - len(lens)), dtype=torch.int32).to(self.device)
        self.ctx.q8_store_prompt(k, v, n, t_first, t0, lens, self.K8, self.V8, self.scales, self.pos)

    def begin_decode(self, t0, prompt_lens):
        """As DecodeState's; refuses a prompt longer than the cache, whose last rows load_prompt_rows() has left out."""
        if max(prompt_lens) > self.cfg.capacity:
            raise ValueError(f"gkv: a prompt of {max(prompt_lens)} rows does not fit a capacity of {self.cfg.capacity}")
        super().begin_decode(t0, prompt_lens)

    def load_prefix(self, k, v, t0=0):
        """As DecodeState's, quantised on the way."""
        n = k.shape[0]
        assert n <= self.cfg.budget
        self.pos.fill_(-1)
        self.load_prompt_rows(t0, k, v, t0 + n, [n] * self.cfg.batch)
        self.set_state(n, t0 + n, 0, 0)

    def read(self, step, K=None, V=None):
        """The rows held before decode step `step` as a cache of the configuration's type, in the layout of d_state: into
        K and V, or into new buffers (rows that are not held are zero then)."""
        if K is None and V is None:
            K, V = (torch.zeros(self.K8.shape, dtype=self.qwin.dtype, device=self.device) for _ in range(2))
        for x in (K, V):
            if x is not None and (x.shape != self.K8.shape or x.dtype != self.qwin.dtype or x.device != self.K8.device):
                raise ValueError(f"gkv: K and V have to be {tuple(self.K8.shape)} of {self.qwin.dtype} on {self.K8.device}")
        self.ctx.q8_read(self.K8, self.V8, self.scales, self.d_state, step, K, V)
        return K, V

    def attend_decode(self, q, k_new, v_new, step, prefix=None, rotary=None):
        if rotary is not None:
            q, k_new = self._turned(q, k_new, step, rotary)
        if prefix is not None:
            prefix.attend(q, self)
        self.ctx.q8_attend_decode(q, k_new, v_new, self.K8, self.V8, self.scales, self.pos, step, self.qwin, self.d_state,
                                  self.len_host, None if prefix is None else prefix.part, self.out, self.workspace)
        return self._stepped_on(k_new)

    def score_window(self, step):
        self.ctx.q8_score_window(self.qwin, self.K8, self.scales, self.d_state, step, self.len_host, self.S, self.workspace)

    def _parts(self):
        """The (layer, sequence)s in parts: [(first, context of that many sequences)].  A part is a whole round of the redundancy kernel, a
        workgroup for each compute unit; the last two share what is left, as launches of up to 128 (sequence, KV head)s go another way.
        (us, all of K at once / parts twice as large / these: 896 units of 640 rows 166 / 172 / 182, 18432 of 1088 7420 / 7400 / 7770.)"""
        if self._part_ctx is None:
            cfg, n = self.cfg, self.cfg.n_layers * self.cfg.batch
            at_once = max(1, 256 // cfg.n_kv_heads)
            cuts = list(range(0, n, at_once)) + [n]
            if len(cuts) > 2 and (n - cuts[-2]) * cfg.n_kv_heads <= 128:
                cuts[-2] = (cuts[-3] + n) // 2
            self._part_ctx = [(lo, self.ctx.part(hi - lo)) for lo, hi in zip(cuts, cuts[1:])]
            most = max(hi - lo for lo, hi in zip(cuts, cuts[1:]))
            self._K_part = torch.empty(most, *self.K8.shape[2:], dtype=self.qwin.dtype, device=self.device)
        return self._part_ctx

    def redundancy_combine(self, step, lam, tau, n_recent, eps=1e-8):
        of = lambda x, lo, n: x.flatten(0, 1)[lo:lo + n]
        for lo, ctx in self._parts():
            n = ctx.cfg.batch
            K, d_state = self._K_part[:n], of(self.d_state, lo, n)
            ctx.q8_read(of(self.K8, lo, n), None, of(self.scales, lo, n), d_state, step + 1, K, None)
            ctx.redundancy_combine(K, d_state, step, self.len_host, of(self.F, lo, n), lam, tau, eps, n_recent,
                                   of(self.R, lo, n), of(self.F_sel, lo, n), None)

    def compact(self, step):
        self.ctx.q8_compact(self.keep_idx, self.F, self.K8, self.V8, self.scales, self.F_hist, self.pos, self.d_state, step,
                            self.workspace)
        self._after_compression()

    def evict(self, step):
        self.ctx.q8_evict(self.qwin, self.K8, self.V8, self.scales, self.F_hist, self.pos, self.d_state, step, self.len_host,
                          self.S, self.F, self.keep_idx, self.workspace)
        self._after_compression()


def _recording():
    return torch.cuda.is_initialized() and torch.cuda.is_current_stream_capturing()


class PagedDecodeState:
    """Device state of L layers x B sequences whose rows are all kept, in pages: full attention beside the capped caches, or to compare
    with.  Of cfg the shapes, type and scale count.  Pages are handed out as sequences grow and come back with release().

    max_rows: rows a sequence may have at most.  n_pages: pages of the cache, for all sequences together (default: enough for all of that length).
    rotary: a Rotary; queries and keys are turned by their positions on the way in, which are their rows unless given."""

    def __init__(self, cfg: GkvConfig, max_rows, page_rows=64, n_pages=None, rotary=None, device="cuda:0", params=None):
        self.cfg, self.ctx, self.rotary, self.page_rows = cfg, Context(cfg), rotary, page_rows
        for name, val in (params or {}).items():
            self.ctx.set_param(name, val)
        L, B, Hq, Hkv, d = cfg.n_layers, cfg.batch, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim
        self.device, dt = torch.device(device), _TORCH_DTYPE[cfg.dtype]
        if max_rows < 1 or page_rows < 1:
            raise ValueError("gkv: sequences and pages have at least one row")
        width = -(-max_rows // page_rows)
        n_pages = B * width if n_pages is None else n_pages
        if n_pages < 1 or width * page_rows > 1 << 30:
            raise ValueError("gkv: a cache has at least one page, and a sequence at most 2^30 rows")
        z = lambda *s, dtype=dt: torch.zeros(*s, dtype=dtype, device=self.device)
        self.K, self.V = z(L, n_pages, Hkv, page_rows, d), z(L, n_pages, Hkv, page_rows, d)
        self.page_table = torch.full((B, width), -1, dtype=torch.int32, device=self.device)
        self.d_len = z(B, dtype=torch.int32)
        if rotary is not None:
            self.ctx._turns(rotary, self.K.device)
        self.out, self.q_turned = z(L, B, Hq, d), z(L, B, Hq, d)
        self.workspace = z(self.ctx.paged_workspace_bytes(), dtype=torch.uint8)
        self._table = torch.full((B, width), -1, dtype=torch.int32)          # host mirror
        self._free = list(range(n_pages))[::-1]
        self._pages = [0] * B                                                # of each sequence
        self._settle([0] * B)

    def _settle(self, lens):
        """Host mirror of the lengths (-1: takes no part), as of now; _grown rows later for all that take part, and at most _room of them
        until one needs a page more."""
        self._len0, self._grown = lens, 0
        self._room = min([p * self.page_rows - n for p, n in zip(self._pages, lens) if n >= 0], default=1 << 30)

    @property
    def _len(self):
        return [n + self._grown if n >= 0 else n for n in self._len0]

    @property
    def lengths(self):
        """Rows of each sequence."""
        return [max(n, 0) for n in self._len]

    def reserve(self, rows):
        """Pages for sequences of so many rows (one number, or one for each): steps up to there change the lengths alone and can be recorded.
        Calls that need pages send the whole table and wait for it, so a growing batch reserves ahead."""
        rows = [rows] * self.cfg.batch if isinstance(rows, int) else list(rows)
        if len(rows) != self.cfg.batch:
            raise ValueError(f"gkv: lengths of {self.cfg.batch} sequences are wanted")
        want = [max(-(-n // self.page_rows), have) for n, have in zip(rows, self._pages)]
        if want == self._pages:
            return
        if max(want) > self._table.shape[1]:
            raise ValueError(f"gkv: a sequence of {max(rows)} rows is longer than {self._table.shape[1]} pages of {self.page_rows}")
        if sum(want) - sum(self._pages) > len(self._free):
            raise ValueError(f"gkv: {sum(want) - sum(self._pages)} pages are needed, {len(self._free)} are free")
        if _recording():
            raise ValueError("gkv: pages are not handed out while steps are recorded: reserve() comes first")
        for i, n in enumerate(want):
            for p in range(self._pages[i], n):
                self._table[i, p] = self._free.pop()
        self._pages = want
        self._settle(self._len)
        self.page_table.copy_(self._table)

    def release(self, i):
        """Sequence i's pages come back, and it takes no part until append() gives it tokens again."""
        if not 0 <= i < self.cfg.batch:
            raise ValueError(f"gkv: there is no sequence {i}")
        if _recording():
            raise ValueError("gkv: a sequence does not leave while steps are recorded")
        self._free += [int(p) for p in self._table[i, :self._pages[i]].flip(0)]
        self._table[i] = -1
        self._pages[i] = 0
        self._settle([-1 if k == i else n for k, n in enumerate(self._len)])
        self.page_table[i] = -1
        self.d_len[i] = -1

    def append(self, k, v, counts=None, q=None, positions=None, q_out=None):
        """New tokens k, v [L, tokens, h_kv, d], packed: counts of them for each sequence (None: one for each that takes part, tokens = B); tokens
        behind the last are padding.  Returns q [L, tokens, h_q, d] turned, in q_out or a new tensor, if it is given."""
        cfg, ctx = self.cfg, self.ctx
        # all that can be wrong is looked at before anything grows
        if k is None or v is None:
            raise ValueError("gkv: keys and values are wanted")
        if q is None and q_out is not None:
            raise ValueError("gkv: q_out is for queries that are given")
        ctx._heads(k, k.shape[1], cfg.n_kv_heads, "k")
        ctx._heads(v, k.shape[1], cfg.n_kv_heads, "v")
        ctx._heads(q, k.shape[1], cfg.n_q_heads, "q")
        ctx._heads(q_out, k.shape[1], cfg.n_q_heads, "q_out", False)
        ctx._ints(positions, (k.shape[1],), "positions", True)
        if positions is not None and not positions.is_contiguous():
            raise ValueError("gkv: positions must be contiguous")
        here = self.K.device
        for x in (k, v, q, q_out, positions):
            if x is not None and x.device != here:
                raise ValueError(f"gkv: tensors have to be on {here}")
        if self.K.is_cuda and here.index != torch.cuda.current_device():
            raise ValueError(f"gkv: the state is on {here}, which is not the current GPU")
        if q_out is not None and q_out.data_ptr() == q.data_ptr() and not q.is_contiguous():
            raise ValueError("gkv: queries that lie apart are not turned in place")
        if counts is not None and (len(counts) != cfg.batch or min(counts) < 0 or sum(counts) > k.shape[1]):
            raise ValueError(f"gkv: {cfg.batch} counts of {k.shape[1]} tokens are wanted")
        if counts is None and k.shape[1] != cfg.batch:
            raise ValueError(f"gkv: one token for each of {cfg.batch} sequences is wanted")
        if cfg.n_layers * k.shape[1] >= 1 << 24:
            raise ValueError(f"gkv: {k.shape[1]} tokens of {cfg.n_layers} layers are too many for one call")
        if self.rotary is None and q is not None:
            raise ValueError("gkv: queries are turned where there is a rotary")
        if self.rotary is not None:
            ctx._turns(self.rotary, here)
        if counts is not None and _recording():
            raise ValueError("gkv: counts come from the host and are not recorded")
        start = None if counts is None else torch.tensor([0, *counts], dtype=torch.int32).cumsum(0, dtype=torch.int32).to(self.device)
        if q is not None and q_out is None:
            q_out = torch.zeros(q.shape, dtype=q.dtype, device=q.device)
        if counts is not None:
            lens = [max(n, 0) + m if m else n for n, m in zip(self._len, counts)]
            self.reserve(lens)
            self._settle(lens)
        else:
            if self._room < 1:
                self.reserve([n + 1 if n >= 0 else 0 for n in self._len])
            self._grown += 1
            self._room -= 1
        ctx.paged_advance(self.d_len, start)
        ctx.paged_append(q, k, v, start, self.d_len, positions, self.rotary, self.page_table, self.K, self.V, q_out)
        return q_out

    def attend(self, q):
        """The newest tokens' queries, turned, over all rows."""
        self.ctx.paged_attend_decode(q, self.K, self.V, self.page_table, self.d_len, max(self._pages) * self.page_rows, self.out, self.workspace)
        return self.out

    def attend_decode(self, q, k_new, v_new, positions=None):
        """One decode step: q [L, B, h_q, d], k_new, v_new [L, B, h_kv, d]."""
        # (queries that attend() would refuse, before anything grows)
        if q is None:
            raise ValueError("gkv: q is wanted")
        self.ctx._heads(q, self.cfg.batch, self.cfg.n_q_heads, "q", self.rotary is not None)
        if q.device != self.K.device:
            raise ValueError(f"gkv: tensors have to be on {self.K.device}")
        if self.rotary is None:
            self.append(k_new, v_new)
        else:
            q = self.append(k_new, v_new, None, q, positions, self.q_turned)
        return self.attend(q)

    def replayed(self, steps=1):
        """So many decode steps are made by replays of recorded ones that this object does not know of (recording a step counts it once).
        Say so before they run: steps beyond the reserved rows are refused, since rows without a page are not stored."""
        if steps < 0:
            raise ValueError("gkv: a number of steps is wanted")
        if steps > self._room:
            raise ValueError(f"gkv: {steps} steps of {self._room} that there are pages for: reserve() comes first")
        self._grown += steps
        self._room -= steps


class SharedPrefix:
    """Keys and values [L, h_kv, rows, d] of a prompt that the sequences of a DecodeState (or Q8DecodeState) share, held
    once; with first and count, those sequences of the batch alone."""

    def __init__(self, state: DecodeState, k, v, first=0, count=None, part=None):
        """part: another SharedPrefix of the same state whose sequences are others: one step then joins both, through
        attend() of this one and attend_decode(..., prefix=the other); where that has a rotary, attend(q, step=step, rotary=rotary)."""
        dt, cfg = state.qwin.dtype, state.cfg
        if k.dim() != 4 or (k.shape[0], k.shape[1], k.shape[3]) != (cfg.n_layers, cfg.n_kv_heads, cfg.head_dim) or v.shape != k.shape:
            raise ValueError(f"gkv: a prefix's k and v have to be [{cfg.n_layers}, {cfg.n_kv_heads}, rows, {cfg.head_dim}]")
        if part is not None and part.ctx is not state.ctx:
            raise ValueError("gkv: the other prefix is of another state")
        self.ctx, self._q_turned = state.ctx, state._q_turned
        self.K, self.V = k.to(state.device, dt).contiguous(), v.to(state.device, dt).contiguous()
        self.rows, self.first = k.shape[2], first
        self.count = state.cfg.batch - first if count is None else count
        need = self.ctx.prefix_bytes(self.rows)
        self.part = torch.zeros(need, dtype=torch.uint8, device=state.device) if part is None else part.part
        if self.part.numel() < need:
            raise ValueError("gkv: make the longer prefix first, its buffer holds the shorter one's pieces too")

    def attend(self, q, state=None, step=None, rotary=None):
        """The newest queries over the prefix; attend_decode() with a prefix does it by itself.  rotary: a Rotary; q is not turned yet, `step` is
        its position.  Without one q is taken as it is: turned, where the prefix's keys are."""
        if state is not None and state.ctx is not self.ctx:
            raise ValueError("gkv: the prefix is of another state")
        if rotary is not None:
            if step is None:
                raise ValueError("gkv: a rotary needs the step that queries are turned by")
            self.ctx.rotate(q, None, None, step, rotary, self._q_turned, None)
            q = self._q_turned
        self.ctx.prefix_attend(q, self.K, self.V, self.rows, self.rows, self.first, self.count, self.part)

"""Timing cases of the operators around the decode path that hold the cache in 8 bits or share a prefix.

A case is one of seven kinds of call:
  store    q8_store_prompt: prompt rows of K and V quantised into an 8-bit cache
  read     q8_read: an 8-bit cache read back into a cache of the configuration's type
  attend   q8_attend_decode: one decode step of all layers that share a context, on an 8-bit cache
  window   the last w decode steps before a compression and the window score behind them (8-bit cache)
  score    q8_score_window on its own: the rows' softmax statistics are not there yet
  compact  q8_compact: the kept rows of an 8-bit cache moved to the front, in place
  shared   prefix_attend and the decode step that joins it: a prompt held once for the whole batch

An element of an 8-bit cache is an e4m3 code times its row's scale, a power of two:
  e = min { e >= -126 : max |x| <= 448 * 2^e },   code = e4m3(x * 2^-e),   value = code * 2^e.
K rows below n_tiled lie chunk by chunk in tiles of 16 rows (16-byte chunks), the others row by row.

Shapes are the workload configurations in gkv_traces and the head shapes, dtypes and window sizes the
tests cover.  Keys have outlier channels and a few boosted positions ("recurring") or Student-t
entries ("heavy_tail").
"""
import math

import torch

own = False

_DT = {"bf16": torch.bfloat16, "f32": torch.float32}
F8 = torch.float8_e4m3fn


def _case(name, kind, L, B, hq, hkv, d, dtype, b, w, s, rows=0, recipe="recurring", **more):
    """rows: prompt rows (store), cache rows when the call is made (read, attend: before the step; shared: of the
    sequences' own caches) or rows the compression sees (window, score, compact; 0 = b + s)."""
    c = dict(name=name, kind=kind, L=L, B=B, hq=hq, hkv=hkv, d=d, dtype=dtype, b=b, w=w, s=s,
             rows=rows or b + s, recipe=recipe, lens="equal", prefix=0, cache="q8")
    c.update(more)
    return c


def listed():
    return [
        # a short prompt of the tiny fp32 configuration: latency
        _case("store_tiny_f32", "store", 1, 1, 8, 2, 64, "f32", 64, 8, 16, rows=37),
        # prompts of different lengths at the headline configuration, all 28 layers
        _case("store_ragged_28layer", "store", 28, 8, 28, 4, 128, "bf16", 512, 16, 128, rows=509, lens="ragged"),
        # one layer's cache read back, for a call that wants the configuration's type
        _case("read_layer", "read", 1, 32, 28, 4, 128, "bf16", 1024, 16, 128, rows=1090),
        # the whole cache of 28 layers and a batch of 16
        _case("read_28layer_b1024", "read", 28, 16, 28, 4, 128, "bf16", 1024, 16, 128, rows=1151),
        # a decode step of the tiny fp32 configuration: latency
        _case("attend_tiny_f32", "attend", 1, 1, 8, 2, 64, "f32", 64, 8, 16, rows=72),
        # the large-batch configuration's decode step: 5 GB of cache, heavy-tailed keys
        _case("attend_large_batch", "attend", 36, 64, 40, 8, 128, "bf16", 1024, 32, 64, rows=1056, recipe="heavy_tail"),
        # the headline configuration's last 16 decode steps before a compression, and its scoring
        _case("window_28layer_b512", "window", 28, 8, 28, 4, 128, "bf16", 512, 16, 128),
        # scoring of a cache that was loaded and not decoded here
        _case("score_layer_b2048", "score", 1, 16, 40, 8, 128, "bf16", 2048, 32, 64),
        # compaction of one sequence's layer: latency
        _case("compact_layer", "compact", 1, 1, 28, 4, 128, "bf16", 512, 16, 128),
        # compaction at budget 2048, batch 16, 28 layers
        _case("compact_28layer_b2048", "compact", 28, 16, 28, 4, 128, "bf16", 2048, 16, 128),
        # four answers to one prompt, one layer of the small-model head shape, plain cache: latency
        _case("shared_few", "shared", 1, 4, 10, 2, 64, "bf16", 512, 32, 32, rows=300, prefix=2011, cache="plain"),
        # 64 answers to one long prompt at the 40q/8kv shape, four layers of a model in pieces
        _case("shared_batch64_p16k", "shared", 4, 64, 40, 8, 128, "bf16", 1024, 32, 64, rows=1056, prefix=16384),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["store", "read", "attend", "attend", "attend", "window", "score", "compact", "shared", "shared", "shared"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "bf16", "f32"])
    d = rng.choice([128, 128, 128, 64])
    hkv = rng.choice([1, 2, 4, 8])
    g = rng.choice([1, 2, 3, 4, 5, 7, 7, 8, 16])
    w = rng.choice([8, 16, 16, 32])
    s = rng.choice([32, 48, 64, 100, 128])
    b = _log_int(rng, 64, 2048)
    recipe = rng.choice(["recurring", "recurring", "heavy_tail"])
    lens, rows, prefix, cache = "equal", 0, 0, "q8"
    units = _log_int(rng, 4, 4000)
    limit = 1 << 28                                   # elements of K
    if kind == "store":
        rows, lens = _log_int(rng, 1, b), rng.choice(["equal", "ragged"])
    elif kind == "read":
        rows, lens = _log_int(rng, 1, b + s), rng.choice(["equal", "ragged"])
    elif kind == "attend":
        rows = b + rng.randrange(s)
        lens = rng.choice(["equal", "equal", "ragged"])
        limit = 1 << (28 if dtype == "f32" else 29)
    elif kind in ("window", "score"):
        limit = min(1 << 26, (1 << 28) * d // (w * g))  # the plain form holds w * g logits a key
    elif kind == "shared":
        rows = _log_int(rng, 1, b + s - 1)
        prefix = _log_int(rng, 1, 65536)
        cache = rng.choice(["q8", "plain"])
        units = _log_int(rng, 4, 1000)
        # units * g * (rows + prefix) logits
        limit = min(1 << 26, (1 << (27 if dtype == "bf16" else 25)) * d // (g * (rows + prefix)) * rows)
    units = max(hkv, min(units, limit // (d * (rows or b + s))))
    lb = max(1, units // hkv)
    L = rng.choice([x for x in (1, 1, 2, 4, 14, 28) if x <= lb])
    if kind == "shared":
        while L > 1 and L * hkv * prefix * d > 1 << 28:
            L //= 2
    return {k: v for k, v in _case("", kind, L, max(1, lb // L), g * hkv, hkv, d, dtype, b, w, s, rows, recipe,
                                   lens=lens, prefix=prefix, cache=cache).items() if k != "name"}


# ---- shapes ---------------------------------------------------------------------------------
def _lens(case):
    B, n = case["B"], case["rows"]
    if case["lens"] == "equal":
        return [n] * B
    return [max(1, n * (i + 1) // B - (i * 7) % 13) for i in range(B)]


def _cap(case):
    return -(-max(case["b"] + case["s"], case["rows"] + 1) // 32) * 32


def _tiled(case):
    """Leading K rows that an earlier compression left in tiles; prompts lie row by row."""
    T = case["b"] // 16 * 16
    return 0 if case["lens"] == "ragged" or case["rows"] < case["b"] or case["kind"] == "store" else T


def _filled(case):
    """Rows in the cache before the call."""
    return case["rows"] - case["w"] if case["kind"] == "window" else case["rows"]


# ---- inputs ---------------------------------------------------------------------------------
class _Inputs:
    """Draws, layer by layer, from one generator: the same values for prepare() and exact()."""

    def __init__(self, case, seed):
        self.c = case
        self.dev = torch.device("cuda")
        self.g = torch.Generator(device="cuda").manual_seed(int(seed) * 1000003 + 29)
        L, hkv, d = case["L"], case["hkv"], case["d"]
        u = torch.randn(L, hkv, d, generator=self.g, device=self.dev)
        self.u = u / u.norm(dim=-1, keepdim=True)
        self.scale = torch.ones(L, hkv, d, device=self.dev)
        ch = torch.rand(L, hkv, d, generator=self.g, device=self.dev).topk(4, dim=-1).indices
        self.scale.scatter_(-1, ch, 10.0)
        self.boost = math.sqrt(8.0 * math.sqrt(d))

    def _n(self, *shape):
        return torch.randn(*shape, generator=self.g, device=self.dev)

    def keys(self, layer, *lead):
        """[*lead, hkv, d] keys of one layer on the case's dtype grid."""
        shape = (*lead, self.c["hkv"], self.c["d"])
        k = self._n(*shape)
        if self.c["recipe"] == "heavy_tail":
            chi = self._n(*shape).square_()
            chi += self._n(*shape).square_()
            chi += self._n(*shape).square_()
            k /= (chi / 3.0).sqrt_()
        else:
            k *= self.scale[layer]
            hit = torch.rand(*lead, 1, 1, generator=self.g, device=self.dev) < 0.01
            k += hit * (self.boost * self.u[layer])
        return k.to(_DT[self.c["dtype"]])

    def values(self, *lead):
        return self._n(*lead, self.c["hkv"], self.c["d"]).to(_DT[self.c["dtype"]])

    def queries(self, layer, n):
        """[n, B, hq, d]; a recall burst covers a tenth of the steps."""
        c = self.c
        q = self._n(n, c["B"], c["hq"], c["d"])
        if c["recipe"] != "heavy_tail":
            hit = torch.rand(n, 1, 1, 1, generator=self.g, device=self.dev) < 0.1
            q += hit * (self.boost * self.u[layer].repeat_interleave(c["hq"] // c["hkv"], dim=0))
        return q.to(_DT[c["dtype"]])

    def cache(self, layer, rows):
        """K, V [B, hkv, rows, d] of one layer."""
        k = self.keys(layer, self.c["B"], rows).transpose(1, 2).contiguous()
        v = self.values(self.c["B"], rows).transpose(1, 2).contiguous()
        return k, v

    def prefix(self, layer):
        """K, V [hkv, prefix, d] of one layer's shared prompt."""
        n = self.c["prefix"]
        k = self.keys(layer, n).transpose(0, 1).contiguous()
        v = self.values(n).transpose(0, 1).contiguous()
        return k, v

    def tokens(self, n):
        """q [n, L, B, hq, d], k, v [n, L, B, hkv, d]."""
        c = self.c
        q, k, v = [], [], []
        for layer in range(c["L"]):
            q.append(self.queries(layer, n))
            k.append(self.keys(layer, n, c["B"]))
            v.append(self.values(n, c["B"]))
        return [torch.stack(x, dim=1).contiguous() for x in (q, k, v)]

    def keep(self, n_cand, n_keep):
        c = self.c
        r = torch.rand(c["L"], c["B"], c["hkv"], n_cand, generator=self.g, device=self.dev)
        return r.topk(n_keep, dim=-1).indices.sort(dim=-1).values.int()

    def scores(self, rows):
        c = self.c
        return torch.rand(c["L"], c["B"], c["hkv"], rows, generator=self.g, device=self.dev).pow_(4)


# ---- the plain form: elementary operations in 32 bits ----------------------------------------
def _exponent(x):
    """Exponents of the rows' scales, [..., 1]."""
    m, e = torch.frexp(x.abs().amax(dim=-1, keepdim=True))
    e = e - 9 + (m > 0.875).to(e.dtype)
    return torch.where(m == 0, torch.zeros_like(e), e.clamp(min=-126))


def _power_of_two(e):
    """2^e for -126 <= e <= 127, from its bits (pow() is not always exact)."""
    return ((e + 127) << 23).view(torch.float32)


def _quantise(x):
    """codes [..., d] (e4m3) and scales [..., 1] of float32 rows."""
    e = _exponent(x).int()
    return (x * _power_of_two(-e)).to(F8), _power_of_two(e)


def _tile(rows, T):
    """K rows [..., n, d] -> the cache's order with the first T rows in tiles."""
    if not T:
        return rows
    *lead, n, d = rows.shape
    E = 16 // rows.element_size()
    t = rows[..., :T, :].reshape(*lead, T // 16, 16, d // E, E).transpose(-3, -2).reshape(*lead, T, d)
    return torch.cat([t, rows[..., T:, :]], dim=-2)


def _untile(cache, T):
    if not T:
        return cache
    *lead, n, d = cache.shape
    E = 16 // cache.element_size()
    t = cache[..., :T, :].reshape(*lead, T // 16, d // E, 16, E).transpose(-3, -2).reshape(*lead, T, d)
    return torch.cat([t, cache[..., T:, :]], dim=-2)


def _values(S, which, n):
    """float32 rows [0, n) of the 8-bit K (0) or V (1)."""
    codes = (S.K8, S.V8)[which].view(torch.uint8)[..., : -(-n // 16) * 16, :]
    rows = _untile(codes, S.T)[..., :n, :] if which == 0 else codes[..., :n, :]
    return rows.view(F8).float() * S.scales[..., :n, which:which + 1].float()


def _append(S, k, v, at, step):
    """The new rows [L, B, hkv, d] into row at[i] of sequence i, and what goes with them."""
    seq = torch.arange(S.c["B"], device=k.device)
    if S.c["cache"] == "q8":
        for which, cache, x in ((0, S.K8, k), (1, S.V8, v)):
            code, scale = _quantise(x.float())
            cache.view(torch.uint8)[:, seq, :, at] = code.view(torch.uint8).transpose(0, 1)
            S.scales[:, seq, :, at, which] = scale[..., 0].to(S.scales.dtype).transpose(0, 1)
    else:
        S.K[:, seq, :, at] = k.transpose(0, 1)
        S.V[:, seq, :, at] = v.transpose(0, 1)
    S.pos[:, seq, :, at] = step


def _cached(S, n):
    if S.c["cache"] == "q8":
        return _values(S, 0, n), _values(S, 1, n)
    m = -(-n // 16) * 16
    return _untile(S.K[..., :m, :], S.T)[..., :n, :].float(), S.V[..., :n, :].float()


def _logits(S, q, K, seen):
    """[L, B, hkv, g, n] logits of q [L, B, hq, d]; sequence i sees rows [0, seen[i])."""
    c = S.c
    z = torch.matmul(q.float().view(c["L"], c["B"], c["hkv"], -1, c["d"]), K.transpose(-1, -2)) / math.sqrt(c["d"])
    dead = torch.arange(K.shape[-2], device=K.device).view(1, 1, 1, 1, -1) >= seen.view(1, -1, 1, 1, 1)
    return z.masked_fill(dead, float("-inf"))


def _attend(S, q, k, v, step, at, most):
    _append(S, k, v, at, step)
    K, V = _cached(S, most)
    z = _logits(S, q, K, at + 1)
    p = torch.exp(z - z.amax(dim=-1, keepdim=True))
    o = torch.matmul(p, V) / p.sum(dim=-1, keepdim=True)
    S.qwin[step % S.c["w"]] = q
    return o.view(q.shape).to(q.dtype)


def _shared(S):
    c = S.c
    L, B, hkv, d, P = c["L"], c["B"], c["hkv"], c["d"], c["prefix"]
    _append(S, S.k, S.v, S.at, S.step)
    K, V = _cached(S, max(S.lens) + 1)
    z = _logits(S, S.q, K, S.at + 1)
    qp = S.q.float().view(L, B, hkv, -1, d).transpose(1, 2).reshape(L, hkv, -1, d)
    zp = torch.matmul(qp, S.Kp.float().transpose(-1, -2)) / math.sqrt(d)
    zp = zp.view(L, hkv, B, -1, P)
    m = torch.maximum(z.amax(dim=-1, keepdim=True), zp.amax(dim=-1, keepdim=True).transpose(1, 2))
    p = torch.exp(z - m)
    pp = torch.exp(zp - m.transpose(1, 2))
    total = p.sum(dim=-1, keepdim=True) + pp.sum(dim=-1, keepdim=True).transpose(1, 2)
    op = torch.matmul(pp.view(L, hkv, -1, P), S.Vp.float()).view(L, hkv, B, -1, d).transpose(1, 2)
    S.qwin[S.step % c["w"]] = S.q
    return ((torch.matmul(p, V) + op) / total).reshape(S.q.shape).to(S.q.dtype)


def _score(S, step):
    """Local scores of the candidates: the window rows' softmax over the keys each saw, the largest of a group's
    heads, the mean over the window."""
    c = S.c
    w, l = c["w"], c["rows"]
    K = _values(S, 0, l)
    order = (step - w + 1 + torch.arange(w, device=K.device)) % w
    q = S.qwin[order].float().view(w, c["L"], c["B"], c["hkv"], -1, c["d"]).permute(1, 2, 3, 0, 4, 5)
    z = torch.matmul(q.reshape(*q.shape[:3], -1, c["d"]), K.transpose(-1, -2)) / math.sqrt(c["d"])
    z = z.view(*q.shape[:5], l)
    dead = torch.arange(l, device=K.device) > l - w + torch.arange(w, device=K.device).view(w, 1, 1)
    z = z.masked_fill(dead, float("-inf"))
    p = torch.exp(z - z.amax(dim=-1, keepdim=True))
    p = p / p.sum(dim=-1, keepdim=True)
    S.S[..., : l - w] = p[..., : l - w].amax(dim=4).mean(dim=3)
    return S.S


def _store(S):
    c = S.c
    n, t0 = c["rows"], c["rows"]
    P = S.prompt_len.long()
    row = torch.arange(n, device=P.device)
    t = (row + t0 - P.view(-1, 1)).clamp(max=n - 1)                       # [B, n]
    fits = (row < P.view(-1, 1)).view(1, -1, 1, n, 1)
    seq = torch.arange(c["B"], device=P.device).view(-1, 1)

    def rows_of(x):                                                       # [n, L, B, hkv, m] -> [L, B, hkv, n, m]
        return x[t, :, seq].permute(2, 0, 3, 1, 4)

    for which, cache, x in ((0, S.K8, S.k), (1, S.V8, S.v)):
        code, scale = _quantise(x.float())
        to = cache.view(torch.uint8)[..., :n, :]
        to.copy_(torch.where(fits, rows_of(code.view(torch.uint8)), to))
        to = S.scales[..., :n, which:which + 1]
        to.copy_(torch.where(fits, rows_of(scale).to(S.scales.dtype), to))
    to = S.pos[..., :n]
    to.copy_(torch.where(fits[..., 0], t.view(1, -1, 1, n).to(to.dtype), to))
    return {"K8": S.K8, "V8": S.V8, "scales": S.scales, "pos": S.pos}


def _read(S):
    n = max(S.lens)
    seen = (torch.arange(_cap(S.c), device=S.K8.device) < S.at.view(-1, 1)).view(1, S.c["B"], 1, -1, 1)
    T = S.T
    for which, to in ((0, S.K), (1, S.V)):
        rows = _values(S, which, n).to(to.dtype)
        old = _untile(to, T)[..., :n, :] if which == 0 else to[..., :n, :]
        rows = torch.where(seen[..., :n, :], rows, old)
        to[..., :n, :] = _tile(rows, T) if which == 0 else rows
    return {"K": S.K, "V": S.V}


def _compact(S):
    c = S.c
    l, b, w, T = c["rows"], c["b"], c["w"], S.T
    window = torch.arange(l - w, l, device=S.keep.device, dtype=S.keep.dtype).expand(*S.keep.shape[:-1], w)
    src = torch.cat([S.keep, window], dim=-1).long()
    at = src[..., None]
    d = c["d"]
    K = _untile(S.K8.view(torch.uint8)[..., : -(-l // 16) * 16, :], T)
    S.K8.view(torch.uint8)[..., :b, :] = _tile(K.gather(-2, at.expand(*src.shape, d)), T)
    V = S.V8.view(torch.uint8)
    V[..., :b, :] = V.gather(-2, at.expand(*src.shape, d))
    S.scales[..., :b, :] = S.scales.gather(-2, at.expand(*src.shape, 2))
    S.pos[..., :b] = S.pos.gather(-1, src)
    S.F_hist[..., : b - w] = S.F.gather(-1, S.keep.long())
    S.d_state.copy_(torch.tensor([b, S.step + 1, b - w, b // 16 * 16], dtype=torch.int32).expand(S.d_state.shape))


# ---- one pass -------------------------------------------------------------------------------
class _State:
    pass


def prepare(case, seed):
    c, x, S = case, _Inputs(case, seed), _State()
    L, B, hq, hkv, d, w = c["L"], c["B"], c["hq"], c["hkv"], c["d"], c["w"]
    kind, dt, dev, cap, n = c["kind"], _DT[c["dtype"]], x.dev, _cap(c), _filled(c)
    S.c, S.T, S.lens = c, _tiled(c), _lens(c)
    q8 = c["cache"] == "q8"
    S.pos = torch.full((L, B, hkv, cap), -1, dtype=torch.int32, device=dev)
    S.qwin = torch.zeros(w, L, B, hq, d, dtype=dt, device=dev)
    if q8:
        S.K8, S.V8 = (torch.zeros(L, B, hkv, cap, d, dtype=torch.uint8, device=dev).view(F8) for _ in range(2))
        S.scales = torch.ones(L, B, hkv, cap, 2, dtype=torch.bfloat16, device=dev)
    if not q8 or kind == "read":
        S.K, S.V = (torch.zeros(L, B, hkv, cap, d, dtype=dt, device=dev) for _ in range(2))
    S.at = torch.tensor(S.lens, device=dev)
    S.step = c["rows"] + 1024
    if kind == "store":
        _, S.k, S.v = x.tokens(n)
        S.prompt_len = S.at.int()
    else:
        for layer in range(L):
            k, v = x.cache(layer, n)
            if not q8:
                S.K[layer, :, :, :n], S.V[layer, :, :, :n] = _tile(k, S.T), v
                continue
            (kc, ks), (vc, vs) = _quantise(k.float()), _quantise(v.float())
            S.K8.view(torch.uint8)[layer, :, :, :n] = _tile(kc.view(torch.uint8), S.T)
            S.V8.view(torch.uint8)[layer, :, :, :n] = vc.view(torch.uint8)
            S.scales[layer, :, :, :n] = torch.cat([ks, vs], dim=-1).to(S.scales.dtype)
            del k, v, kc, vc
        S.pos[..., :n] = torch.arange(n, dtype=torch.int32, device=dev)
    S.n_hist = c["b"] - w if S.T else 0
    first = S.step - (n - (S.n_hist + w)) if S.T else S.step              # the step behind the last compression
    rec = [[r - (S.step - first) if S.T else r, first, S.n_hist, S.T] for r in ([n] * B if kind == "window" else S.lens)]
    S.d_state = torch.tensor(rec, dtype=torch.int32, device=dev).expand(L, B, 4).contiguous()
    if kind in ("attend", "shared"):
        q, k, v = x.tokens(1)
        S.q, S.k, S.v = q[0], k[0], v[0]
    if kind == "shared":
        pre = [x.prefix(layer) for layer in range(L)]
        S.Kp, S.Vp = torch.stack([a for a, _ in pre]), torch.stack([a for _, a in pre])
    if kind == "window":
        q, k, v = x.tokens(w)
        S.q, S.k, S.v = q.unbind(0), k.unbind(0), v.unbind(0)
    if kind == "score":
        q, _, _ = x.tokens(w)
        S.step -= 1                                                      # the latest decode step
        S.qwin[(S.step - w + 1 + torch.arange(w, device=dev)) % w] = q
    if kind in ("window", "score"):
        S.S = torch.zeros(L, B, hkv, cap, device=dev)
    if kind == "compact":
        S.step -= 1
        S.keep, S.F = x.keep(n - w, c["b"] - w), x.scores(cap)
        S.F_hist = torch.zeros(L, B, hkv, cap, device=dev)
    S.outs = torch.zeros(w if kind == "window" else 1, L, B, hq, d, dtype=dt, device=dev)
    S.out = S.outs.unbind(0)
    if own:
        from paper_2512_00504_amd import Context, make_config
        S.ctx = Context(make_config(L, B, hq, hkv, d, c["b"], w, c["s"], cap, c["dtype"]))
        S.workspace = torch.zeros(S.ctx.workspace_bytes(), dtype=torch.uint8, device=dev)
        S.ctx.workspace_init(S.workspace)
        if kind == "shared":
            S.part = torch.zeros(S.ctx.prefix_bytes(c["prefix"]), dtype=torch.uint8, device=dev)
    return S


def run(S):
    c, kind, w, n = S.c, S.c["kind"], S.c["w"], S.c["rows"]
    if kind == "store":
        if not own:
            return _store(S)
        S.ctx.q8_store_prompt(S.k, S.v, n, 0, n, S.prompt_len, S.K8, S.V8, S.scales, S.pos)
        return {"K8": S.K8, "V8": S.V8, "scales": S.scales, "pos": S.pos}
    if kind == "read":
        if not own:
            return _read(S)
        S.ctx.q8_read(S.K8, S.V8, S.scales, S.d_state, S.step, S.K, S.V)
        return {"K": S.K, "V": S.V}
    if kind == "attend":
        if own:
            S.ctx.q8_attend_decode(S.q, S.k, S.v, S.K8, S.V8, S.scales, S.pos, S.step, S.qwin, S.d_state, n, None,
                                   S.out[0], S.workspace)
            out = S.out[0]
        else:
            out = _attend(S, S.q, S.k, S.v, S.step, S.at, max(S.lens) + 1)
        return {"out": out, "K8": S.K8, "V8": S.V8, "scales": S.scales, "pos": S.pos, "qwin": S.qwin}
    if kind == "window":
        if own:
            for i in range(w):
                S.ctx.q8_attend_decode(S.q[i], S.k[i], S.v[i], S.K8, S.V8, S.scales, S.pos, S.step + i, S.qwin, S.d_state,
                                       n - w + i, None, S.out[i], S.workspace)
            S.ctx.q8_score_window(S.qwin, S.K8, S.scales, S.d_state, S.step + w - 1, n, S.S, S.workspace)
            outs = S.outs
        else:
            outs = torch.stack([_attend(S, S.q[i], S.k[i], S.v[i], S.step + i, S.at - w + i, n - w + i + 1) for i in range(w)])
            _score(S, S.step + w - 1)
        return {"out": outs, "S": S.S, "K8": S.K8, "V8": S.V8, "scales": S.scales, "pos": S.pos}
    if kind == "score":
        if not own:
            return {"S": _score(S, S.step)}
        S.ctx.q8_score_window(S.qwin, S.K8, S.scales, S.d_state, S.step, n, S.S, S.workspace)
        return {"S": S.S}
    if kind == "compact":
        # the rows behind the budget are there again (the decode steps' part), and the next compression comes as
        # many steps later
        if own:
            S.ctx.q8_compact(S.keep, S.F, S.K8, S.V8, S.scales, S.F_hist, S.pos, S.d_state, S.step, S.workspace)
        else:
            _compact(S)
        S.step += n - c["b"]
        return {"K8": S.K8, "V8": S.V8, "scales": S.scales, "pos": S.pos, "F_hist": S.F_hist, "d_state": S.d_state}
    if own:
        S.ctx.prefix_attend(S.q, S.Kp, S.Vp, c["prefix"], c["prefix"], 0, c["B"], S.part)
        if c["cache"] == "q8":
            S.ctx.q8_attend_decode(S.q, S.k, S.v, S.K8, S.V8, S.scales, S.pos, S.step, S.qwin, S.d_state, n, S.part,
                                   S.out[0], S.workspace)
        else:
            S.ctx.attend_decode_prefix(S.q, S.k, S.v, S.K, S.V, S.pos, S.step, S.qwin, S.d_state, n, S.part, S.out[0],
                                       S.workspace)
        out = S.out[0]
    else:
        out = _shared(S)
    return {"out": out, "pos": S.pos, "qwin": S.qwin}


# ---- what a pass cannot do without ----------------------------------------------------------
def work(case):
    c = case
    e, d, g, w, b = (4 if c["dtype"] == "f32" else 2), c["d"], c["hq"] // c["hkv"], c["w"], c["b"]
    units, heads, l = c["L"] * c["B"] * c["hkv"], c["L"] * c["hkv"], c["rows"]
    all_rows = sum(_lens(c)) * heads
    row8 = 2 * d + 4                                         # K and V codes, both scales
    step = (2 * g + 2) * e * d + row8 + 4 + g * e * d        # q, out, new rows in; row and position out, q to the ring

    if c["kind"] == "store":
        return {"bytes": all_rows * (2 * e * d + row8 + 4), "flops": 0}
    if c["kind"] == "read":
        return {"bytes": all_rows * (row8 + 2 * e * d), "flops": 0}
    if c["kind"] == "attend":
        return {"bytes": all_rows * row8 + units * step, "flops": 4.0 * g * d * (all_rows + units)}
    score = (l * (d + 2) + g * w * e * d + 4 * (l - w), 2.0 * g * w * d * l)
    if c["kind"] == "window":
        rows = sum(range(l - w, l))
        return {"bytes": units * (rows * row8 + w * step + score[0]), "flops": units * (4.0 * g * d * (rows + w) + score[1])}
    if c["kind"] == "score":
        return {"bytes": units * score[0], "flops": units * score[1]}
    if c["kind"] == "compact":
        return {"bytes": units * (2 * (row8 + 4) * b + 3 * 4 * (b - w)), "flops": 0}
    P = c["prefix"]
    row = row8 if c["cache"] == "q8" else 2 * e * d
    return {"bytes": all_rows * row + units * step + heads * P * 2 * e * d,
            "flops": 4.0 * g * d * (all_rows + units) + 4.0 * units * g * d * P}


# ---- the same in 64 bits, from the definitions -------------------------------------------------
def _held(x):
    """What an 8-bit row holds of x: codes and scales, float64.  e4m3 numbers have steps of 2^(max(k, -6) - 3) in
    [2^k, 2^(k+1))."""
    x = x.double()
    top = x.abs().amax(dim=-1, keepdim=True)

    def two_to(e):                                                       # 2^e in float64, exactly
        return ((e.long() + 1023) << 52).view(torch.float64)

    e = torch.ceil(torch.log2(top / 448.0)).clamp(min=-500)
    e = torch.where(448.0 * two_to(e - 1) >= top, e - 1, e)              # log2 may be off by its rounding
    e = torch.where(448.0 * two_to(e) < top, e + 1, e)
    e = torch.where(top == 0, torch.zeros_like(e), e.clamp(min=-126))
    y = x / two_to(e)
    k = torch.frexp(y)[1] - 1
    step = two_to(k.clamp(min=-6) - 3)
    return torch.round(y / step) * step, two_to(e)


def _pad(x, n, dim, value=0.0):
    to = list(x.shape)
    to[dim] = n - x.shape[dim]
    return torch.cat([x, torch.full(to, value, dtype=x.dtype, device=x.device)], dim=dim)


def _in_tiles(x, T, E):
    x = x.clone()
    *lead, n, d = x.shape
    if T:
        x[..., :T, :] = x[..., :T, :].view(*lead, T // 16, 16, d // E, E).transpose(-3, -2).reshape(*lead, T, d)
    return x


def _softmax64(z):
    z = torch.exp(z - z.amax(dim=-1, keepdim=True))
    return z / z.sum(dim=-1, keepdim=True)


def exact(case, seed):
    c = case
    kind, L, B, hkv, d, w, n = c["kind"], c["L"], c["B"], c["hkv"], c["d"], c["w"], _filled(c)
    if kind == "compact":
        return None
    x, cap, T, lens = _Inputs(c, seed), _cap(c), _tiled(c), _lens(c)
    if kind == "store":
        _, k, v = x.tokens(n)
        codes, scales = [], []
        for y in (k, v):
            code, scale = _held(y)
            C = torch.zeros(L, B, hkv, cap, d, dtype=torch.float64, device=x.dev)
            s = torch.ones(L, B, hkv, cap, dtype=torch.float64, device=x.dev)
            for i, P in enumerate(lens):
                C[:, i, :, :P] = code[n - P:, :, i].permute(1, 2, 0, 3)
                s[:, i, :, :P] = scale[n - P:, :, i, :, 0].permute(1, 2, 0)
            codes.append(C)
            scales.append(s)
        return {"K8": codes[0], "V8": codes[1], "scales": torch.stack(scales, dim=-1), "pos": None}
    caches = [x.cache(layer, n) for layer in range(L)]
    if kind == "read":
        K, V = [], []
        E = 4 if c["dtype"] == "f32" else 8
        seen = (torch.arange(n, device=x.dev) < torch.tensor(lens, device=x.dev).view(-1, 1)).view(B, 1, n, 1)
        for k, v in caches:
            k, v = ((code * scale) * seen for code, scale in (_held(k), _held(v)))
            K.append(_pad(_in_tiles(k, T, E), cap, -2))
            V.append(_pad(v, cap, -2))
        return {"K": torch.stack(K), "V": torch.stack(V)}
    steps = w if kind in ("window", "score") else 1
    q, k, v = x.tokens(steps)
    prefix = [x.prefix(layer) for layer in range(L)] if kind == "shared" else None

    def held(y):
        if c["cache"] != "q8":
            return y.double()
        code, scale = _held(y)
        return code * scale

    outs, scores = [], []
    for layer in range(L):
        K, V = held(caches[layer][0]), held(caches[layer][1])
        caches[layer] = None
        if kind != "score":
            kn, vn = (held(y[:, layer].permute(1, 2, 0, 3)) for y in (k, v))
            K, V = _pad(K, n + steps, -2), _pad(V, n + steps, -2)
            at = torch.tensor([n] * B if kind == "window" else lens, device=x.dev).view(-1, 1, 1, 1) + torch.arange(steps, device=x.dev).view(1, 1, -1, 1)
            at = at.expand(B, hkv, steps, d)
            K.scatter_(-2, at, kn)
            V.scatter_(-2, at, vn)
            out = []
            for i in range(steps):
                m = n + steps if kind != "window" else n + i + 1
                z = torch.matmul(q[i, layer].double().view(B, hkv, -1, d), K[:, :, :m].transpose(-1, -2).contiguous()) / math.sqrt(d)
                if kind != "window":
                    z.masked_fill_(torch.arange(m, device=x.dev) > torch.tensor(lens, device=x.dev).view(-1, 1, 1, 1), float("-inf"))
                if kind == "shared":
                    Kp, Vp = (y.double() for y in prefix[layer])
                    zp = torch.matmul(q[i, layer].double().view(B, hkv, -1, d), Kp.transpose(-1, -2).contiguous()) / math.sqrt(d)
                    p = _softmax64(torch.cat([zp, z], dim=-1))
                    o = torch.matmul(p[..., : c["prefix"]], Vp) + torch.matmul(p[..., c["prefix"]:], V[:, :, :m])
                    del zp, p
                else:
                    o = torch.matmul(_softmax64(z), V[:, :, :m])
                out.append(o.view(B, -1, d))
            outs.append(torch.stack(out))
        if kind in ("window", "score"):
            l = c["rows"]
            total = torch.zeros(B, hkv, l - w, dtype=torch.float64, device=x.dev)
            for i in range(w):
                z = torch.matmul(q[i, layer].double().view(B, hkv, -1, d), K[:, :, : l - w + i + 1].transpose(-1, -2).contiguous()) / math.sqrt(d)
                total += _softmax64(z)[..., : l - w].amax(dim=2)
            scores.append(_pad(total / w, cap, -1))
    got = {}
    if outs:
        got["out"] = torch.stack(outs, dim=1)
        if kind != "window":
            got["out"] = got["out"][0]
    if scores:
        got["S"] = torch.stack(scores)
    return got

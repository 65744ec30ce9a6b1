"""Rotary positions and paged caches in 64 bits, from their definitions (torch, CPU)."""
import math

import torch

from q8_reference import joint

HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def angles(positions, freq):
    return positions.double().view(-1, 1, 1) * torch.as_tensor(freq, dtype=torch.float64)


def pairs(x, dim, layout):
    """The two channels of each pair, float64."""
    x = x.double()
    return (x[..., : dim // 2], x[..., dim // 2: dim]) if layout == "half" else (x[..., 0:dim:2], x[..., 1:dim:2])


def turned(x, positions, freq, layout, amplitude=1.0, transposed=False, dtype="bf16"):
    """x [L, n, h, d] and a bound of the error.  32 bits: a cosine or sine is off by 3.2 * 2^-24 (the reduced angle, at most pi/4, rounded:
    0.8; the polynomial's last sum 1 and the sums before it 0.3; the remainder 0.1; the amplitude's product 1), so a channel by
    3.2 (|u| + |v|) m, and by a product's rounding and the sum's, (|u| + |v|) m each: 6 in all.  The angle in 64 bits: its product is off by
    2^-53 of it here and there, the reduction by as much again.  Then the rounding to the type."""
    dim = 2 * len(freq)
    a = angles(positions, freq)
    u, v = pairs(x, dim, layout)
    c, s = torch.cos(a) * amplitude, torch.sin(a) * amplitude * (-1 if transposed else 1)
    y, tol = x.double().clone(), torch.zeros_like(x, dtype=torch.float64)
    size = (u.abs() + v.abs()) * abs(amplitude) * (6 * 2.0 ** -24 + 4 * 2.0 ** -53 * a.abs())
    for to, one, two in ((y, u * c - v * s, u * s + v * c), (tol, size, size)):
        if layout == "half":
            to[..., : dim // 2], to[..., dim // 2: dim] = one, two
        else:
            to[..., 0:dim:2], to[..., 1:dim:2] = one, two
    tol = tol + (tol > 0) * HALF_STEP[dtype] * (y.abs() + tol) + (tol > 0) * 2.0 ** -133
    return y, tol


def place(lens, starts, t):
    """Sequence and row of packed token t; lens with the new tokens.  None: of none."""
    for i in range(len(lens)):
        if starts[i] <= t < starts[i + 1]:
            row = lens[i] - (starts[i + 1] - t)
            return (i, row) if row >= 0 else None
    return None


def gathered(pool, table, n):
    """Rows 0 .. n-1 of one sequence and layer, [n, h_kv, d] float64, and which of them are there.  pool [n_pages, h_kv, page_rows, d]."""
    pages, _, rows, _ = pool.shape
    row = torch.arange(n)
    ids = table.long()[row // rows]
    ok = (ids >= 0) & (ids < pages)
    return pool[torch.where(ok, ids, torch.zeros_like(ids)), :, row % rows].double(), ok


def attended(q, K, V, table, lens, scale, dtype):
    """out [L, B, h_q, d] float64 and a bound: joint()'s, a weight's 2^-15 as the sum of two bf16 numbers (the upper half of its bits, and the
    rest of 2^-7 of it rounded to 2^-8), the result's half step."""
    L, B, hq, d = q.shape
    hkv = K.shape[2]
    g = hq // hkv
    out, tol = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    for l in range(L):
        for i in range(B):
            n = max(0, min(int(lens[i]), table.shape[1] * K.shape[3]))
            k, ok = gathered(K[l], table[i], n)
            v, _ = gathered(V[l], table[i], n)
            k, v = k[ok], v[ok]
            for j in range(hkv):
                heads = slice(j * g, (j + 1) * g)
                ref, t = joint(q[l, i, heads].double(), [(k[:, j], v[:, j])], scale)
                top = v[:, j].abs().max().item() if len(v) else 0.0
                out[l, i, heads] = ref
                tol[l, i, heads] = t + HALF_STEP[dtype] * ref.abs() + (2.0 ** -15 * top if dtype == "bf16" else 0.0)
    return out, tol


def scale_of(d):
    return 1 / math.sqrt(d)

"""The operators on caches in 8 bits and shared prefixes in 64 bits, from their definitions (torch, CPU)."""
import math

import torch

F8 = torch.float8_e4m3fn


def held(x):
    """codes and exponents [..., 1] of rows [..., d]: e = min{e >= -126: max|x| <= 448 2^e} over the finite entries, codes
    x 2^-e rounded to steps of 2^(max(k, -6) - 3) in [2^k, 2^(k+1)), ties to even; what is not finite is NaN."""
    x = x.double()
    finite = torch.isfinite(x)
    top = torch.where(finite, x.abs(), torch.zeros_like(x)).amax(dim=-1, keepdim=True)
    m, k = torch.frexp(top)                                        # top = m 2^k, m in [0.5, 1); 448 = 0.875 * 2^9
    e = k - 9 + (m > 0.875).int()
    e = torch.where(top == 0, torch.zeros_like(e), e.clamp(min=-126))
    y = torch.ldexp(x, -e.double())
    k = (torch.frexp(torch.where(finite, y, torch.ones_like(y)))[1] - 1).clamp(min=-6) - 3
    c = torch.ldexp(torch.round(torch.ldexp(y, -k.double())), k.double())
    return torch.where(finite, c, torch.full_like(c, float("nan"))), e


def values(x):
    c, e = held(x)
    return torch.ldexp(c, e.double())


def same(a, b):
    """Equal numbers, NaN where the other has NaN."""
    a, b = a.double(), b.double()
    return torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(torch.nan_to_num(a, nan=0.0), torch.nan_to_num(b, nan=0.0))


def joint(q, parts, scale):
    """softmax over all keys of `parts` together: q [g, d], parts [(K [n, d], V [n, d])], float64.  Returns out [g, d] and a bound of what
    32-bit arithmetic may differ by: a logit is a sum of d products (d + 4 roundings of 2^-24 of the sum of their magnitudes: products,
    sums, the scale, the row's scale), which moves each probability by that relative amount twice (it and the sum); n + 32 roundings of
    the sums of n weighted values (and their joining over pieces)."""
    K = torch.cat([k for k, _ in parts])
    V = torch.cat([v for _, v in parts])
    if not len(K):
        return torch.zeros(q.shape, dtype=torch.float64), 0.0
    z = q @ K.T * scale
    p = torch.exp(z - z.amax(dim=-1, keepdim=True))
    p = p / p.sum(dim=-1, keepdim=True)
    size = (q.abs() @ K.abs().T * scale).amax().item()
    eps = 2.0 ** -24
    return p @ V, (2 * (q.shape[1] + 4) * size + len(K) + 32) * eps * V.abs().amax().item()


def rounding(dtype, ref, top):
    """Of the result to its type; bf16: and of the probabilities to 8 bits, half a step each of the largest value (the kernels keep 8
    bits at least)."""
    return 2.0 ** -8 * ref.abs() + 2.0 ** -8 * top if dtype == "bf16" else 2.0 ** -24 * ref.abs()


def local_score(q, K, scale):
    """q [w, g, d] in the order of their steps, K [l, d]: S [l - w] of the candidates."""
    w, l = q.shape[0], K.shape[0]
    S = torch.zeros(l - w, dtype=torch.float64)
    for k in range(w):
        z = q[k] @ K[: l - w + k + 1].T * scale
        S += torch.softmax(z, dim=-1)[:, : l - w].amax(dim=0)
    return S / w


def logit_error(q, K, scale):
    """A bound of the relative error of a probability in 32 bits, see joint()."""
    return 2 * (q.shape[-1] + 4 + math.log2(len(K) + 1) + 8) * (q.abs() @ K.abs().T * scale).amax().item() * 2.0 ** -24 + len(K) * 2.0 ** -24

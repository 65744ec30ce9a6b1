"""Inputs whose result shows every edge row, and how far a kernel may be from 64 bits on them.

Queries are u + noise with u of +-1, ordinary keys and all values have unit variance, and a planted key is u * z / sqrt(d): its
logit is about z, chosen so that each planted row takes a like share of the weight.  A row that is lost, doubled or taken from another
place then moves the result by a tenth and more of its values, tens of times the bound below."""
import math

import torch

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def direction(gen, d):
    return (torch.randint(0, 2, (d,), generator=gen) * 2 - 1).double()


def queries(gen, u, dtype, *shape):
    return (u + 0.25 * torch.randn(*shape, len(u), generator=gen).double()).to(DT[dtype])


def rows(gen, dtype, *shape):
    return torch.randn(*shape, generator=gen).to(DT[dtype])


def height(keys):
    """The logit that gives a planted row about the weight of all `keys` ordinary ones: their logits have a variance of 1.06."""
    return math.log(keys + 1) + 0.53


def plant(K, u, at, z):
    """Row `at` (second to last dimension) of K gets a logit of about z."""
    K[..., at, :] = (u * z / math.sqrt(len(u))).to(K.dtype)


def weights(q, K, scale):
    return torch.softmax(q @ K.T * scale, dim=-1)


def bound(q, K, V, out, scale, dtype):
    """Per (head, channel), for q [g, d], K, V [n, d] and out [g, d] in 64 bits.
    Weights: a logit of n is a sum of d products (of 3 d where an operand enters as three bf16 numbers), each product and each partial sum
    and the scale rounded to 24 bits, so a weight is relatively off by (3 d + 8) 2^-24 sum_c |q_c k_c| scale, times 2 for the weights'
    sum it is divided by, and by 2^-22 for the exponential and the factors between pieces.
    bf16: weights enter the products with V rounded to 8 bits, off by 2^-8 each.
    Sums of n numbers: n + 64 roundings of 2^-24.  The result: half a step of its type, and once more its own error."""
    p = weights(q, K, scale)
    size = q.abs() @ K.abs().T * scale
    off = 2 * (3 * q.shape[1] + 8) * 2.0 ** -24 * size + 2.0 ** -22 + (len(K) + 64) * 2.0 ** -24
    if dtype == "bf16":
        off = off + 2.0 ** -8
    inner = (p * off) @ V.abs()
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    return inner * (1 + half) + half * out.abs() + 2.0 ** -126


def attend(q, K, V, scale):
    return weights(q, K, scale) @ V


def score(q, K, scale):
    """q [w, g, d] in the order of their steps, K [l, d]: S [l - w]."""
    w, l = q.shape[0], K.shape[0]
    S = torch.zeros(l - w, dtype=torch.float64)
    for k in range(w):
        S += torch.softmax(q[k] @ K[: l - w + k + 1].T * scale, dim=-1)[:, : l - w].amax(dim=0)
    return S / w


def score_bound(q, K, scale):
    """Relative, per candidate: a probability is off as in bound() by its own logit's error and the weighted mean of those in its sum (at most the
    largest that has weight)."""
    size = (q.abs().flatten(0, -2) @ K.abs().T * scale).amax(dim=0)
    p = torch.softmax(q.flatten(0, -2) @ K.T * scale, dim=-1).amax(dim=0)
    return (3 * q.shape[-1] + 8) * 2.0 ** -24 * (size[: len(K) - len(q)] + size[p > 2.0 ** -30].max()) + 2.0 ** -21 + (len(K) + 64) * 2.0 ** -24

"""The bounds of planted.py refuse results that lack a row or have other logits, and hold for what rounds as the kernels may."""
import math

import pytest
import torch

from planted import DT, attend, bound, direction, height, plant, queries, rows, score, score_bound
from q8_reference import values


def _inputs(dtype, d, own, prefix, seed):
    """Keys and values of own rows (the new one last) and of a prefix, planted at their ends."""
    gen = torch.Generator().manual_seed(seed)
    u = direction(gen, d)
    q = queries(gen, u, dtype, 7)
    K, V = rows(gen, dtype, own + prefix, d), rows(gen, dtype, own + prefix, d)
    at = sorted({0, own - 2, own - 1, own, own + prefix - 1} & set(range(own + prefix)))
    for n in at:
        plant(K, u, n, height(own + prefix))
    return q.double(), K, V, at


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("held", [False, True])
@pytest.mark.parametrize("d,own,prefix", [(128, 40, 700), (64, 300, 31), (64, 20, 5000), (128, 3000, 0), (64, 2, 1)])
def test_lost_rows_and_other_logits_are_refused(dtype, held, d, own, prefix):
    scale = 1 / math.sqrt(d)
    for seed in range(3):
        q, K, V, at = _inputs(dtype, d, own, prefix, seed)
        k, v = (values(K), values(V)) if held else (K.double(), V.double())
        ref = attend(q, k, v, scale)
        tol = bound(q, k, v, ref, scale, dtype)
        assert (tol < 0.05).all()
        passes = lambda x: bool(((x - ref).abs() <= tol).all())
        everything = torch.arange(own + prefix)
        for n in at:
            keep = everything != n
            assert not passes(attend(q, k[keep], v[keep], scale)), n
            twice = torch.cat([everything, torch.tensor([n])])
            assert not passes(attend(q, k[twice], v[twice], scale)), n
        if prefix:
            assert not passes(attend(q, k[:own], v[:own], scale)) and not passes(attend(q, k[own:], v[own:], scale))
        if own + prefix > len(at):                             # (planted rows alone have one logit)
            assert not passes(attend(q, k, v, scale * 1.01))
        if held:
            assert not passes(attend(q, K.double(), V.double(), scale))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,own,prefix", [(128, 40, 700), (64, 20, 5000)])
def test_arithmetic_of_the_type_passes(dtype, d, own, prefix):
    # logits and sums in 32 bits, bf16: weights rounded to it, in pieces of 64 keys with a maximum each; the result rounded
    scale = 1 / math.sqrt(d)
    q, K, V, _ = _inputs(dtype, d, own, prefix, 5)
    ref = attend(q, K.double(), V.double(), scale)
    z = (q.float() @ K.float().T) * scale
    out, l, m = torch.zeros(7, d), torch.zeros(7, 1), z.amax(dim=-1, keepdim=True)
    for n in range(0, len(K), 64):
        zz = z[:, n:n + 64]
        top = zz.amax(dim=-1, keepdim=True)
        p = torch.exp(zz - top)
        f = torch.exp(top - m)
        out += f * (p.to(DT[dtype]).float() @ V[n:n + 64].float())
        l += f * p.sum(dim=-1, keepdim=True)
    got = (out / l).to(DT[dtype]).double()
    assert ((got - ref).abs() <= bound(q, K.double(), V.double(), ref, scale, dtype)).all()


@pytest.mark.parametrize("d,g,w,l", [(64, 3, 8, 300), (128, 7, 16, 1100)])
def test_scores_of_other_rows_are_refused(d, g, w, l):
    gen = torch.Generator().manual_seed(d)
    u = direction(gen, d)
    q, K = queries(gen, u, "bf16", w, g).double(), rows(gen, "bf16", l, d)
    at = [0, l - w - 1, l - w, l - 1]
    for n in at:
        plant(K, u, n, height(l))
    K = values(K)
    ref, tol = score(q, K, d ** -0.5), score_bound(q, K, d ** -0.5)
    assert (tol < 1e-2).all()
    passes = lambda x: bool(((x - ref).abs() <= tol * ref).all())
    for n in at:
        other = K.clone()
        other[n] = 0
        assert not passes(score(q, other, d ** -0.5)), n
    assert not passes(score(q, K, d ** -0.5 * 1.01)) and not passes(score(q[:, 1:], K, d ** -0.5))

"""What the checks of the attention's precision let through: weights of 24 digits; and what they do not: fewer."""
import math

import pytest
import torch

from precision_ref import Rms, cancelling, cancelling_bound, pieces, plain, rms_parts

FEWER = {"one piece": pieces(1), "float16": lambda p: p.half().float()}
DTYPES = [torch.bfloat16, torch.float32]


def _heavy(group, d, n, seed, dtype):
    gen = torch.Generator().manual_seed(seed)
    u = torch.randn(1, d, generator=gen)
    u /= u.norm()
    k = torch.randn(n, d, generator=gen) + 0.25 * math.sqrt(d) * -torch.rand(n, 1, generator=gen).log() * u
    return (torch.randn(group, d, generator=gen) + 4.0 * u).to(dtype), k.to(dtype), torch.randn(n, d, generator=gen).to(dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [(4, 64, 33), (4, 128, 200), (8, 64, 700), (16, 128, 3000)])
def test_rms_check(shape, dtype):
    g, d, n = shape
    q, k, v = _heavy(g, d, n, n, dtype)
    live = torch.rand(n, generator=torch.Generator().manual_seed(1)) < 0.8
    parts = rms_parts(q, k, v, live, d ** -0.5)

    def ratio(weights):
        r = Rms(dtype)
        r.add(plain(q, k, v, live, d ** -0.5, dtype, weights), *parts)
        return r.ratio()
    assert ratio(lambda p: p) < 1.5 and ratio(pieces(3)) < 1.5
    for name, weights in FEWER.items():
        assert ratio(weights) > 10, name


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("group,d", [(16, 64), (20, 128)])
def test_cancelling_values(group, d, dtype):
    def worst(weights):
        most = 0.0
        for seed in range(4):
            q, k, v, scale = cancelling(group, d, seed, dtype)
            ref, bound = cancelling_bound(q, dtype)
            out = plain(q, k, v, torch.ones(3, dtype=torch.bool), scale, dtype, weights).double()
            most = max(most, float(((out.diagonal() - ref).abs() / bound).max()))
        return most
    assert worst(lambda p: p) < 1 and worst(pieces(3)) < 1
    for name, weights in {"two pieces": pieces(2), **FEWER}.items():
        assert worst(weights) > 1.5, name


def test_three_pieces_are_a_float32():
    p = torch.rand(100000, generator=torch.Generator().manual_seed(2)) ** 4
    assert torch.equal(pieces(3)(p), p)

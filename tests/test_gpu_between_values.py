"""Joins, the recurrence and log probabilities with values that are no ordinary ones: logits far from zero, scales that leave little of a row, infinities and NaN in one of several sequences.
Bounds are those of between_ref.py, which hold for any finite logits."""
import math

import pytest

from test_gpu_between import DTYPES, env, gen_of, logp_case  # noqa: F401

pytestmark = pytest.mark.gpu
ROWS = [(4, 1000, 0), (3, 5000, 20), (300, 700, 5), (2, 40000, 0), (5, 33001, 3)]              # rows by one block and by several, with and without alternatives


def step(dtype, at):
    """the distance of numbers of the type at this one"""
    return 2.0 ** (math.floor(math.log2(abs(at))) - (23 if dtype == "f32" else 7))


# ---- log probabilities ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("at", [1e5, -1e5, 2.3e6, -2.3e6, 1e7, -1e7, 3e7, -1e9, 1e9, -1e20, 1e30])
@pytest.mark.parametrize("rows,vocab,k", ROWS)
def test_logp_far_from_zero(env, dtype, at, rows, vocab, k):
    """all the same, spread over thirty of the type's steps, and half of a row there (an ordinary mask where it is negative)"""
    torch = env[0]
    g, d = gen_of(torch, rows, vocab, at), step(dtype, at)
    z = at + d * torch.randint(0, 30, (rows, vocab), generator=g, device="cuda").double()
    z[0] = at
    z[1, ::2] = torch.randn(z[1, ::2].shape, generator=g, device="cuda").double()
    for scale in (1.0, 0.5 / d):                                    # powers of two
        logp_case(env, dtype, rows, vocab, k, scale=scale, logits=z)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("scale", [1e3, 1e4, 1e5, 1e6, 1e7, 1e8])
@pytest.mark.parametrize("rows,vocab,k", ROWS)
def test_logp_of_ordinary_logits_with_a_large_scale(env, dtype, scale, rows, vocab, k):
    """sampling at a temperature next to nothing"""
    logp_case(env, dtype, rows, vocab, k, scale=scale)
    g = gen_of(env[0], rows, vocab, scale)
    z = 4 + env[0].randint(0, 40, (rows, vocab), generator=g, device="cuda").double() * step(dtype, 4.0)           # neighbours, so that more than one counts
    logp_case(env, dtype, rows, vocab, k, scale=scale, logits=z)

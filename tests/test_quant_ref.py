"""The definitions that the tests of the 8-bit cache and of the verification compare with:
e4m3 and its scales against torch's own type, and that what a verified sequence receives
is distributed as the target's samples."""

import itertools
import math

import pytest
import torch

from quant_ref import Verified, codes_of, e4m3_values, nearest_code, quantize, scale_exponent


def test_values_are_those_of_the_type():
    v = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    assert torch.equal(v, e4m3_values())
    assert torch.isnan(torch.tensor([127], dtype=torch.uint8).view(torch.float8_e4m3fn).float()).all()


def test_rounding():
    v = e4m3_values()
    mid = (v[1:] + v[:-1]) / 2
    x = torch.cat([v, mid, mid * (1 + 2.0 ** -20), mid * (1 - 2.0 ** -20)])
    x = torch.cat([x, -x])
    assert torch.equal(nearest_code(x), x.float().to(torch.float8_e4m3fn).double())


@pytest.mark.parametrize("most,e", [(448.0, 0), (449.0, 1), (0.0, -100), (1.0, -8), (1.75, -8), (1.7578125, -7),
                                    (3.3e38, 119), (1e-40, -100)])
def test_scales(most, e):
    assert scale_exponent(most) == e


def test_error_of_a_value():
    """At most half a step: 2^-4 of the value, or 2^-10 of the scale."""
    x = torch.randn((64, 32), generator=torch.Generator().manual_seed(1)).double() * 3
    x[5, 3], x[40, 1] = math.inf, math.nan
    codes, es = quantize(x, torch.ones(64, dtype=torch.bool), 32)
    for i, e in enumerate(es):
        a, c = x[32 * i:32 * i + 32], codes[32 * i:32 * i + 32]
        ok = torch.isfinite(a)
        assert torch.equal(torch.isnan(c), ~ok)
        gap = (a - c * 2.0 ** e).abs()[ok]
        assert bool((gap <= torch.maximum(a[ok].abs() * 2.0 ** -4, torch.tensor(2.0 ** (e - 10)))).all())
    assert torch.equal(codes_of(codes[:32] * 4.0, 2)[torch.isfinite(codes[:32])], codes[:32][torch.isfinite(codes[:32])])


@pytest.mark.parametrize("drafted", [False, True])
@pytest.mark.parametrize("parents,tokens", [([-1, 0, 0], [0, 2, 1]), ([-1, 0, 0], [0, 1, 1]), ([-1, 0, 1], [0, 3, 0]),
                                            ([-1, 0, 0, 0], [0, 2, 1, 2])])
def test_received_tokens_are_the_targets(drafted, parents, tokens):
    """The first token that a sequence receives (an accepted child of row 0, or the draw) has
    the probabilities p, whatever was drafted: summed over a fine grid of the numbers, and
    over the tokens that the draft draws. A test is decided by its number's interval, so a
    grid of n points a number is off by at most 1 / n for each."""
    n, V, S = 48, 4, len(parents)
    gen = torch.Generator().manual_seed(4)
    logits = torch.randn((S, V), generator=gen)
    q = torch.softmax(torch.randn((S, V), generator=gen), -1)
    p = torch.softmax(logits[0].double(), -1)
    kids = [r for r in range(S) if parents[r] == 0]
    grid = [(i + 0.5) / n for i in range(n)]
    if len(kids) == 3:
        grid = grid[::4]
    got = torch.zeros(V, dtype=torch.float64)
    draws = itertools.product(range(V), repeat=len(kids)) if drafted else [tuple(tokens[r] for r in kids)]
    for xs in draws:
        chance = math.prod(float(q[0, x]) for x in xs) if drafted else 1.0
        t = list(tokens)
        for r, x in zip(kids, xs):
            t[r] = x
        # a child's token first, where one is accepted; else the draw's distribution
        for us in itertools.product(grid, repeat=len(kids)):
            u = [0.5] * S
            for r, x in zip(kids, us):
                u[r] = x
            s = Verified.__new__(Verified)
            s.z, s.V, s.parents, s.tokens, s.u, s.T = logits.double(), V, parents, t, u, 1.0
            s.draft = q.double() if drafted else None
            w, took = s.test(0, p)
            if took is not None:
                got[t[took]] += chance / len(grid) ** len(kids)
            else:
                got += chance / len(grid) ** len(kids) * w / w.sum()
    assert float((got - p).abs().max()) <= len(kids) / len(grid)
    assert abs(float(got.sum()) - 1) < 1e-5


def test_walk():
    z = torch.full((4, 5), -5.0)
    z[0, 1] = z[1, 2] = z[2, 2] = z[3, 4] = 8.0
    s = Verified(z, [0, 3, 1, 2], [0.5] * 4, parents=[-1, 0, 0, 2])
    assert s.path == [0, 2, 3] and s.next == 4 and not s.flag
    assert Verified(z, [0, 1, 2, 2], None, temperature=0).path == [0, 1, 2, 3]
    s = Verified(z, [0, 1, 3, 2], None, temperature=0)
    assert s.path == [0, 1] and s.next == 2
    z[1, 0] = math.nan
    s = Verified(z, [0, 1, 3, 2], [0.5] * 4)
    assert s.path == [0, 1] and s.next == -1 and s.flag

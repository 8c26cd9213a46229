"""How far a value of the 8-bit cache may be from what was written, in float64 on the CPU from the
definitions in quant_ref.py: one rounding, magnitudes past the largest scale's, and codes rounded
again each time their block's scale is raised."""

import math

import torch

from quant_ref import MOST, codes_of, e4m3_values, nearest_code, scale_exponent


def test_one_rounding():
    """Every exponent of the largest magnitude of a block, and values down from it."""
    gen = torch.Generator().manual_seed(1)
    for top in list(range(-126, 127, 7)) + [126]:
        x = (1.0 + torch.rand(400, generator=gen, dtype=torch.float64)) * \
            2.0 ** (top - 30 * torch.rand(400, generator=gen, dtype=torch.float64)).floor()
        x[0] = 2.0 ** (top + 1)
        e = scale_exponent(float(x.max()))
        assert float(x.max()) <= 448.0 * 2.0 ** e
        err = (codes_of(x, e) * 2.0 ** e - x).abs()
        assert bool((err <= torch.maximum(x / 16, torch.full_like(x, 2.0 ** (e - 10)))).all())


def test_past_the_largest_scale():
    largest = float(torch.finfo(torch.float32).max)
    x = torch.linspace(448.0 * 2.0 ** MOST, largest, 1000, dtype=torch.float64)
    assert scale_exponent(largest) == MOST
    got = codes_of(x, MOST) * 2.0 ** MOST
    assert bool((got == 448.0 * 2.0 ** MOST).all())
    worst = float(((x - got) / x).max())
    assert 0.124 < worst <= 0.125


def test_raised_scales():
    """Values of a block whose scale is 1 at first, under every run of rises by 2^1 to 2^3 up to
    2^12 in all, and by single larger ones: the roundings add up to less than 2^-9 of the scale
    beside the first, and to more than the 2^-10 of one."""
    v = e4m3_values()
    x = torch.cat([v, (v[1:] + v[:-1]) / 2, v[:-1] * 0.49 + v[1:] * 0.51])
    first = nearest_code(x)
    beyond = 0

    def go(code, scale, left):
        nonlocal beyond
        off = (code * scale - x).abs()
        assert bool((off <= x / 16 + 2.0 ** -9 * scale).all())
        beyond += int((off > torch.maximum(x / 16, torch.full_like(x, 2.0 ** -10 * scale))).sum())
        for step in (1, 2, 3):
            if step <= left:
                go(nearest_code(code * 2.0 ** -step), scale * 2.0 ** step, left - step)

    go(first, 1.0, 12)
    for step in (4, 9, 17, 18, 40, 219):
        off = (nearest_code(first * 2.0 ** -step) * 2.0 ** step - x).abs()
        assert bool((off <= x / 16 + math.ldexp(1.0, step - 9)).all())
    assert beyond > 0

"""The attention over a cache and the accumulated weights in float64, from the
formulas, and the error a kernel of fp32 logits may make on them.

Errors (u = 2^-24, half a step of fp32, relative):
  logit       |z - z*| <= (d + 3) u scale sum_c |q_c k_c| =: e, over the largest sum of
              any visible pair (d products and additions; the scale and its
              base-2 form rounded)
  exponent    its argument is rounded at the magnitude of the larger of |z| and |lse|,
              in powers of two: 4 u (|z| + |lse|) log2 e
  lse         e, the same rounding, and the sum over n terms in fp32, taken as the
              kernels take it: at most n u relative (n the row's tokens; far less by chunks)
  weight      exp of both errors: relative 2 (e + exponent) + n u + 4 u =: p
  acc         p and the sum over rows: (p + R u) sum_r rw p
  out         (p + h) sum_i p_i |v_i| + h |out|, h half a step of the type (the weights
              are rounded to it for bf16; fp32: the products' sum, n u)
"""

import math

import torch

U = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def sees_tree(tree, S, b):
    """bool [S][S] from int64 masks [B][S][words], or the chain where null."""
    j = torch.arange(S)
    if tree is None:
        return j[None, :] <= j[:, None]
    return (tree[b].cpu()[:, j // 64] >> (j % 64) & 1) == 1


def softmax_rows(z):
    """(weights, lse) of rows of logits in float64; a row of -inf: zeros, -inf."""
    lse = torch.logsumexp(z, -1)
    p = torch.where((lse > -math.inf)[..., None], torch.exp(z - lse[..., None]), torch.zeros_like(z))
    # a NaN row stays NaN
    return torch.where(torch.isnan(lse)[..., None], torch.full_like(z, math.nan), p), lse


class Weights:
    """float64 results and bounds of one unit: rows R = G S against n tokens."""

    def __init__(self, q, k, scale, visible):
        q, k = q.double(), k.double()
        self.z = (q @ k.t().contiguous()) * scale
        self.z[~visible] = -math.inf
        size = (q.abs() @ k.abs().t().contiguous()) * scale
        size[~visible] = 0.0
        size = torch.nan_to_num(size, nan=0.0, posinf=0.0)
        d, n = q.shape[1], k.shape[0]
        self.e = (d + 3) * U * (float(size.max()) if size.numel() else 0.0)
        self.n = n
        self.p, self.lse = softmax_rows(self.z)
        finite = self.lse[torch.isfinite(self.lse)]
        top = float(finite.abs().max()) if finite.numel() else 0.0
        zf = self.z[torch.isfinite(self.z)]
        top += float(zf.abs().max()) if zf.numel() else 0.0
        self.expo = 4 * U * top * 1.4427
        self.lse_tol = self.e + 2 * self.expo + (n + 4) * U
        self.rel = 2 * (self.e + self.expo) + (n + 8) * U


def check(got, want, tol, what):
    """|got - want| <= tol elementwise; infinities and NaN alike."""
    got = got.double()
    want = want.double()
    special = ~torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN elsewhere"
    assert torch.equal(got[special & ~torch.isnan(want)], want[special & ~torch.isnan(want)]), what
    tol = tol.expand_as(want) if torch.is_tensor(tol) else torch.full_like(want, tol)
    gap = ((got - want).abs() - tol)[~special]
    assert gap.numel() == 0 or float(gap.max()) <= 0, \
        f"{what}: over its bound by {float(gap.max()):.3e} (bound there {float(tol[~special].max()):.3e})"

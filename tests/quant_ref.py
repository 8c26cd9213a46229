"""The 8-bit cache and the verification of drafted tokens in float64, from their
definitions, without the library."""

import math

import torch

LEAST, MOST = -100, 119   # exponents of a scale


def e4m3_values():
    """The finite non-negative values: 2^-9 times 0 .. 7, then 1 + i / 8 times 2^-6 .. 2^8
    less the last (NaN's place)."""
    small = [i * 2.0 ** -9 for i in range(8)]
    return torch.tensor(small + [(1 + i / 8) * 2.0 ** e for e in range(-6, 9) for i in range(8)][:-1],
                        dtype=torch.float64)


def nearest_code(x):
    """x float64 (finite, |x| <= 448) rounded to the nearest value, ties to the even code."""
    v = e4m3_values().to(x.device)
    a = x.abs()
    hi = torch.searchsorted(v, a).clamp(max=len(v) - 1)
    lo = (hi - 1).clamp(min=0)
    up, down = v[hi] - a, a - v[lo]
    take = torch.where(up == down, hi % 2 == 0, up < down)
    return torch.copysign(torch.where(take, v[hi], v[lo]), x)


def scale_exponent(most):
    """The least e in LEAST .. MOST with most <= 448 2^e (python floats are exact here)."""
    e = LEAST
    while e < MOST and most > 448.0 * 2.0 ** e:
        e += 1
    return e


def codes_of(x, e):
    """Codes (as values) of x (float64) in units of 2^e; NaN where x is not finite."""
    y = nearest_code((torch.nan_to_num(x, nan=0.0, posinf=0.0, neginf=0.0) * 2.0 ** -e).clamp(-448.0, 448.0))
    return torch.where(torch.isfinite(x), y, torch.full_like(y, math.nan))


def block_exponents(x, tokens, block):
    """Exponents [T / block] of x [T][d] (float64) whose tokens are the rows of `tokens`."""
    size = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x)).amax(-1)
    size = torch.where(tokens, size, torch.zeros_like(size)).view(-1, block).amax(-1)
    return [scale_exponent(m) for m in size.tolist()]


def quantize(x, tokens, block):
    """(codes as values [T][d], exponents) of one unit's K or V."""
    es = block_exponents(x, tokens, block)
    return torch.cat([codes_of(x[i * block:(i + 1) * block], e) for i, e in enumerate(es)]), es


class Verified:
    """One sequence: rows of logits [S][V], tokens, uniform numbers, parents, draft rows."""

    def __init__(self, logits, tokens, uniform, parents=None, draft=None, temperature=1.0):
        S, V = logits.shape
        z = logits.double().cpu()
        self.z, self.V = z, V
        self.parents = list(parents) if parents is not None else [r - 1 for r in range(S)]
        self.tokens = [int(t) for t in tokens]
        self.u = [float(x) for x in uniform] if uniform is not None else [0.0] * S
        self.draft = None if draft is None else draft.double().cpu()
        self.T = temperature
        self.path, self.flag = [0], False
        self.walk()

    def children(self, node):
        return [r for r in range(node + 1, len(self.tokens))
                if self.parents[r] == node and 0 <= self.tokens[r] < self.V]

    def walk(self):
        node = 0
        while True:
            z = self.z[node]
            if self.T == 0:
                ok = torch.where(torch.isnan(z), torch.full_like(z, -math.inf), z)
                if not bool((ok > -math.inf).any()):
                    self.next, self.flag = -1, True
                    return
                best = int((ok == ok.max()).nonzero()[0, 0])
                took = next((r for r in self.children(node) if self.tokens[r] == best), None)
            else:
                if bool(torch.isnan(z).any()) or not math.isfinite(float(z.max())):
                    self.next, self.flag = -1, True
                    return
                p = torch.softmax(z / self.T, 0)
                w, took = self.test(node, p)
            if took is None:
                break
            node = took
            self.path.append(node)
        if self.T == 0:
            self.next = best
            return
        if bool(torch.isnan(w).any()):
            self.next, self.flag = -1, True
            return
        if float(w.sum()) == 0.0:
            w = p
        mass = torch.cumsum(w, 0)
        over = (mass > self.u[0] * mass[-1]).nonzero()
        self.next = int(over[0, 0]) if len(over) else int((w > 0).nonzero()[-1, 0])

    def test(self, node, p):
        w = p.clone()
        for r in self.children(node):
            x = self.tokens[r]
            if self.draft is None:
                if self.u[r] * float(w.sum()) < float(w[x]):
                    return w, r
                w[x] = 0.0
            else:
                q = self.draft[node]
                left = float(w.sum())
                if self.u[r] * float(q[x]) * left < float(w[x]):
                    return w, r
                w = w - left * q          # (p - C q)+ once more less N q, as C grows by N
                w = torch.where(w < 0, torch.zeros_like(w), w)
        return w, None

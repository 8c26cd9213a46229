"""jacap_quantize, jacap_append_quant, jacap_attend_quant and jacap_attn_weights_quant
against their definitions in float64 (quant_ref.py, attention_ref.py).

Codes and scales are exact. Attention over the cache is attention over codes times
scales, which are exact in bf16 and fp32, so its bounds are attention_ref.py's. For fp32
rows each logit is three sums of d products (the terms of q, the smaller two together
below 2^-7 of the largest: (d + 1) (1 + 2^-7) additions' roundings, within the d + 3 there) and
the output's sum has three products a token in place of one: 3 (n + S) u."""

import math

import pytest
import torch

import test_gpu_attention
from attention_ref import U, Weights, check, half_step, sees_tree
from quant_ref import codes_of, quantize, scale_exponent
from test_gpu_attention import BF, F32, Case

pytestmark = pytest.mark.gpu
E4 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def jacap():
    from paper_2609_08131_amd import jacap as j
    return j


def up_to(n, block):
    return max(1, -(-n // block)) * block


class QuantCase(Case):
    """A Case whose cache is held in 8 bits; k and v are its values. Rows without tokens
    hold NaN codes. Scales are of each block's tokens, times 2^spread of its number."""

    def __init__(self, jacap, lens, S, dtype=BF, d=128, block=32, spare=0, token_major=False, **kw):
        rows = [up_to(n + spare, block) for n in lens]
        super().__init__(rows, S, dtype, d, token_major=token_major, **kw)
        self.lens, self.rows, self.block = lens, rows, block
        self.live = torch.tensor(lens, dtype=torch.int32, device="cuda")
        L, H, T, _ = self.k.shape
        shape = (L, T, H, d) if token_major else (L, H, T, d)
        made = []
        self.scales = torch.empty((L, H, T // block, 2), device="cuda")
        for i, name in enumerate(("k", "v")):
            x = getattr(self, name).float()
            e = torch.randint(-9, -5, (L, H, T // block), device="cuda").float()
            self.scales[..., i] = 2.0 ** e
            fine = self.scales[..., i].repeat_interleave(block, 2)[..., None]
            codes = (x / fine).clamp(-448, 448).to(E4)
            for b, n in enumerate(lens):
                codes.view(torch.uint8)[:, :, self.starts[b] + n:self.starts[b + 1]] = 0x7F
            held = torch.empty(shape, dtype=E4, device="cuda")
            held = held.transpose(1, 2) if token_major else held
            held.copy_(codes)
            made.append(held)
            setattr(self, name, (codes.float() * fine).to(dtype))
            assert dtype == F32 or torch.equal(torch.nan_to_num((codes.float() * fine)),
                                               torch.nan_to_num(getattr(self, name).float()))
        self.cache = jacap.QuantCache(made[0], made[1], self.scales, block)


def run_attend(jacap, c, use_acc, accumulate, decay=1.0, row_weight=None):
    p = jacap.AttentionParams(accumulate=accumulate, decay=decay, live_lens=c.live, tree=c.tree,
                              row_weight=row_weight)
    prob = jacap.prepare_attend_quant(c.q, c.cache, c.kd, c.vd, c.offsets, c.rows, p)
    acc = c.acc.clone() if use_acc or accumulate else None
    prob.out.fill_(7.0)
    prob.lse.fill_(7.0)
    jacap.run_attend_quant(prob, c.q, c.cache, c.kd, c.vd, acc=acc)
    assert jacap.read_status(prob.ws) == 0
    return prob, acc


def check_attend(c, prob, acc, use_acc, accumulate, decay=1.0, row_weight=None):
    S, G = c.S, c.G
    h_ = half_step(c.q.dtype)
    for b, n in enumerate(c.lens):
        sees = sees_tree(c.tree, S, b).cuda().repeat(G, 1)
        rw = torch.ones(G * S, dtype=torch.float64, device="cuda")
        if row_weight is not None:
            rw = row_weight[b].double().repeat(G)
        for l in range(c.L):
            for h in range(c.H):
                q, sl = c.unit(b, l, h)
                vis = torch.ones((G * S, n + S), dtype=torch.bool, device="cuda")
                vis[:, n:] = sees
                hidden = c.acc[l, h, sl] < 0
                if use_acc or accumulate:
                    vis[:, :n] &= ~hidden
                w = Weights(q, torch.cat([c.k[l, h, sl], c.kd[b, l, h]]), c.scale, vis)
                v = torch.cat([c.v[l, h, sl], c.vd[b, l, h]]).double()
                v = torch.where(vis.any(0)[:, None], v, torch.zeros_like(v))
                tag = f"b{b} l{l} h{h} n{n}"
                out = w.p @ v
                got = prob.out[b, l, h * G:(h + 1) * G].reshape(G * S, -1)
                extra = h_ if c.q.dtype == BF else 3 * (n + S) * U
                check(got, out, (w.rel + extra) * (w.p @ v.abs()) + h_ * out.abs() + 1e-30, f"out {tag}")
                check(prob.lse[b, l, h * G:(h + 1) * G].reshape(-1), w.lse, w.lse_tol, f"lse {tag}")
                if not accumulate:
                    continue
                given = (rw[:, None] * w.p).sum(0)
                tol = (w.rel + (G * S + 4) * U) * (rw.abs()[:, None] * w.p).sum(0) + 1e-30
                check(prob.acc_draft[b, l, h], given[n:], tol[n:], f"acc_draft {tag}")
                old = c.acc[l, h, sl].double()
                want = torch.where(hidden, old, decay * old + given[:n])
                check(acc[l, h, sl], want, tol[:n] + 4 * U * want.abs(), f"acc {tag}")
    if acc is not None:
        for b, n in enumerate(c.lens):
            a, e = c.starts[b] + n, c.starts[b + 1]
            assert torch.equal(acc[:, :, a:e], c.acc[:, :, a:e])


# ---------------------------------------------------------------------------
# Writing
# ---------------------------------------------------------------------------
def wide_case(dtype, d, block, lens, spare=0, token_major=False, L=2, H=2, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows = [up_to(n + spare, block) for n in lens]
    starts = [sum(rows[:b]) for b in range(len(lens) + 1)]
    T = starts[-1]

    def make():
        # magnitudes of many decades, rounding ties, zeros
        x = torch.randn((L, H, T, d), generator=gen, device="cuda")
        x = x * 2.0 ** torch.randint(-12, 4, (L, H, T, 1), generator=gen, device="cuda").float()
        tie = torch.randint(-64, 64, (L, H, T, d), generator=gen, device="cuda").float() / 32
        x = torch.where(torch.rand((L, H, T, d), generator=gen, device="cuda") < 0.3, tie, x)
        x[:, :, ::7] = 0.0
        x = x.to(dtype)
        return x.transpose(1, 2).contiguous().transpose(1, 2) if token_major else x
    return rows, starts, make(), make()


def empty_cache(jacap, L, H, T, d, block, token_major, fill=0x2A):
    shape = (L, T, H, d) if token_major else (L, H, T, d)
    k, v = (torch.full(shape, fill, dtype=torch.uint8, device="cuda").view(E4) for _ in range(2))
    if token_major:
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    return jacap.QuantCache(k, v, torch.full((L, H, T // block, 2), -7.0, device="cuda"), block)


def check_quantized(cache, x2, starts, lens, block, tokens=None, fill=0x2A):
    L, H, T, d = cache.k.shape
    for i, (codes, x) in enumerate(zip((cache.k, cache.v), x2)):
        raw = codes.view(torch.uint8)
        for l in range(L):
            for h in range(H):
                live = torch.zeros(T, dtype=torch.bool, device="cuda")
                for b, n in enumerate(lens):
                    live[starts[b]:starts[b] + n] = True
                if tokens is not None:
                    live &= tokens[l, h]
                want, es = quantize(x[l, h].double(), live, block)
                scales = torch.tensor([2.0 ** e for e in es], device="cuda", dtype=torch.float32)
                assert torch.equal(cache.scales[l, h, :, i], scales), f"scales l{l} h{h} {'kv'[i]}"
                got = codes[l, h].double()
                same = (got == want) | (torch.isnan(got) & torch.isnan(want))
                assert bool(same[live].all()), f"codes l{l} h{h} {'kv'[i]}"
                assert bool((raw[l, h][~live] == fill).all())


@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
@pytest.mark.parametrize("token_major,spare", [(False, 0), (True, 40)])
def test_quantize(jacap, dtype, d, block, token_major, spare):
    lens = [0, 1, 15, 16, 17, 128, 129, 300]
    rows, starts, k, v = wide_case(dtype, d, block, lens, spare, token_major, seed=block)
    k[0, 0, starts[7] + 3, 5], v[1, 1, starts[6] + 100, 0] = math.nan, -math.inf
    k[0, 1, starts[5] + 2, 1] = 3.3e38
    k[:, :, starts[4] + 16:starts[5]] = math.nan       # behind the tokens
    cache = empty_cache(jacap, *k.shape[:4], block, token_major)
    off = torch.tensor(starts, dtype=torch.int32, device="cuda")
    live = torch.tensor(lens, dtype=torch.int32, device="cuda")
    prob = jacap.prepare_quantize(k, v, cache, off, rows, live_lens=live)
    print(f"[quantize] {dtype} d{d} block {block}", flush=True)
    jacap.run_quantize(prob, k, v, cache)
    check_quantized(cache, (k, v), starts, lens, block)
    # empty slots have no token: their codes stay, their values count for nothing
    acc = torch.rand(k.shape[:3], device="cuda")
    acc[torch.rand(k.shape[:3], device="cuda") < 0.3] = -1.0
    k[acc < 0], v[acc < 0] = 1e30, math.nan
    cache2 = empty_cache(jacap, *k.shape[:4], block, token_major)
    jacap.run_quantize(prob, k, v, cache2, acc=acc)
    check_quantized(cache2, (k, v), starts, lens, block, tokens=acc >= 0)


def test_every_bfloat16_value(jacap):
    """Each of the 65536 patterns, alone in its block (a block of 16 equal tokens)."""
    bits = torch.arange(65536, dtype=torch.int32, device="cuda").to(torch.int16)
    x = bits.view(BF)[:, None, None].expand(65536, 16, 64).reshape(1, 1, -1, 64).contiguous()
    T = x.shape[2]
    cache = empty_cache(jacap, 1, 1, T, 64, 16, False)
    off = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    prob = jacap.prepare_quantize(x, x, cache, off, [T])
    jacap.run_quantize(prob, x, x, cache)
    one = x[0, 0, ::16, 0].double()
    es = torch.tensor([scale_exponent(abs(a) if math.isfinite(a) else 0.0) for a in one.tolist()],
                      device="cuda", dtype=torch.float64)
    want = torch.cat([codes_of(one[es == e], int(e)) for e in es.unique()])
    order = torch.cat([(es == e).nonzero()[:, 0] for e in es.unique()])
    assert torch.equal(cache.scales[0, 0, :, 0].double(), torch.exp2(es.cpu()).cuda())
    for codes in (cache.k, cache.v):
        got = codes[0, 0].view(65536, 16 * 64).double()
        assert torch.equal(torch.nan_to_num(got, nan=1e9).amax(1), torch.nan_to_num(got, nan=1e9).amin(1))
        same = (got[order, 0] == want) | (torch.isnan(got[order, 0]) & torch.isnan(want))
        assert bool(same.all())


class Appended:
    """The cache after an append, unit by unit."""

    def __init__(self, cache, acc, starts, rows):
        self.codes = [cache.k.double(), cache.v.double()]
        self.scales = cache.scales.double().clone()
        self.acc, self.starts, self.rows, self.block = acc.clone(), starts, rows, cache.block

    def unit(self, b, l, h, todo, src, acc_draft):
        """todo: (row of src, position) in order; src: K's and V's rows [S][d] in float64."""
        lo, bk = self.starts[b], self.block
        todo = [(r, at) for i, (r, at) in enumerate(todo) if 0 <= at < self.rows[b] and r >= 0
                and at not in [x for _, x in todo[i + 1:]]]
        for i in range(2):
            need = {}
            for r, at in todo:
                x = src[i][r]
                a = x[torch.isfinite(x)].abs()
                blk = (lo + at) // bk
                need[blk] = max(need.get(blk, -1000), scale_exponent(float(a.max()) if len(a) else 0.0))
            for blk, e in need.items():
                old = int(math.log2(float(self.scales[l, h, blk, i])))
                if e > old:
                    part = self.codes[i][l, h, blk * bk:(blk + 1) * bk]
                    part.copy_(codes_of(part, e - old))
                    self.scales[l, h, blk, i] = 2.0 ** e
            for r, at in todo:
                e = int(math.log2(float(self.scales[l, h, (lo + at) // bk, i])))
                self.codes[i][l, h, lo + at] = codes_of(src[i][r], e)
        for r, at in todo:
            self.acc[l, h, lo + at] = acc_draft[r] if acc_draft is not None else 0.0

    def check(self, cache, acc):
        assert torch.equal(cache.scales.double(), self.scales)
        for got, want in zip((cache.k, cache.v), self.codes):
            got = got.double()
            assert bool(((got == want) | (torch.isnan(got) & torch.isnan(want))).all())
        assert torch.equal(acc, self.acc)


def filled(jacap, dtype, d, block, lens, spare, token_major=False, seed=0, L=2, H=2):
    rows, starts, k, v = wide_case(dtype, d, block, lens, spare, token_major, L=L, H=H, seed=seed)
    cache = empty_cache(jacap, L, H, starts[-1], d, block, token_major, fill=0x31)
    off = torch.tensor(starts, dtype=torch.int32, device="cuda")
    live = torch.tensor(lens, dtype=torch.int32, device="cuda")
    jacap.run_quantize(jacap.prepare_quantize(k, v, cache, off, rows, live_lens=live), k, v, cache)
    return rows, starts, off, live, cache


def new_tokens(dtype, B, L, H, S, d, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = [(torch.randn((B, L, H, S, d), generator=gen, device="cuda") *
          2.0 ** torch.randint(-3, 9, (B, L, H, S, 1), generator=gen, device="cuda").float()).to(dtype)
         for _ in range(2)]
    return x[0], x[1], torch.rand((B, L, H, S), generator=gen, device="cuda")


@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("block,S,token_major", [(16, 1, False), (32, 4, True), (64, 9, False), (128, 40, True)])
def test_append_behind_the_tokens(jacap, dtype, d, block, S, token_major):
    """Accepted rows of a path, blocks begun and continued; a second append goes on in place."""
    lens = [0, 1, 16, 31, 200]
    rows, starts, off, live, cache = filled(jacap, dtype, d, block, lens, 2 * S + 1, token_major, seed=S)
    kd, vd, ad = new_tokens(dtype, 5, 2, 2, S, d, seed=3)
    kd[1, 0, 1, 0, 3], vd[2, 1, 0, S - 1, 0] = math.inf, math.nan
    acc = torch.rand(cache.k.shape[:3], device="cuda")
    gen = torch.Generator().manual_seed(5)
    prob = jacap.prepare_append_quant(kd, vd, cache, off, rows)
    start = live.clone()
    for turn in range(2):
        count = torch.randint(0, S + 1, (5,), generator=gen)
        count[4] = S
        path = torch.full((5, S), -1, dtype=torch.int32)
        for b in range(5):
            path[b, :count[b]] = torch.randperm(S, generator=gen)[:count[b]].sort().values.int()
        want = Appended(cache, acc, starts, rows)
        at = start.tolist()
        for b in range(5):
            todo = [(int(path[b, j]), at[b] + j) for j in range(int(count[b]))]
            for l in range(2):
                for h in range(2):
                    want.unit(b, l, h, todo, (kd[b, l, h].double(), vd[b, l, h].double()), ad[b, l, h])
        print(f"[append] {dtype} d{d} block {block} S{S} turn {turn}", flush=True)
        jacap.run_append_quant(prob, kd, vd, cache, start=start, rows=path.cuda(), count=count.int().cuda(),
                               acc=acc, acc_draft=ad, start_out=start)
        want.check(cache, acc)
        assert start.tolist() == [a + int(n) for a, n in zip(at, count)]
    assert int(prob.status) == 0


@pytest.mark.parametrize("dtype,d,S,block", [(BF, 128, 5, 32), (F32, 64, 31, 16), (BF, 64, 300, 128)])
def test_append_into_slots(jacap, dtype, d, S, block):
    """Evicted slots of each unit in any order, a slot listed twice, lists that run out, -1s and
    positions that are not the sequence's: what is not written is flagged, the rest is."""
    lens = [400, 0, 37, 512]
    rows, starts, off, live, cache = filled(jacap, dtype, d, block, lens, 0, seed=S)
    kd, vd, ad = new_tokens(dtype, 4, 2, 2, S, d, seed=4)
    acc = torch.rand(cache.k.shape[:3], device="cuda")
    prob = jacap.prepare_append_quant(kd, vd, cache, off, rows)
    gen = torch.Generator().manual_seed(7)
    cap = S + 3
    slots = torch.full((4, 2, 2, cap), -1, dtype=torch.int32)
    for b, n in enumerate(lens):
        for l in range(2):
            for h in range(2):
                m = min(n, cap)
                slots[b, l, h, :m] = torch.randperm(n, generator=gen)[:m].int() if n else slots[b, l, h, :m]
    first = torch.tensor([2, 0, 1, 3], dtype=torch.int32)
    for bad in (False, True):
        if bad:
            slots[0, 1, 1, 3] = slots[0, 1, 1, 4]      # twice
            slots[3, 0, 0, 3] = 512                     # not a row
            slots[3, 1, 0, 4] = -5
        want = Appended(cache, acc, starts, rows)
        for b in range(4):
            for l in range(2):
                for h in range(2):
                    todo = [(j, int(slots[b, l, h, int(first[b]) + j])) for j in range(S)
                            if int(first[b]) + j < cap]
                    want.unit(b, l, h, todo, (kd[b, l, h].double(), vd[b, l, h].double()), None)
        prob.status.zero_()
        print(f"[slots] {dtype} d{d} S{S} bad {bad}", flush=True)
        jacap.run_append_quant(prob, kd, vd, cache, start=first.cuda(), slots=slots.cuda(), acc=acc)
        want.check(cache, acc)
        assert prob.start_out.tolist() == [int(x) + S for x in first]
        assert int(prob.status) == jacap.FLAG_BAD_OFFSETS    # (sequence 1 has no slot)
    kept = cache.k.clone(), cache.scales.clone()
    jacap.run_append_quant(prob, kd, vd, cache, start=torch.tensor([-9, 5, 10 ** 9, 512], dtype=torch.int32).cuda(),
                           rows=torch.full((4, S), S, dtype=torch.int32).cuda(),
                           count=torch.tensor([1, 1, S + 9, -3], dtype=torch.int32).cuda())
    assert torch.equal(cache.k.view(torch.uint8), kept[0].view(torch.uint8)) and torch.equal(cache.scales, kept[1])


# ---------------------------------------------------------------------------
# Attention
# ---------------------------------------------------------------------------
ODD = [0, 1, 15, 16, 17, 33, 63, 65, 127, 129, 255, 257, 1000]


@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("S,G,tree,holes,spare,block,token_major", [
    (1, 4, None, 0.0, 0, 32, False), (1, 1, None, 0.1, 3, 16, True), (1, 7, None, 0.1, 0, 64, False),
    (5, 3, "tree", 0.1, 5, 128, False), (4, 4, "sparse", 0.0, 0, 16, False), (17, 2, "sparse", 0.2, 1, 32, True),
    (33, 4, "tree", 0.1, 0, 16, False), (67, 1, "sparse", 0.0, 2, 64, False), (16, 8, None, 0.0, 0, 128, True),
])
def test_attend(jacap, dtype, d, S, G, tree, holes, spare, block, token_major):
    c = QuantCase(jacap, ODD, S, dtype, d, block, spare, token_major, G=G, holes=holes, tree=tree, L=2, seed=S * G)
    for accumulate in (False, True):
        print(f"[attend] {dtype} d{d} S{S} G{G} block {block} accumulate {accumulate}", flush=True)
        prob, acc = run_attend(jacap, c, holes > 0, accumulate, decay=0.75)
        check_attend(c, prob, acc, holes > 0, accumulate, decay=0.75)


@pytest.mark.parametrize("dtype,S,lens,block", [
    (BF, 1, [70000, 3, 9000, 513, 512], 32), (BF, 63, [20000, 1, 8193], 16), (F32, 1, [9000, 1, 4096], 128),
    (F32, 9, [8193, 300], 16), (BF, 10, [8193, 300], 64), (BF, 300, [700, 0], 32), (BF, 512, [65], 16),
])
def test_attend_long(jacap, dtype, S, lens, block):
    """Many spans and chunks, the largest numbers of rows, row weights, decay 0."""
    c = QuantCase(jacap, lens, S, dtype, 128, block, H=1, G=2, holes=0.02, tree="tree" if S > 1 else None,
                  seed=5, spread=1.5)
    rw = torch.rand((len(lens), S), device="cuda") + 0.5
    rw[0, 0] = 0.0
    prob, acc = run_attend(jacap, c, True, True, decay=0.0, row_weight=rw)
    check_attend(c, prob, acc, True, True, decay=0.0, row_weight=rw)


@pytest.mark.parametrize("dtype,S,G", [(BF, 1, 2), (F32, 1, 1), (BF, 20, 1), (F32, 24, 2), (BF, 40, 1)])
def test_attend_many_sequences(jacap, dtype, S, G):
    gen = torch.Generator().manual_seed(11)
    lens = [int(x) for x in torch.randint(0, 90, (150,), generator=gen)]
    lens[3], lens[70], lens[149] = 2000, 9000, 700
    c = QuantCase(jacap, lens, S, dtype, 64, 16, 2, H=1, G=G, holes=0.1, tree="tree" if S > 1 else None, seed=8)
    prob, acc = run_attend(jacap, c, True, True)
    check_attend(c, prob, acc, True, True)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("S", [1, 3, 24, 50])
def test_rows_that_see_nothing(jacap, dtype, S):
    c = QuantCase(jacap, [40, 0, 600], S, dtype, 128, 32, tree="sparse", seed=1)
    c.acc.fill_(-1.0)
    c.tree.zero_()
    prob, acc = run_attend(jacap, c, True, True)
    assert torch.equal(prob.out, torch.zeros_like(prob.out))
    assert torch.equal(prob.lse, torch.full_like(prob.lse, -math.inf))
    assert torch.equal(prob.acc_draft, torch.zeros_like(prob.acc_draft))
    assert torch.equal(acc, c.acc)


@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("S", [1, 7, 21, 50])
def test_nan_codes_in_hidden_places(jacap, dtype, d, S):
    """NaN codes of empty slots and behind the tokens, and infinities of a drafted token that
    only its own row sees, take no part; a visible NaN code makes its rows NaN."""
    c = QuantCase(jacap, [50, 700, 0], S, dtype, d, 16, 9, holes=0.3, tree="tree", seed=4)
    hidden = c.acc < 0
    c.cache.k.view(torch.uint8)[hidden] = 0x7F
    c.cache.v.view(torch.uint8)[hidden] = 0xFF
    c.k[hidden] = math.nan
    c.v[hidden] = math.nan
    last = torch.stack([sees_tree(c.tree, S, b) for b in range(3)])[:, :S - 1, S - 1]
    assert not last.any()
    if S > 1:
        c.vd[:, :, :, S - 1, 1::5] = math.inf
        prob, acc = run_attend(jacap, c, True, True)
        out = prob.out.view(3, 1, c.H, c.G, S, d)
        assert torch.isfinite(out[..., :S - 1, :]).all() and torch.isinf(out[..., S - 1, 1::5]).all()
        c.vd[:, :, :, S - 1, 1::5] = 0.5
    prob, acc = run_attend(jacap, c, True, True)
    check_attend(c, prob, acc, True, True)
    at = int((c.acc[0, 0, :50] >= 0).nonzero()[3])
    c.cache.k.view(torch.uint8)[0, 0, at, 2] = 0x7F
    prob, acc = run_attend(jacap, c, True, False)
    assert torch.isnan(prob.lse[0, :, :c.G]).all() and torch.isfinite(prob.lse[:, :, c.G:]).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("S", [3, 40])
def test_layouts(jacap, dtype, S):
    """Codes token-major; query rows and drafted tokens inside larger tensors."""
    c = QuantCase(jacap, [300, 77], S, dtype, 64, 32, 0, True, H=3, G=2, L=2, holes=0.1, tree="tree", seed=3)
    wide = torch.zeros((2, 2, 6, S + 2, 96), dtype=dtype, device="cuda")
    wide[..., 1:-1, 8:72] = c.q
    c.q = wide[..., 1:-1, 8:72]
    big = torch.zeros((2, S, 2, 2, 3, 64), dtype=dtype, device="cuda")
    for i, x in enumerate((c.kd, c.vd)):
        big[:, :, i] = x.permute(0, 3, 1, 2, 4)
    c.kd, c.vd = (big[:, :, i].permute(0, 2, 3, 1, 4) for i in range(2))
    prob, acc = run_attend(jacap, c, True, True)
    check_attend(c, prob, acc, True, True)


@pytest.mark.parametrize("dtype,S,G", [(BF, 1, 4), (F32, 3, 2), (BF, 40, 2)])
def test_bad_offsets_are_flagged(jacap, dtype, S, G):
    """A sequence that begins inside a block, or whose length is not of its rows, is empty."""
    c = QuantCase(jacap, [200, 64, 100], S, dtype, 64, 32, H=2, G=G, seed=6)
    for what in ("offset", "live"):
        off, live = c.offsets.clone(), c.live.clone()
        if what == "offset":
            off[1] += 8        # sequences 0 and 1
        else:
            live[1] = 65
        p = jacap.AttentionParams(live_lens=live)
        prob = jacap.prepare_attend_quant(c.q, c.cache, c.kd, c.vd, off, c.rows, p)
        jacap.run_attend_quant(prob, c.q, c.cache, c.kd, c.vd)
        assert jacap.read_status(prob.ws) == jacap.FLAG_BAD_OFFSETS
        saved, c.lens = c.lens, [0, 0, 100] if what == "offset" else [200, 0, 100]
        check_attend(c, prob, None, False, False)
        c.lens = saved
        wprob = jacap.prepare_attn_weights_quant(c.q, c.cache, off, c.rows, p)
        acc = torch.zeros_like(c.acc)
        jacap.run_attn_weights_quant(wprob, c.q, c.cache, acc, prob.lse.clone())
        assert int(wprob.status) == jacap.FLAG_BAD_OFFSETS
        a, e = c.starts[1], c.starts[2]
        assert torch.equal(acc[:, :, a:e], torch.zeros_like(acc[:, :, a:e])) and bool((acc[:, :, e:e + 100] > 0).all())


# ---------------------------------------------------------------------------
# Accumulated weights of rows whose lse is known
# ---------------------------------------------------------------------------
def check_weights(jacap, c, lse, row_weight=None, decay=1.0):
    p = jacap.AttentionParams(decay=decay, live_lens=c.live, row_weight=row_weight)
    prob = jacap.prepare_attn_weights_quant(c.q, c.cache, c.offsets, c.rows, p)
    acc = c.acc.clone()
    jacap.run_attn_weights_quant(prob, c.q, c.cache, acc, lse)
    assert int(prob.status) == 0
    R = c.G * c.S
    for b, n in enumerate(c.lens):
        rw = (row_weight[b].double() if row_weight is not None else
              torch.ones(c.S, dtype=torch.float64, device="cuda")).repeat(c.G)
        for l in range(c.L):
            for h in range(c.H):
                q, sl = c.unit(b, l, h)
                w = Weights(q, c.k[l, h, sl], c.scale, torch.ones((R, n), dtype=torch.bool, device="cuda"))
                ls = lse[b, l, h * c.G:(h + 1) * c.G].reshape(-1).double()
                use = (rw != 0) & (ls > -math.inf)
                z = (q.double() @ c.k[l, h, sl].double().t().contiguous()) * c.scale
                pr = torch.exp(z - torch.where(use, ls, torch.zeros_like(ls))[:, None])
                given = torch.where(use[:, None], rw[:, None] * pr, torch.zeros_like(pr)).sum(0)
                size = torch.where(use[:, None], (rw[:, None] * pr).abs(), torch.zeros_like(pr)).sum(0)
                top = float(ls[use].abs().max()) if bool(use.any()) else 0.0
                rel = w.rel + 8 * U * top * 1.4427 + (R + 8) * U
                old = c.acc[l, h, sl].double()
                want = torch.where(old < 0, old, decay * old + given)
                check(acc[l, h, sl], want, rel * size + 4 * U * want.abs() + 1e-30, f"acc b{b} l{l} h{h} n{n}")
        a, e = c.starts[b] + n, c.starts[b + 1]
        assert torch.equal(acc[:, :, a:e], c.acc[:, :, a:e])
    return acc


@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("S,G,block,share,decay", [(1, 4, 16, 1.0, 0.0), (31, 2, 32, 0.2, 0.98), (63, 4, 64, 0.1, 1.0),
                                                   (300, 5, 128, 0.9, 0.5), (8, 1, 16, 0.0, 0.5)])
def test_weights(jacap, dtype, d, S, G, block, share, decay):
    c = QuantCase(jacap, ODD, S, dtype, d, block, 3, H=1, G=G, L=2, holes=0.1, seed=S)
    gen = torch.Generator(device="cuda").manual_seed(2)
    rw = (torch.rand((len(ODD), S), generator=gen, device="cuda") < share).float() * 1.5
    lse = 4.0 + torch.rand((len(ODD), 2, G, S), generator=gen, device="cuda")
    lse[:, :, :, S // 2] = -math.inf
    lse[3] = math.nan
    rw[3] = 0.0                 # rows of weight 0 add nothing, whatever they hold
    c.q[3] = math.nan
    print(f"[weights] {dtype} d{d} S{S} G{G}", flush=True)
    acc = check_weights(jacap, c, lse, rw, decay)
    c.q[3] = 0.25
    lse[3] = 5.0
    check_weights(jacap, c, lse, None, decay)


# ---------------------------------------------------------------------------
# Graphs, streams, two problems
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,S,G", [(BF, 1, 4), (BF, 63, 4), (F32, 5, 2)])
def test_captured_step(jacap, dtype, S, G):
    """Append and attention captured together and replayed as the lengths grow, eager work
    between the replays: each replay is the eager step's result, to the bit."""
    lens = [100, 0, 31, 700]
    c = QuantCase(jacap, lens, S, dtype, 64, 32, 5 * S, H=2, G=G, holes=0.0, tree="tree" if S > 1 else None, seed=3)
    acc = c.acc.clone()
    p = jacap.AttentionParams(accumulate=True, live_lens=c.live, tree=c.tree)
    prob = jacap.prepare_attend_quant(c.q, c.cache, c.kd, c.vd, c.offsets, c.rows, p)
    ap = jacap.prepare_append_quant(c.kd, c.vd, c.cache, c.offsets, c.rows)

    def step():
        jacap.run_attend_quant(prob, c.q, c.cache, c.kd, c.vd, acc=acc)
        jacap.run_append_quant(ap, c.kd, c.vd, c.cache, start=c.live, acc=acc, acc_draft=prob.acc_draft,
                               start_out=c.live)

    state = [c.cache.k.view(torch.uint8), c.cache.v.view(torch.uint8), c.cache.scales, acc, c.live]
    saved = [x.clone() for x in state]
    results = []
    for _ in range(4):
        step()
        results.append([x.clone() for x in state + [prob.out, prob.lse]])
    for x, y in zip(state, saved):
        x.copy_(y)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step()
    for x, y in zip(state, saved):
        x.copy_(y)
    for want in results:
        graph.replay()
        torch.cuda.synchronize()
        for got, w in zip(state + [prob.out, prob.lse], want):
            assert torch.equal(torch.nan_to_num(got.float()), torch.nan_to_num(w.float()))
        prob.out.zero_()
        torch.randn((64, 64), device="cuda").sum()
        torch.cuda.synchronize()
    assert int(ap.status) == 0 and jacap.read_status(prob.ws) == 0


def test_streams_and_repeats(jacap):
    """Two problems on two streams at once, each the same every time."""
    cases = [QuantCase(jacap, [5000, 33], S, BF, 128, 32, H=2, G=4, seed=S) for S in (1, 33)]
    probs = [jacap.prepare_attend_quant(c.q, c.cache, c.kd, c.vd, c.offsets, c.rows,
                                        jacap.AttentionParams(live_lens=c.live)) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    first = None
    for _ in range(5):
        for c, p, s in zip(cases, probs, streams):
            jacap.run_attend_quant(p, c.q, c.cache, c.kd, c.vd, stream=s)
        torch.cuda.synchronize()
        got = [(p.out.clone(), p.lse.clone()) for p in probs]
        first = first or got
        assert all(torch.equal(a, b) for x, y in zip(first, got) for a, b in zip(x, y))
    for c, p in zip(cases, probs):
        check_attend(c, p, None, False, False)


@pytest.mark.parametrize("dtype,S,G", [(BF, 1, 4), (F32, 5, 2), (BF, 40, 2)])
def test_no_cached_tokens_at_all(jacap, dtype, S, G):
    """A cache of no rows: attention of the drafted tokens among themselves."""
    c = Case([0, 0], S, dtype, 64, H=2, G=G, seed=2)
    cache = jacap.alloc_quant_cache(1, 2, 0, 64)
    for accumulate in (False, True):
        p = jacap.AttentionParams(accumulate=accumulate)
        prob = jacap.prepare_attend_quant(c.q, cache, c.kd, c.vd, c.offsets, [0, 0], p)
        acc = torch.zeros((1, 2, 0), device="cuda")
        jacap.run_attend_quant(prob, c.q, cache, c.kd, c.vd, acc=acc)
        assert jacap.read_status(prob.ws) == 0
        c.acc, c.live = acc, None
        check_attend(c, prob, acc, False, accumulate)
    wp = jacap.prepare_attn_weights_quant(c.q, cache, c.offsets, [0, 0], p)
    jacap.run_attn_weights_quant(wp, c.q, cache, acc, prob.lse)
    k = torch.empty((1, 2, 0, 64), dtype=dtype, device="cuda")
    jacap.run_quantize(jacap.prepare_quantize(k, k, cache, c.offsets, [0, 0]), k, k, cache)
    ap = jacap.prepare_append_quant(c.kd, c.vd, cache, c.offsets, [0, 0])
    jacap.run_append_quant(ap, c.kd, c.vd, cache, start=torch.zeros(2, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    assert int(ap.status) == jacap.FLAG_BAD_OFFSETS      # there is no room


def test_offsets_past_32_bits(jacap):
    """Codes and drafted rows more than 2^32 bytes apart: a cache of 34 M rows of one head (4.4
    GB each of K and V), two sequences at its ends, the rows between them reserved."""
    T, d = 34 * (1 << 20), 128
    ends = [200, 333]
    cache = jacap.QuantCache(torch.empty((1, 1, T, d), dtype=E4, device="cuda"),
                             torch.empty((1, 1, T, d), dtype=E4, device="cuda"),
                             torch.full((1, 1, T // 32, 2), 2.0 ** -100, device="cuda"), 32)
    rows = [T - 512, 512]
    off = torch.tensor([0, T - 512, T], dtype=torch.int32, device="cuda")
    live = torch.tensor(ends, dtype=torch.int32, device="cuda")
    c = Case(ends, 3, BF, d, H=1, G=2, seed=31)
    S = 3
    # the tokens are appended, some at a time, to where each sequence begins
    start = torch.zeros(2, dtype=torch.int32, device="cuda")
    kd, vd = torch.zeros((2, 1, 1, 333, d), dtype=BF, device="cuda"), torch.zeros((2, 1, 1, 333, d), dtype=BF, device="cuda")
    for b, n in enumerate(ends):
        sl = slice(c.starts[b], c.starts[b] + n)
        kd[b, 0, 0, :n], vd[b, 0, 0, :n] = c.k[0, 0, sl], c.v[0, 0, sl]
    ap = jacap.prepare_append_quant(kd, vd, cache, off, rows)
    jacap.run_append_quant(ap, kd, vd, cache, start=start, count=live, start_out=start)
    assert start.tolist() == ends and int(ap.status) == 0
    for b, n in enumerate(ends):
        lo = int(off[b])
        for x, codes, i in ((c.k, cache.k, 0), (c.v, cache.v, 1)):
            rowsn = up_to(n, 32)
            fine = cache.scales[0, 0, lo // 32:(lo + rowsn) // 32, i].repeat_interleave(32)[:n, None]
            got = codes[0, 0, lo:lo + n].float() * fine
            ref = x[0, 0, c.starts[b]:c.starts[b] + n]
            assert bool(((got - ref.float()).abs() <= torch.maximum(ref.float().abs() / 16, fine / 1024)).all())
            ref.copy_(got.to(BF))
    prob = jacap.prepare_attend_quant(c.q, cache, c.kd, c.vd, off, rows, jacap.AttentionParams(live_lens=live))
    jacap.run_attend_quant(prob, c.q, cache, c.kd, c.vd)
    c.live = None
    check_attend(c, prob, None, False, False)


@pytest.mark.parametrize("B", [300, 700])
def test_many_sequences_that_accumulate(jacap, B):
    """More sequences than a workgroup has threads: each finds the blocks of its tokens."""
    gen = torch.Generator().manual_seed(B)
    lens = [int(x) for x in torch.randint(0, 40, (B,), generator=gen)]
    lens[17], lens[B - 2] = 2500, 1100
    c = QuantCase(jacap, lens, 1, BF, 64, 16, 1, H=1, G=2, holes=0.1, seed=B)
    prob, acc = run_attend(jacap, c, True, True, decay=0.5)
    check_attend(c, prob, acc, True, True, decay=0.5)


@pytest.mark.parametrize("wide", [False, True])
def test_accumulation_at_lengths_far_apart(jacap, wide):
    """A long sequence among short and empty ones, with slots that are not full: the weights are
    joined by blocks of the tokens there are."""
    gen = torch.Generator().manual_seed(3)
    lens = [int(x) for x in torch.randint(0, 40, (300,), generator=gen)]
    lens[17], lens[280], lens[299] = 20000, 1100, 0
    kw = dict(H=1, G=2, holes=0.1, seed=5)
    if wide:
        c = Case(lens, 1, BF, 64, spare=7, **kw)
        prob, acc = test_gpu_attention.run_attend(jacap, c, True, True, decay=0.5)
        test_gpu_attention.check_attend(c, prob, acc, True, True, decay=0.5)
    else:
        c = QuantCase(jacap, lens, 1, BF, 64, 16, 1, **kw)
        prob, acc = run_attend(jacap, c, True, True, decay=0.5)
        check_attend(c, prob, acc, True, True, decay=0.5)


def test_another_device_is_refused(jacap, monkeypatch):
    """A run with another device current, or on another device's stream, enqueues nothing."""
    c = QuantCase(jacap, [50, 20], 3, BF, 64, 32, H=2, G=2, seed=26)
    p = jacap.AttentionParams(accumulate=True, live_lens=c.live)
    prob = jacap.prepare_attend_quant(c.q, c.cache, c.kd, c.vd, c.offsets, c.rows, p)
    wp = jacap.prepare_attn_weights_quant(c.q, c.cache, c.offsets, c.rows, p)
    qp = jacap.prepare_quantize(c.k, c.v, c.cache, c.offsets, c.rows, live_lens=c.live)
    ap = jacap.prepare_append_quant(c.kd, c.vd, c.cache, c.offsets, c.rows)
    logits = torch.randn((2, 3, 50), device="cuda")
    tokens = torch.zeros((2, 3), dtype=torch.int32, device="cuda")
    vp = jacap.prepare_verify(logits, jacap.VerifyParams(temperature=0.0))
    acc, start = c.acc.clone(), c.live.clone()
    held = [x.view(torch.uint8).clone() for x in (c.cache.k, c.cache.v, c.cache.scales)]
    for x in (prob.out, vp.next):
        x.fill_(7)

    class Elsewhere:
        device_index, cuda_stream = 1, 0

    def refused(stream):
        for run in (lambda: jacap.run_attend_quant(prob, c.q, c.cache, c.kd, c.vd, acc=acc, stream=stream),
                    lambda: jacap.run_attn_weights_quant(wp, c.q, c.cache, acc, prob.lse, stream=stream),
                    lambda: jacap.run_quantize(qp, c.k, c.v, c.cache, stream=stream),
                    lambda: jacap.run_append_quant(ap, c.kd, c.vd, c.cache, start=start, stream=stream),
                    lambda: jacap.run_verify(vp, logits, tokens, stream=stream)):
            with pytest.raises(ValueError):
                run()

    refused(Elsewhere)
    with monkeypatch.context() as m:
        m.setattr(torch.cuda, "current_device", lambda: 1)
        refused(None)
    torch.cuda.synchronize()
    assert torch.equal(acc, c.acc) and bool((prob.out == 7).all()) and bool((vp.next == 7).all())
    for x, y in zip((c.cache.k, c.cache.v, c.cache.scales), held):
        assert torch.equal(x.view(torch.uint8), y)
    side = torch.cuda.Stream()
    jacap.run_attend_quant(prob, c.q, c.cache, c.kd, c.vd, acc=acc, stream=side)
    torch.cuda.synchronize()
    check_attend(c, prob, acc, True, True)


def test_refusals(jacap):
    c = QuantCase(jacap, [100, 20], 3, BF, 64, 32, H=2, G=2, seed=1)
    p = jacap.AttentionParams(live_lens=c.live)
    prep = lambda **kw: jacap.prepare_attend_quant(**{**dict(
        q=c.q, cache=c.cache, kd=c.kd, vd=c.vd, seq_offsets=c.offsets, seq_lens=c.rows, params=p), **kw})
    Q = jacap.QuantCache
    prob = prep()
    for bad in (dict(q=c.q.float()), dict(kd=c.kd[..., :32]), dict(seq_lens=[120, 40]), dict(seq_lens=[128]),
                dict(cache=Q(c.cache.k, c.cache.v, c.scales, 64)), dict(cache=Q(c.cache.k, c.cache.v, c.scales, 8)),
                dict(cache=Q(c.cache.k.float(), c.cache.v, c.scales, 32)),
                dict(cache=Q(c.cache.k, c.cache.v, c.scales.double(), 32)),
                dict(cache=Q(c.cache.k, c.cache.v[:, :, :32], c.scales, 32)), dict(seq_offsets=c.offsets.long())):
        with pytest.raises(ValueError):
            prep(**bad)
    with pytest.raises(ValueError):
        jacap.run_attend_quant(prob, c.q, c.cache, c.kd, c.vd.float())
    with pytest.raises(ValueError):
        jacap.run_attend_quant(prob, c.q, Q(c.cache.k, c.cache.v, c.scales[:, :, :1], 32), c.kd, c.vd)
    ap = jacap.prepare_append_quant(c.kd, c.vd, c.cache, c.offsets, c.rows)
    with pytest.raises(ValueError):
        jacap.run_append_quant(ap, c.kd, c.vd, c.cache)
    with pytest.raises(ValueError):
        jacap.run_append_quant(ap, c.kd, c.vd, c.cache, start=c.live.long())
    with pytest.raises(ValueError):
        jacap.prepare_quantize(c.k[:, :, :32], c.v[:, :, :32], c.cache, c.offsets, c.rows)
    with pytest.raises(ValueError):
        jacap.alloc_quant_cache(1, 1, 100, 64, block=32)

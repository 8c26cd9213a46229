"""jacap_attend and jacap_attn_weights against the formulas in float64, with the
bounds of attention_ref.py: ragged lengths around the tiles and chunks, trees,
empty slots, rows that see nothing, NaN in hidden places, layouts, lengths of
their own, graphs, streams."""

import math

import pytest
import torch

from attention_ref import U, Weights, check, half_step, sees_tree

pytestmark = pytest.mark.gpu

BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def jacap():
    from paper_2609_08131_amd import jacap as j
    return j


class Case:
    """A cache of B sequences with query rows and drafted tokens."""

    def __init__(self, lens, S, dtype=BF, d=128, H=2, G=4, L=1, holes=0.0, spare=0, tree=None,
                 token_major=False, seed=0, spread=1.0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.randn(s, generator=gen, device="cuda")
        B = len(lens)
        self.lens, self.S, self.d, self.H, self.G, self.L = lens, S, d, H, G, L
        self.rows = [n + spare for n in lens]
        self.starts = [sum(self.rows[:b]) for b in range(B + 1)]
        T = self.starts[-1]
        if token_major:
            self.k = rnd(L, T, H, d).to(dtype).transpose(1, 2)
            self.v = rnd(L, T, H, d).to(dtype).transpose(1, 2)
        else:
            self.k, self.v = rnd(L, H, T, d).to(dtype), rnd(L, H, T, d).to(dtype)
        self.q = (spread * rnd(B, L, H * G, S, d)).to(dtype)
        self.kd, self.vd = rnd(B, L, H, S, d).to(dtype), rnd(B, L, H, S, d).to(dtype)
        self.acc = torch.rand((L, H, T), generator=gen, device="cuda")
        if holes:
            self.acc[torch.rand((L, H, T), generator=gen, device="cuda") < holes] = -1.0
        self.offsets = torch.tensor(self.starts, dtype=torch.int32, device="cuda")
        self.live = torch.tensor(lens, dtype=torch.int32, device="cuda") if spare else None
        self.scale = d ** -0.5
        self.tree = None
        host = torch.Generator().manual_seed(seed + 1)
        if tree == "tree":
            sees = torch.zeros((B, S, S), dtype=torch.bool)
            for b in range(B):
                for j in range(S):
                    up = int(torch.randint(-1, j, (1,), generator=host)) if j else -1
                    if up >= 0:
                        sees[b, j] = sees[b, up]
                    sees[b, j, j] = True
        elif tree == "sparse":      # any mask, rows that see no drafted token among them
            sees = torch.rand((B, S, S), generator=host) < 0.3
            sees[:, ::3] = False
        if tree:
            words = (S + 63) // 64
            bits = torch.zeros((B, S, words * 64), dtype=torch.int64)
            bits[:, :, :S] = sees.long()
            t = (bits.view(B, S, words, 64) << torch.arange(64)).sum(-1)
            self.tree = t.cuda()

    def unit(self, b, l, h):
        lo, n = self.starts[b], self.lens[b]
        q = self.q[b, l, h * self.G:(h + 1) * self.G].reshape(self.G * self.S, self.d)
        return q, slice(lo, lo + n)


def run_attend(jacap, c, use_acc, accumulate, decay=1.0, row_weight=None):
    p = jacap.AttentionParams(accumulate=accumulate, decay=decay, live_lens=c.live, tree=c.tree,
                              row_weight=row_weight)
    prob = jacap.prepare_attend(c.q, c.k, c.v, c.kd, c.vd, c.offsets, c.rows, p)
    acc = c.acc.clone() if use_acc or accumulate else None
    prob.out.fill_(7.0)
    prob.lse.fill_(7.0)
    jacap.run_attend(prob, c.q, c.k, c.v, c.kd, c.vd, acc=acc)
    assert jacap.read_status(prob.ws) == 0
    return prob, acc


def check_attend(c, prob, acc, use_acc, accumulate, decay=1.0, row_weight=None):
    S, G, H = c.S, c.G, c.H
    h_ = half_step(c.k.dtype)
    for b, n in enumerate(c.lens):
        sees = sees_tree(c.tree, S, b).cuda().repeat(G, 1)
        rw = torch.ones(G * S, dtype=torch.float64, device="cuda")
        if row_weight is not None:
            rw = row_weight[b].double().repeat(G)
        for l in range(c.L):
            for h in range(H):
                q, sl = c.unit(b, l, h)
                vis = torch.ones((G * S, n + S), dtype=torch.bool, device="cuda")
                vis[:, n:] = sees
                hidden = c.acc[l, h, sl] < 0
                if use_acc or accumulate:
                    vis[:, :n] &= ~hidden
                w = Weights(q, torch.cat([c.k[l, h, sl], c.kd[b, l, h]]), c.scale, vis)
                v = torch.cat([c.v[l, h, sl], c.vd[b, l, h]]).double()
                # V of what no row sees may hold anything
                v = torch.where(vis.any(0)[:, None], v, torch.zeros_like(v))
                out = w.p @ v
                tag = f"b{b} l{l} h{h} n{n}"
                got = prob.out[b, l, h * G:(h + 1) * G].reshape(G * S, -1)
                extra = h_ if c.k.dtype == BF else (n + S) * U
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
    if acc is not None and c.live is not None:   # rows past the live lengths stay
        for b, n in enumerate(c.lens):
            a, e = c.starts[b] + n, c.starts[b + 1]
            assert torch.equal(acc[:, :, a:e], c.acc[:, :, a:e])


ODD = [0, 1, 15, 16, 17, 33, 127, 129, 255, 257, 1000]


@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("S,G,tree,holes,spare", [
    (1, 4, None, 0.0, 0), (1, 1, None, 0.1, 3), (1, 7, None, 0.1, 0), (5, 3, "tree", 0.1, 5),
    (4, 4, "sparse", 0.0, 0), (17, 2, "sparse", 0.2, 1), (33, 4, "tree", 0.1, 0), (67, 1, "sparse", 0.0, 2),
    (16, 8, None, 0.0, 0),
])
def test_attend(jacap, dtype, d, S, G, tree, holes, spare):
    c = Case(ODD, S, dtype, d, G=G, holes=holes, spare=spare, tree=tree, L=2, seed=S * G)
    for accumulate in (False, True):
        print(f"[attend] {dtype} d{d} S{S} G{G} accumulate {accumulate}", flush=True)
        prob, acc = run_attend(jacap, c, holes > 0, accumulate, decay=0.75)
        check_attend(c, prob, acc, holes > 0, accumulate, decay=0.75)


@pytest.mark.parametrize("dtype,S,lens", [
    (BF, 1, [70000, 3, 9000, 513, 512]), (BF, 63, [20000, 1, 8193]), (F32, 1, [9000, 1, 4096]),
    (F32, 9, [8193, 300]), (BF, 300, [700, 0]), (BF, 512, [65]),
])
def test_attend_long(jacap, dtype, S, lens):
    """Many chunks, the largest numbers of rows, row weights, decay 0."""
    c = Case(lens, S, dtype, 128, H=1, G=2, holes=0.02, tree="tree" if S > 1 else None, seed=5,
             spread=1.5)
    rw = torch.rand((len(lens), S), device="cuda") + 0.5
    rw[0, 0] = 0.0
    prob, acc = run_attend(jacap, c, True, True, decay=0.0, row_weight=rw)
    check_attend(c, prob, acc, True, True, decay=0.0, row_weight=rw)


@pytest.mark.parametrize("dtype,S,G", [(BF, 1, 2), (F32, 1, 1), (BF, 20, 1), (F32, 24, 2), (BF, 40, 1)])
def test_attend_many_sequences(jacap, dtype, S, G):
    """More sequences than a wave has lanes, most of them short, one long: the spans'
    search, units that begin and end inside a span, rows of several blocks (fp32)."""
    gen = torch.Generator().manual_seed(11)
    lens = [int(x) for x in torch.randint(0, 90, (150,), generator=gen)]
    lens[3], lens[70], lens[149] = 2000, 9000, 700
    c = Case(lens, S, dtype, 64, H=1, G=G, holes=0.1, spare=2, tree="tree" if S > 1 else None, seed=8)
    prob, acc = run_attend(jacap, c, True, True)
    check_attend(c, prob, acc, True, True)


@pytest.mark.parametrize("lens", [[0], [0, 0, 0], [1], [0, 200000, 0, 5]])
def test_attend_lengths_of_nothing_beside_long_ones(jacap, lens):
    c = Case(lens, 1, BF, 64, H=2, G=1, seed=14)
    prob, acc = run_attend(jacap, c, False, True)
    check_attend(c, prob, acc, False, True)


def test_capacity_far_above_the_lengths(jacap):
    """Caches with room for far more than they hold."""
    c = Case([900, 3, 0, 257], 1, BF, 128, H=2, G=4, spare=30000, holes=0.05, seed=15)
    prob, acc = run_attend(jacap, c, True, True)
    check_attend(c, prob, acc, True, True)


def test_attend_longest_context(jacap):
    c = Case([131072], 1, BF, 128, H=1, G=8, seed=9)
    prob, acc = run_attend(jacap, c, False, True)
    check_attend(c, prob, acc, False, True)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("S", [3, 40])
def test_layouts(jacap, dtype, S):
    """K and V token-major; query rows, drafted tokens and outputs inside larger tensors."""
    c = Case([300, 77], S, dtype, 64, H=3, G=2, L=2, token_major=True, holes=0.1, tree="tree", seed=3)
    wide = torch.zeros((2, 2, 6, S + 2, 96), dtype=dtype, device="cuda")
    wide[..., 1:-1, 8:72] = c.q
    c.q = wide[..., 1:-1, 8:72]
    big = torch.zeros((2, S, 2, 2, 3, 64), dtype=dtype, device="cuda")  # [B][S][kv][L][H][d]
    for i, x in enumerate((c.kd, c.vd)):
        big[:, :, i] = x.permute(0, 3, 1, 2, 4)
    c.kd, c.vd = (big[:, :, i].permute(0, 2, 3, 1, 4) for i in range(2))
    prob, acc = run_attend(jacap, c, True, True)
    check_attend(c, prob, acc, True, True)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("S", [1, 3, 24])
def test_rows_that_see_nothing(jacap, dtype, S):
    """Every slot empty and masks without a bit: out 0, lse -inf, weights 0."""
    c = Case([40, 0, 600], S, dtype, 128, tree="sparse", seed=1)
    c.acc.fill_(-1.0)
    c.tree.zero_()
    prob, acc = run_attend(jacap, c, True, True)
    assert torch.equal(prob.out, torch.zeros_like(prob.out))
    assert torch.equal(prob.lse, torch.full_like(prob.lse, -math.inf))
    assert torch.equal(prob.acc_draft, torch.zeros_like(prob.acc_draft))
    assert torch.equal(acc, c.acc)


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("S", [2, 7, 11, 21, 50])
def test_non_finite_values_in_hidden_places(jacap, dtype, d, S, value):
    """K and V of empty slots, of rows past the live lengths and of drafted tokens
    that a row does not see take no part in that row."""
    c = Case([50, 700, 0], S, dtype, d, holes=0.3, spare=9, tree="tree", seed=4)
    hidden = c.acc < 0
    for b, n in enumerate(c.lens):
        hidden[:, :, c.starts[b] + n:c.starts[b + 1]] = True
    c.k[hidden] = value
    c.v[hidden] = value
    # the last drafted token is seen by its own row only
    sees = torch.stack([sees_tree(c.tree, S, b) for b in range(3)])
    assert not sees[:, :S - 1, S - 1].any()
    c.vd[:, :, :, S - 1, 1::5] = value
    prob, acc = run_attend(jacap, c, True, True)
    for b, n in enumerate(c.lens):
        for h in range(c.H):
            q, sl = c.unit(b, 0, h)
            vis = torch.ones((c.G * S, n + S), dtype=torch.bool, device="cuda")
            vis[:, :n] = ~(c.acc[0, h, sl] < 0)
            vis[:, n:] = sees[b].cuda().repeat(c.G, 1)
            w = Weights(q, torch.cat([c.k[0, h, sl], c.kd[b, 0, h]]), c.scale, vis)
            v = torch.cat([c.v[0, h, sl], c.vd[b, 0, h]]).double()
            out = torch.zeros((c.G * S, c.d), dtype=torch.float64, device="cuda")
            size = torch.zeros_like(out)
            for r in range(c.G * S):
                seen = vis[r]
                out[r] = w.p[r, seen] @ v[seen]
                size[r] = w.p[r, seen] @ v[seen].abs()
            h_ = half_step(dtype)
            tol = (w.rel + h_ + (n + S) * U) * size + h_ * out.abs() + 1e-30
            got = prob.out[b, 0, h * c.G:(h + 1) * c.G].reshape(c.G * S, -1)
            check(got, out, torch.nan_to_num(tol), f"b{b} h{h}")
            check(prob.lse[b, 0, h * c.G:(h + 1) * c.G].reshape(-1), w.lse, w.lse_tol, "lse")
    assert torch.isfinite(prob.acc_draft).all()
    assert torch.isfinite(acc).all()


def test_non_finite_queries_stay_in_their_rows(jacap):
    c = Case([300], 6, BF, 128, tree="tree", seed=6)
    c.q[0, 0, 3, 2, 5] = math.nan
    prob, _ = run_attend(jacap, c, False, False)
    bad = torch.zeros(prob.lse.shape, dtype=torch.bool, device="cuda")
    bad[0, 0, 3, 2] = True
    assert torch.equal(torch.isnan(prob.lse), bad)
    assert torch.equal(torch.isnan(prob.out).any(-1), bad)


def test_large_logits(jacap):
    """Logits of thousands: the weights are those of the largest."""
    c = Case([500, 31], 3, BF, 128, seed=8, spread=400.0)
    prob, acc = run_attend(jacap, c, False, True)
    check_attend(c, prob, acc, False, True)


# ---------------------------------------------------------------------------
# attn_weights
# ---------------------------------------------------------------------------
def check_weights(jacap, c, causal, given=None, row_weight=None, decay=1.0):
    w_, G, H = c.S, c.G, c.H
    p = jacap.AttentionParams(causal=causal, live_lens=c.live, row_weight=row_weight, decay=decay)
    prob = jacap.prepare_attn_weights(c.q, c.k, c.offsets, c.rows, p)
    acc = c.acc.clone()
    jacap.run_attn_weights(prob, c.q, c.k, acc, lse=given)
    assert jacap.read_status(prob.ws) == 0
    for b, n in enumerate(c.lens):
        pos = torch.arange(w_, device="cuda") + n - w_
        rw = torch.ones(w_, dtype=torch.float64, device="cuda")
        if row_weight is not None:
            rw = row_weight[b].double()
        use = (rw != 0).repeat(G)
        for l in range(c.L):
            for h in range(H):
                q, sl = c.unit(b, l, h)
                q = torch.where(use[:, None] | (given is None), q, torch.zeros_like(q))
                old = c.acc[l, h, sl].double()
                hidden = old < 0
                vis = ~hidden[None].expand(G * w_, n).clone()
                if causal:
                    vis &= (torch.arange(n, device="cuda")[None] <= pos[:, None]).repeat(G, 1)
                w = Weights(q, c.k[l, h, sl], c.scale, vis)
                tag = f"b{b} l{l} h{h} n{n}"
                if given is None:
                    check(prob.lse[b, l, h * G:(h + 1) * G].reshape(-1), w.lse, w.lse_tol, f"lse {tag}")
                    pw, rel = w.p, w.rel
                else:
                    ls = given[b, l, h * G:(h + 1) * G].reshape(-1).double()
                    pw = torch.where((ls > -math.inf)[:, None], torch.exp(w.z - ls[:, None]),
                                     torch.zeros_like(w.z))
                    known = ls[torch.isfinite(ls)].abs()
                    big = float(known.max()) if known.numel() else 0.0
                    rel = w.rel + 4 * U * big * 1.45
                weigh = rw.repeat(G)[:, None] * torch.where(use[:, None], pw, torch.zeros_like(pw))
                want = torch.where(hidden, old, decay * old + weigh.sum(0))
                tol = (rel + (G * w_ + 4) * U) * weigh.abs().sum(0) + 4 * U * want.abs() + 1e-30
                check(acc[l, h, sl], want, tol, f"acc {tag}")
        a, e = c.starts[b] + n, c.starts[b + 1]
        assert torch.equal(acc[:, :, a:e], c.acc[:, :, a:e])
    return acc


@pytest.mark.parametrize("dtype,d", [(BF, 128), (BF, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("w,G,causal,holes,spare", [
    (1, 1, True, 0.0, 0), (1, 4, False, 0.1, 2), (7, 3, True, 0.1, 3), (16, 1, True, 0.0, 0),
    (33, 2, False, 0.2, 0), (64, 4, True, 0.0, 1), (300, 2, True, 0.1, 0),
])
def test_attn_weights(jacap, dtype, d, w, G, causal, holes, spare):
    """Windows shorter and longer than the sequences, rows before their start."""
    c = Case(ODD, w, dtype, d, G=G, holes=holes, spare=spare, L=2, seed=w + G)
    check_weights(jacap, c, causal, decay=0.5)


@pytest.mark.parametrize("dtype,w,lens,G", [
    (BF, 64, [40000, 5], 4), (BF, 2500, [2500, 1], 2), (BF, 1111, [2500, 1111, 700], 3),
    (F32, 32, [9000, 100], 2), (F32, 700, [700], 1), (BF, 1, [30000], 1),
])
def test_attn_weights_long(jacap, dtype, w, lens, G):
    """Several chunks, several row parts, whole prompts; decay 0 overwrites."""
    c = Case(lens, w, dtype, 128, H=1, G=G, seed=2, holes=0.01)
    check_weights(jacap, c, True, decay=0.0)


@pytest.mark.parametrize("dtype,d,w,G,causal", [
    (BF, 128, 64, 4, True), (BF, 128, 33, 3, False), (BF, 64, 256, 1, True), (BF, 64, 13, 5, True),
    (F32, 128, 32, 4, True), (F32, 64, 64, 4, True), (F32, 64, 11, 3, False)])
def test_attn_weights_in_long_stretches(jacap, dtype, d, w, G, causal):
    """Stretches of several blocks per workgroup, the last ones of each sequence cut short."""
    c = Case([40003, 0, 3, 30001, 257], w, dtype, d, H=2, G=G, L=2, holes=0.05, spare=2, seed=21)
    check_weights(jacap, c, causal, decay=0.75)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("causal", [False, True])
def test_attn_weights_of_accepted_rows(jacap, dtype, causal):
    """lse known; rows of weight 0 hold NaN and add nothing; a row of lse -inf too."""
    c = Case([900, 40, 0, 17], 21, dtype, 128, G=2, holes=0.1, seed=12)
    gen = torch.Generator(device="cuda").manual_seed(1)
    rw = (torch.rand((4, 21), generator=gen, device="cuda") < 0.4).float() * 0.5
    rw[0] = 0.0
    lse = 5.0 + torch.rand((4, 1, 4, 21), generator=gen, device="cuda")
    lse[1, 0, 2, 5] = -math.inf
    off = (rw == 0)
    c.q[off[:, None, None, :].expand(4, 1, 4, 21)] = math.nan
    lse[off[:, None, None, :].expand(4, 1, 4, 21)] = math.nan
    acc = check_weights(jacap, c, causal, given=lse, row_weight=rw)
    assert torch.equal(acc[:, :, :900], c.acc[:, :, :900])


@pytest.mark.parametrize("dtype", [BF, F32])
def test_attn_weights_ignores_hidden_keys(jacap, dtype):
    """NaN keys in empty slots and past the live lengths; a window that no token precedes."""
    c = Case([70, 5, 0], 24, dtype, 64, G=2, holes=0.3, spare=4, seed=13)
    hidden = c.acc < 0
    for b, n in enumerate(c.lens):
        hidden[:, :, c.starts[b] + n:c.starts[b + 1]] = True
    c.k[hidden] = math.nan
    acc = check_weights(jacap, c, True)
    assert torch.isfinite(acc).all()


# ---------------------------------------------------------------------------
# Lengths, devices, graphs, streams
# ---------------------------------------------------------------------------
def test_bad_lengths_are_flagged_and_taken_as_empty(jacap):
    for bad in (-1, 51, 2 ** 31 - 1):
        c = Case([40, 50], 2, BF, 64, spare=0, seed=3)
        c.live = torch.tensor([40, bad], dtype=torch.int32, device="cuda")
        p = jacap.AttentionParams(live_lens=c.live, accumulate=True)
        prob = jacap.prepare_attend(c.q, c.k, c.v, c.kd, c.vd, c.offsets, c.rows, p)
        acc = c.acc.clone()
        jacap.run_attend(prob, c.q, c.k, c.v, c.kd, c.vd, acc=acc)
        assert jacap.read_status(prob.ws) == jacap.FLAG_BAD_OFFSETS
        assert torch.equal(acc[:, :, 40:], c.acc[:, :, 40:])
        wp = jacap.prepare_attn_weights(c.q, c.k, c.offsets, c.rows, jacap.AttentionParams(live_lens=c.live))
        jacap.run_attn_weights(wp, c.q, c.k, acc)
        assert jacap.read_status(wp.ws) == jacap.FLAG_BAD_OFFSETS
        assert torch.equal(acc[:, :, 40:], c.acc[:, :, 40:])
        c.lens = [40, 0]
        c.live = None
        check_attend(c, prob, None, False, False)


@pytest.mark.parametrize("S", [1, 40])
def test_inconsistent_offsets(jacap, S):
    """Offsets that go back, or past the rows: flagged, the sequence taken as empty."""
    for offs in ([0, 40, 10, 50], [0, 40, 90, 200], [0, 40, -3, 5]):
        c = Case([40, 0, 0], S, BF, 64, seed=3)
        big = Case([40, 50, 0], S, BF, 64, seed=3)
        c.k, c.v, c.acc = big.k, big.v, big.acc
        c.offsets = torch.tensor(offs, dtype=torch.int32, device="cuda")
        p = jacap.AttentionParams()
        prob = jacap.prepare_attend(c.q, c.k, c.v, c.kd, c.vd, c.offsets, [40, 40, 10], p)
        jacap.run_attend(prob, c.q, c.k, c.v, c.kd, c.vd)
        assert jacap.read_status(prob.ws) == jacap.FLAG_BAD_OFFSETS
        c.lens = [40]
        check_attend(c, prob, None, False, False)


def test_deterministic(jacap):
    c = Case([9000, 77, 1300], 9, BF, 128, tree="tree", seed=3)
    a, acc_a = run_attend(jacap, c, False, True)
    b, acc_b = run_attend(jacap, c, False, True)
    for x, y in ((a.out, b.out), (a.lse, b.lse), (a.acc_draft, b.acc_draft), (acc_a, acc_b)):
        assert torch.equal(x, y)


def test_far_offsets(jacap):
    """A sequence behind 2^31 elements of the cache (token rows past 2^24)."""
    rows, d = (1 << 24) + 500, 128
    gen = torch.Generator(device="cuda").manual_seed(3)
    k = torch.zeros((1, 1, rows, d), dtype=BF, device="cuda")
    v = torch.zeros_like(k)
    lens, starts = [5, 300], [0, rows - 300, rows]
    for t in (k, v):
        for a, n in zip(starts, lens):
            t[0, 0, a:a + n] = torch.randn((n, d), generator=gen, device="cuda").to(BF)
    c = Case([5, 300], 2, BF, d, H=1, G=2, seed=21)
    c.k, c.v, c.starts, c.rows = k, v, starts, [rows - 300, 300]
    c.offsets = torch.tensor(starts, dtype=torch.int32, device="cuda")
    c.live = torch.tensor(lens, dtype=torch.int32, device="cuda")
    c.acc = torch.rand((1, 1, rows), generator=gen, device="cuda")
    prob, acc = run_attend(jacap, c, False, True)
    check_attend(c, prob, acc, False, True)
    check_weights(jacap, c, True)


@pytest.mark.parametrize("S,w", [(1, 8), (40, 200)])
def test_graph_replays(jacap, S, w):
    """One graph of attend (accumulating) and attn_weights, replayed with other
    lengths and data, eager work and synchronisation between the replays."""
    c = Case([600, 90, 0], S, BF, 128, holes=0.1, spare=200, tree="tree" if S > 1 else None, seed=31)
    cw = Case([600, 90, 0], w, BF, 128, spare=200, seed=32)
    p = jacap.AttentionParams(accumulate=True, live_lens=c.live, tree=c.tree)
    prob = jacap.prepare_attend(c.q, c.k, c.v, c.kd, c.vd, c.offsets, c.rows, p)
    wp = jacap.prepare_attn_weights(cw.q, c.k, c.offsets, c.rows, jacap.AttentionParams(live_lens=c.live))
    acc = c.acc.clone()

    def both():
        jacap.run_attend(prob, c.q, c.k, c.v, c.kd, c.vd, acc=acc)
        jacap.run_attn_weights(wp, cw.q, c.k, acc)

    both()
    torch.cuda.synchronize()
    g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            both()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for rep, lens in enumerate(([600, 90, 0], [700, 290, 200], [0, 1, 65], [800, 0, 33])):
        c.live.copy_(torch.tensor(lens, dtype=torch.int32))
        c.q.mul_(-1.0)
        acc.copy_(c.acc)
        both()
        torch.cuda.synchronize()
        want = [t.clone() for t in (prob.out, prob.lse, prob.acc_draft, wp.lse, acc)]
        for t in (prob.out, prob.lse, prob.acc_draft, wp.lse):
            t.fill_(-7.0)
        acc.copy_(c.acc)
        torch.cuda.synchronize()
        print(f"[graph] attend S{S}: replay {rep}", flush=True)
        g.replay()
        torch.cuda.synchronize()
        assert jacap.read_status(prob.ws) == 0 and jacap.read_status(wp.ws) == 0
        for x, y in zip((prob.out, prob.lse, prob.acc_draft, wp.lse, acc), want):
            assert torch.equal(x, y)
    del g


def test_two_streams(jacap):
    """Calls in flight on two streams, each with its own workspace."""
    cs = [Case([5000, 44], 1, BF, 128, seed=41), Case([3000, 7, 200], 30, BF, 64, tree="tree", seed=42)]
    want = []
    probs = []
    for c in cs:
        prob, acc = run_attend(jacap, c, False, True)
        want.append([t.clone() for t in (prob.out, prob.lse, prob.acc_draft, acc)])
        probs.append((prob, c.acc.clone()))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cs]
    for _ in range(3):
        for (prob, acc), c in zip(probs, cs):
            acc.copy_(c.acc)
            prob.out.fill_(-3.0)
        torch.cuda.synchronize()
        for (prob, acc), c, s in zip(probs, cs, streams):
            jacap.run_attend(prob, c.q, c.k, c.v, c.kd, c.vd, acc=acc, stream=s)
        torch.cuda.synchronize()
        for (prob, acc), w in zip(probs, want):
            for x, y in zip((prob.out, prob.lse, prob.acc_draft, acc), w):
                assert torch.equal(x, y)


def test_refusals(jacap):
    """What would read or write out of range is refused before anything is enqueued."""
    c = Case([40, 50], 3, BF, 64, seed=3)
    ok = jacap.AttentionParams()
    prep = lambda **kw: jacap.prepare_attend(*[kw.get(n, getattr(c, n)) for n in ("q", "k", "v", "kd", "vd")],
                                             kw.get("offsets", c.offsets), kw.get("rows", c.rows),
                                             kw.get("params", ok))
    prob = prep()
    for kw in (dict(v=c.v[:, :, 1:]), dict(v=c.v.float()), dict(kd=c.kd[:, :, :, :2]),
               dict(q=c.q[:1]), dict(rows=[40, 51]), dict(rows=[90]), dict(k=c.k.cpu()),
               dict(q=c.q[..., :32]), dict(offsets=c.offsets.long()), dict(vd=c.vd.cpu()),
               dict(params=jacap.AttentionParams(live_lens=torch.zeros(3, dtype=torch.int32, device="cuda"))),
               dict(params=jacap.AttentionParams(live_lens=torch.zeros(2, dtype=torch.int32))),
               dict(params=jacap.AttentionParams(tree=torch.zeros((2, 3), dtype=torch.int64, device="cuda"))),
               dict(params=jacap.AttentionParams(row_weight=torch.zeros((2, 4), device="cuda")))):
        with pytest.raises(ValueError):
            prep(**kw)
    for params in (jacap.AttentionParams(scale=0.0), jacap.AttentionParams(scale=math.inf),
                   jacap.AttentionParams(decay=1.5), jacap.AttentionParams(decay=math.nan)):
        with pytest.raises(jacap.JacapError):
            prep(params=params)
    with pytest.raises(ValueError):
        jacap.run_attend(prob, c.q, c.k.transpose(1, 2).contiguous().transpose(1, 2), c.v, c.kd, c.vd)
    with pytest.raises(ValueError):
        jacap.run_attend(prob, c.q, c.k, c.v, c.kd, c.vd, acc=c.acc[:, :, 1:])
    with pytest.raises(ValueError):
        jacap.run_attend(prep(params=jacap.AttentionParams(accumulate=True)), c.q, c.k, c.v, c.kd, c.vd)
    wp = jacap.prepare_attn_weights(c.q, c.k, c.offsets, c.rows, ok)
    with pytest.raises(ValueError):
        jacap.run_attn_weights(wp, c.q, c.k, c.acc.double())
    with pytest.raises(ValueError):
        jacap.run_attn_weights(wp, c.q, c.k, c.acc, lse=torch.zeros((2, 1, 8, 4), device="cuda"))
    torch.cuda.synchronize()

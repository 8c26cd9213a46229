"""Eviction by accumulated attention weight: the ranking, the copies, the empty
slots, and the whole loop (window weights, eviction, decoding with a tree,
refill of the listed slots) against a plain one."""

import math

import numpy as np
import pytest
import torch

from attention_ref import U, Weights, check, half_step, sees_tree
from oracle import jacap_oracle as jo

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def jacap():
    from paper_2609_08131_amd import jacap as j
    return j


def _cache(lens, L, H, d, dtype, seed, spare=0, holes=0.1):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows = [n + spare for n in lens]
    T = sum(rows)
    k = torch.randn((L, H, T, d), generator=gen, device="cuda").to(dtype)
    v = torch.randn((L, H, T, d), generator=gen, device="cuda").to(dtype)
    acc = torch.rand((L, H, T), generator=gen, device="cuda")
    acc = torch.where(torch.rand(acc.shape, generator=gen, device="cuda") < 0.3, torch.round(acc * 4) / 4, acc)
    acc[torch.rand(acc.shape, generator=gen, device="cuda") < holes] = -1.0
    acc[torch.rand(acc.shape, generator=gen, device="cuda") < 0.02] = math.nan
    offs = torch.tensor(np.concatenate([[0], np.cumsum(rows)]).astype(np.int32), device="cuda")
    live = torch.tensor(lens, dtype=torch.int32, device="cuda") if spare else None
    return k, v, acc, offs, rows, live


LENS = [0, 1, 17, 100, 257, 1000, 4100, 8192, 33000]


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.float32, 64)])
@pytest.mark.parametrize("budget,protect,spare", [(64, 0, 0), (200, 16, 7), (1, 0, 3), (3000, 40, 0),
                                                  (40000, 5, 0)])
def test_evict(jacap, dtype, d, budget, protect, spare):
    L, H = 2, 2
    k, v, acc, offs, rows, live = _cache(LENS, L, H, d, dtype, 3, spare)
    prob = jacap.prepare_evict_weighted(k, v, offs, rows, budget, protect, live)
    prob.k_out.fill_(5.0)
    prob.v_out.fill_(5.0)
    jacap.run_evict_weighted(prob, acc, k, v)
    slots = jacap.alloc_slots(prob, rows)
    marked = acc.clone()
    jacap.run_evict_weighted_slots(prob, marked, slots)
    torch.cuda.synchronize()
    expect = acc.clone()
    for b, n in enumerate(LENS):
        lo, kk = int(offs[b]), min(budget, n)
        for l in range(L):
            for h in range(H):
                a = acc[l, h, lo:lo + n]
                want = jo.select_top(a.cpu().numpy(), budget, protect_last=protect)
                idx = prob.idx[b, l, h].cpu().numpy()
                assert np.array_equal(idx[:kk], want) and (idx[kk:] == -1).all()
                at = torch.as_tensor(want, device="cuda").long()
                assert torch.equal(prob.k_out[b, l, h, :kk], k[l, h, lo + at])
                assert torch.equal(prob.v_out[b, l, h, :kk], v[l, h, lo + at])
                assert (prob.k_out[b, l, h, kk:] == 5.0).all() and (prob.v_out[b, l, h, kk:] == 5.0).all()
                torch.testing.assert_close(prob.acc_out[b, l, h, :kk], a[at], rtol=0, atol=0, equal_nan=True)
                assert (prob.acc_out[b, l, h, kk:] == -1.0).all()
                gone = np.setdiff1d(np.arange(n), want)
                got = slots[b, l, h].cpu().numpy()
                assert np.array_equal(got[:len(gone)], gone) and (got[len(gone):] == -1).all()
                expect[l, h, lo + torch.as_tensor(gone, device="cuda").long()] = -1.0
    torch.testing.assert_close(marked, expect, rtol=0, atol=0, equal_nan=True)


def test_budget_zero_and_no_tokens(jacap):
    k, v, acc, offs, rows, _ = _cache([30, 0, 5], 1, 2, 64, torch.bfloat16, 4)
    prob = jacap.prepare_evict_weighted(k, v, offs, rows, 0)
    jacap.run_evict_weighted(prob, acc, k, v)
    slots = jacap.alloc_slots(prob, rows)
    jacap.run_evict_weighted_slots(prob, acc, slots)
    assert torch.equal(slots[0, 0, 0], torch.arange(30, device="cuda", dtype=torch.int32))
    assert (acc == -1.0).all()
    k, v, acc, offs, rows, _ = _cache([0, 0], 1, 2, 64, torch.bfloat16, 5)
    prob = jacap.prepare_evict_weighted(k, v, offs, rows, 4)
    prob.acc_out.fill_(3.0)
    jacap.run_evict_weighted(prob, acc, k, v)
    assert (prob.idx == -1).all() and (prob.acc_out == -1.0).all()


def test_bad_lengths(jacap):
    k, v, acc, offs, rows, _ = _cache([30, 40], 1, 1, 64, torch.bfloat16, 4)
    live = torch.tensor([31, 40], dtype=torch.int32, device="cuda")
    prob = jacap.prepare_evict_weighted(k, v, offs, rows, 8, live_lens=live)
    jacap.run_evict_weighted(prob, acc, k, v)
    assert (prob.idx[0] == -1).all() and (prob.idx[1] >= 0).all()


def test_refusals(jacap):
    k, v, acc, offs, rows, _ = _cache([30, 40], 1, 2, 64, torch.bfloat16, 4)
    with pytest.raises(ValueError):
        jacap.prepare_evict_weighted(k, v[:, :, 1:], offs, rows, 8)
    with pytest.raises(ValueError):
        jacap.prepare_evict_weighted(k, v, offs, [30, 41], 8)
    with pytest.raises(ValueError):
        jacap.prepare_evict_weighted(k, v, offs, rows, 8, k_out=k.new_empty((2, 1, 2, 7, 64)))
    with pytest.raises(ValueError):
        jacap.prepare_evict_weighted(k, v, offs, rows, 8, acc_out=acc.new_empty((2, 1, 2, 9)))
    prob = jacap.prepare_evict_weighted(k, v, offs, rows, 8)
    with pytest.raises(ValueError):
        jacap.run_evict_weighted(prob, acc[:, :1], k, v)
    with pytest.raises(jacap.JacapError):
        jacap.run_evict_weighted_slots(prob, acc, torch.empty((2, 1, 2, 31), dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        jacap.run_evict_weighted_slots(prob, acc, torch.empty((2, 1, 1, 40), dtype=torch.int32, device="cuda"))


def test_graph_replays(jacap):
    k, v, acc, offs, rows, live = _cache([600, 90, 0, 2176], 2, 2, 64, torch.bfloat16, 6, spare=10)
    prob = jacap.prepare_evict_weighted(k, v, offs, rows, 200, 8, live)
    slots = jacap.alloc_slots(prob, rows)
    work = acc.clone()

    def both():
        jacap.run_evict_weighted(prob, work, k, v)
        jacap.run_evict_weighted_slots(prob, work, slots)

    both()
    torch.cuda.synchronize()
    g, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(g, stream=side):
            both()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for rep in range(3):
        acc = acc.flip(-1).contiguous()
        work.copy_(acc)
        for t in (prob.k_out, prob.v_out, prob.acc_out):
            t.fill_(-7.0)
        both()
        torch.cuda.synchronize()
        want = [t.clone() for t in (prob.idx, prob.k_out, prob.v_out, prob.acc_out, slots, work)]
        work.copy_(acc)
        prob.idx.fill_(-7)
        slots.fill_(-7)
        for t in (prob.k_out, prob.v_out, prob.acc_out):
            t.fill_(-7.0)
        torch.cuda.synchronize()
        print(f"[graph] evict_weighted: replay {rep}", flush=True)
        g.replay()
        torch.cuda.synchronize()
        for x, y in zip((prob.idx, prob.k_out, prob.v_out, prob.acc_out, slots, work), want):
            torch.testing.assert_close(x, y, rtol=0, atol=0, equal_nan=True)
    del g


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_decoding_loop(jacap, dtype):
    """A prompt's weights, eviction into a cache with room, verified trees whose
    accepted tokens fill the free slots, their rows' weights, and the next eviction in
    place: every step against the formulas on the same cache."""
    B, L, H, G, d, w, budget, room, S = 2, 1, 2, 2, 64, 16, 48, 12, 5
    cap = budget + room
    gen = torch.Generator(device="cuda").manual_seed(77)
    rnd = lambda *s: torch.randn(s, generator=gen, device="cuda").to(dtype)
    lens = [300, 129]
    k, v, acc, offs, rows, _ = _cache(lens, L, H, d, dtype, 70, holes=0.0)
    acc.zero_()
    q = rnd(B, L, H * G, w, d)
    wp = jacap.prepare_attn_weights(q, k, offs, rows, jacap.AttentionParams())
    jacap.run_attn_weights(wp, q, k, acc)
    # the retained cache: [L][H][B cap][d], every sequence with room behind its kept rows
    ck, cv = (torch.zeros((L, H, B * cap, d), dtype=dtype, device="cuda") for _ in range(2))
    cacc = torch.full((L, H, B * cap), -1.0, device="cuda")
    view = lambda t: t.view(L, H, B, cap, *t.shape[3:]).movedim(2, 0)[:, :, :, :budget]
    ev = jacap.prepare_evict_weighted(k, v, offs, rows, budget, k_out=view(ck), v_out=view(cv),
                                      acc_out=view(cacc))
    jacap.run_evict_weighted(ev, acc, k, v)
    for b, n in enumerate(lens):
        lo = int(offs[b])
        for h in range(H):
            at = torch.as_tensor(jo.select_top(acc[0, h, lo:lo + n].cpu().numpy(), budget), device="cuda").long()
            assert torch.equal(ck[0, h, b * cap:b * cap + budget], k[0, h, lo + at])
            assert torch.equal(cacc[0, h, b * cap:b * cap + budget], acc[0, h, lo + at])
    # decoding over it: all rows are in range, the free ones are empty slots
    coff = torch.tensor([0, cap, 2 * cap], dtype=torch.int32, device="cuda")
    crows = [cap, cap]
    tree = torch.tensor([[[1], [3], [5], [11], [19]]] * B, dtype=torch.int64, device="cuda")
    # nodes 0 - 1 - (3, 4) and 0 - 2; accepted: 0, 1, 3
    accepted = torch.tensor([[1, 1, 0, 1, 0]] * B, dtype=torch.float32, device="cuda")
    ev2 = jacap.prepare_evict_weighted(ck, cv, coff, crows, budget)
    slots = jacap.alloc_slots(ev2, crows)
    free = [[list(range(budget, cap)) for _ in range(H)] for _ in range(B)]
    for step in range(8):
        if len(free[0][0]) < 3:
            before = cacc.clone()
            jacap.run_evict_weighted_slots(ev2, cacc, slots)
            for b in range(B):
                for h in range(H):
                    a = before[0, h, b * cap:(b + 1) * cap].cpu().numpy()
                    gone = np.setdiff1d(np.arange(cap), jo.select_top(a, budget))
                    assert np.array_equal(slots[b, 0, h].cpu().numpy(), gone)
                    free[b][h] = gone.tolist()
        q, kd, vd = rnd(B, L, H * G, S, d), rnd(B, L, H, S, d), rnd(B, L, H, S, d)
        at = jacap.prepare_attend(q, ck, cv, kd, vd, coff, crows, jacap.AttentionParams(tree=tree))
        jacap.run_attend(at, q, ck, cv, kd, vd, acc=cacc)
        before = cacc.clone()
        add = jacap.prepare_attn_weights(q, ck, coff, crows, jacap.AttentionParams(
            causal=False, row_weight=accepted, decay=0.9))
        jacap.run_attn_weights(add, q, ck, cacc, lse=at.lse)
        h_ = half_step(dtype)
        for b in range(B):
            sl = slice(b * cap, (b + 1) * cap)
            for h in range(H):
                old = before[0, h, sl].double()
                vis = torch.cat([~(old < 0)[None].expand(G * S, cap),
                                 sees_tree(tree, S, b).cuda().repeat(G, 1)], 1)
                x = Weights(q[b, 0, h * G:(h + 1) * G].reshape(G * S, d),
                            torch.cat([ck[0, h, sl], kd[b, 0, h]]), d ** -0.5, vis)
                vv = torch.cat([cv[0, h, sl], vd[b, 0, h]]).double()
                out = x.p @ vv
                check(at.out[b, 0, h * G:(h + 1) * G].reshape(G * S, d), out,
                      (x.rel + h_ + (cap + S) * U) * (x.p @ vv.abs()) + h_ * out.abs(), f"out {step}")
                rw = accepted[b].double().repeat(G)[:, None]
                given = (rw * x.p).sum(0)[:cap]
                want = torch.where(old < 0, old, 0.9 * old + given)
                check(cacc[0, h, sl], want, (2 * x.rel + 64 * U) * given + 4 * U * want.abs(), f"acc {step}")
                # the accepted tokens take free slots
                for node in (0, 1, 3):
                    s = free[b][h].pop(0)
                    ck[0, h, b * cap + s] = kd[b, 0, h, node]
                    cv[0, h, b * cap + s] = vd[b, 0, h, node]
                    cacc[0, h, b * cap + s] = 0.0


@pytest.mark.parametrize("units,n,budget,live", [
    (2, 40000, 300, 0), (2, 40000, 300, 290), (2, 40000, 300, 300), (2, 40000, 300, 310),
    (2, 40000, 300, 9000), (2, 40000, 12000, 11000), (2, 33000, 32000, 20000),
    (1024, 9001, 700, 650), (1024, 9001, 300, 290), (1024, 9001, 300, 310)])
def test_slots_of_mostly_empty_caches(jacap, units, n, budget, live):
    """Units of which all but `live` tokens are empty slots already: fewer than the
    budget, as many, and more; in both launch shapes."""
    gen = torch.Generator().manual_seed(n + budget + live)
    off = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    k = torch.zeros((units, 1, n, 64), dtype=torch.bfloat16, device="cuda")
    p = jacap.prepare_evict_weighted(k, k, off, [n], budget=budget)
    acc = torch.full((units, 1, n), -1.0)
    for u in range(units):
        # values of 50 steps: many equal ones at the threshold
        acc[u, 0, torch.randperm(n, generator=gen)[:live]] = (
            torch.randint(0, 50, (live,), generator=gen).float())
    order = torch.argsort(-acc.double(), dim=-1, stable=True)
    want = acc.clone()
    want.scatter_(-1, order[..., budget:], -1.0)
    gone = torch.sort(order[..., budget:], dim=-1).values
    dev = acc.cuda()
    slots = torch.empty((1, units, 1, n - budget), dtype=torch.int32, device="cuda")
    jacap.run_evict_weighted_slots(p, dev, slots)
    assert torch.equal(dev.cpu(), want)
    assert torch.equal(slots.cpu()[0].long(), gone)

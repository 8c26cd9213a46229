"""Edges of jacap_attend and jacap_attn_weights by kernel: each against the formulas
in float64, with the bounds of attention_ref.py."""

import math

import pytest
import torch

from attention_ref import U
from test_gpu_attention import BF, F32, Case, check_attend, check_weights, run_attend

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def jacap():
    from paper_2609_08131_amd import jacap as j
    return j


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("S,G", [(16, 4), (33, 1), (32, 4), (65, 1), (63, 4), (100, 2), (90, 4)])
@pytest.mark.parametrize("holes", [0.0, 0.1])
def test_large_logits_of_many_rows(jacap, d, S, G, holes):
    """Logits of thousands under 33 to 64, 65 to 128 and more rows per KV head: steps of 32
    visible tokens and steps with hidden ones, the maxima raised again and again."""
    c = Case([500, 31, 3000], S, BF, d, H=1, G=G, holes=holes, seed=8, spread=400.0)
    print(f"[large] d{d} S{S} G{G} holes {holes}", flush=True)
    prob, acc = run_attend(jacap, c, holes > 0, True)
    check_attend(c, prob, acc, holes > 0, True)


@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("w,G,causal", [(8, 1, True), (16, 4, False), (64, 4, True), (300, 2, True)])
def test_large_logits_of_windows(jacap, dtype, d, w, G, causal):
    """The same in the log-sums of 2, 4 and 8 row tiles, and the sums behind them."""
    c = Case([500, 31, 3000], w, dtype, d, H=1, G=G, holes=0.05, seed=9, spread=400.0)
    print(f"[large] {dtype} d{d} w{w} G{G}", flush=True)
    check_weights(jacap, c, causal)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("w,G,given", [(13, 5, False), (64, 1, False), (31, 2, True), (64, 4, True),
                                       (100, 1, True), (300, 2, True), (300, 2, False)])
def test_infinite_keys_that_every_row_gives_nothing(jacap, dtype, w, G, given):
    """A visible token whose logits are -inf in every row receives 0, beside rows of
    weight 0 and the padding of the last row tiles; rows in LDS and staged."""
    c = Case([900, 40, 0, 17], w, dtype, 64, G=G, holes=0.1, spare=2, seed=17)
    c.q[..., 5] = c.q[..., 5].abs() + 0.25
    c.k[:, :, 7::13, 5] = -math.inf
    rw = lse = None
    if given:
        rw = (torch.arange(4 * w, device="cuda").view(4, w) % 3 == 0).float() * 0.5
        lse = 5.0 + torch.rand((4, 1, 2 * G, w), device="cuda")
    acc = check_weights(jacap, c, not given, given=lse, row_weight=rw, decay=0.5)
    assert torch.isfinite(acc).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("w,G", [(21, 2), (64, 1), (300, 2)])
@pytest.mark.parametrize("value", [math.nan, math.inf])
def test_rows_of_weight_zero_beside_non_finite_keys(jacap, dtype, w, G, value):
    """Sequences none of whose rows has a weight keep their accumulators, whatever their
    keys hold; the others' rows of weight 0 add nothing either."""
    c = Case([900, 40, 300], w, dtype, 128, G=G, holes=0.1, seed=18)
    c.k[:, :, 3:900:17] = value             # sequence 0, and one token of sequence 1
    c.k[:, :, 905] = value
    rw = torch.rand((3, w), device="cuda") + 0.5
    rw[0] = 0.0
    rw[1, ::2] = 0.0
    lse = 5.0 + torch.rand((3, 1, 2 * G, w), device="cuda")
    acc = check_weights(jacap, c, False, given=lse, row_weight=rw)
    assert torch.equal(acc[:, :, :900], c.acc[:, :, :900])
    assert torch.isfinite(acc[:, :, 940:]).all()


@pytest.mark.parametrize("dtype,T,w,G", [(BF, 132000, 131072, 4), (F32, 66000, 32768, 4), (BF, 300, 131072, 4),
                                         (F32, 130, 65536, 4)])
@pytest.mark.parametrize("weight", [0.9, 0.5])
def test_sums_of_many_nearly_equal_weights(jacap, dtype, T, w, G, weight):
    """Every row gives every token nearly the same weight (keys of 0, lse given): the
    bound does not grow with the rows. One row part, and many (short caches).

    A weight: lse log2(e) is rounded (u |lse|), and so is the exponent's argument; the
    exponential is within one unit, 2 u. At most 64 additions of a lane in fp32, then fp64
    sums rounded to fp32 at most twice, the 16 lanes' tree 4 u, the part's rounding and the
    last addition's: 2 |lse| u + 2 u + 64 u + 2 u + 4 u + 2 u < 76 u for |lse| < 1."""
    q = torch.zeros((1, 1, G, w, 64), dtype=dtype, device="cuda")
    k = torch.zeros((1, 1, T, 64), dtype=dtype, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(3)
    lse = -torch.log(weight + 0.001 * torch.rand((1, 1, G, w), generator=gen, device="cuda"))
    acc = torch.zeros((1, 1, T), device="cuda")
    prob = jacap.prepare_attn_weights(q, k, torch.tensor([0, T], dtype=torch.int32, device="cuda"), [T],
                                      jacap.AttentionParams(causal=False))
    jacap.run_attn_weights(prob, q, k, acc, lse=lse)
    want = float(torch.exp(-lse.double()).sum())
    worst = float((acc.double() - want).abs().max()) / want
    print(f"[sums] {dtype} T{T} R{G * w} weight {weight}: {worst:.3e}", flush=True)
    assert worst <= 76 * U


def _infinite_logits(c):
    """Tokens whose logits are +inf in the even heads' rows and -inf in the odd ones'."""
    c.q[..., 5] = c.q[..., 5].abs() + 0.25
    c.q[:, :, 1::2, :, 5] *= -1.0
    c.k[:, :, 7:300:97, 5] = math.inf
    return c


@pytest.mark.parametrize("dtype,d", [(BF, 64), (BF, 128), (F32, 64), (F32, 128)])
@pytest.mark.parametrize("S,G", [(1, 2), (5, 3), (20, 2), (40, 2), (130, 2)])
@pytest.mark.parametrize("lens", [[300, 3, 40], [4000, 900, 31]])
def test_infinite_logits(jacap, dtype, d, S, G, lens):
    """lse +inf and out NaN in the rows that have one, whose weights are 0 but for the
    infinite token's own, NaN; the other rows are as without that token."""
    c = _infinite_logits(Case(lens, S, dtype, d, H=2, G=G, holes=0.05, tree="tree" if S > 1 else None, seed=19))
    prob, acc = run_attend(jacap, c, True, True, decay=0.5)
    assert torch.isposinf(prob.lse).any() and torch.isfinite(prob.lse).any()
    check_attend(c, prob, acc, True, True, decay=0.5)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("w,G,causal", [(1, 2, True), (16, 2, False), (64, 4, True), (300, 2, True)])
@pytest.mark.parametrize("lens", [[300, 3, 40], [20000, 900, 31]])
def test_infinite_logits_of_windows(jacap, dtype, w, G, causal, lens):
    c = _infinite_logits(Case(lens, w, dtype, 64, H=2, G=G, holes=0.05, seed=20))
    check_weights(jacap, c, causal, decay=0.5)


@pytest.mark.parametrize("dtype,S,G", [(BF, 1, 2), (BF, 40, 2), (F32, 9, 2), (BF, 130, 4)])
@pytest.mark.parametrize("declared", [2 ** 31 - 1, 2 ** 31 - 1000, 10 ** 6])
def test_declared_length_far_above_the_tokens(jacap, dtype, S, G, declared):
    """max_seq_len is an upper bound, of any size: results as with the longest length."""
    c = Case([3000, 0, 700], S, dtype, 64, H=2, G=G, holes=0.05, seed=23)
    results = []
    for longest in (3000, declared):
        p = jacap.AttentionParams(accumulate=True)
        prob = jacap.prepare_attend(c.q, c.k, c.v, c.kd, c.vd, c.offsets, c.rows, p)
        wp = jacap.prepare_attn_weights(c.q, c.k, c.offsets, c.rows, p)
        for x, size in ((prob, jacap.attend_workspace_size), (wp, jacap.attn_weights_workspace_size)):
            x.batch.max_seq_len = longest
            x.ws = torch.empty(size(x.cfg, x.batch, x.attn), dtype=torch.uint8, device="cuda")
        acc = c.acc.clone()
        jacap.run_attend(prob, c.q, c.k, c.v, c.kd, c.vd, acc=acc)
        assert jacap.read_status(prob.ws) == 0
        check_attend(c, prob, acc, True, True)
        jacap.run_attn_weights(wp, c.q, c.k, acc)
        assert jacap.read_status(wp.ws) == 0
        results.append((wp.lse, acc))
    (lse, acc), (lse2, acc2) = results
    # (the chunks may differ: sums within their bounds, 3000 tokens, at most 520 rows)
    assert torch.equal(torch.isfinite(lse), torch.isfinite(lse2))
    f = torch.isfinite(lse)
    assert float((lse[f] - lse2[f]).abs().max()) <= 2 * 3004 * U + 8 * U * float(lse[f].abs().max())
    seen = acc >= 0
    assert torch.equal(acc < 0, acc2 < 0)
    assert float(((acc - acc2).abs() / acc.abs().clamp_min(1e-30))[seen].max()) <= 4 * (3004 + 524) * U


@pytest.mark.parametrize("S,G,spare", [(40, 1, 0), (40, 2, 300), (70, 4, 3)])
def test_many_rows_of_unequal_sequences(jacap, S, G, spare):
    """The pieces of a ragged batch: sequences of no, one, and several chunks, of any length
    and order; rows reserved behind them."""
    c = Case([0, 9000, 5, 257, 4000, 0, 256, 512, 1, 2300, 700, 6001], S, BF, 64, H=2, G=G, L=2, holes=0.05,
             spare=spare, tree="tree", seed=24)
    prob, acc = run_attend(jacap, c, True, True)
    check_attend(c, prob, acc, True, True)


def test_parameters_may_change_after_they_were_used(jacap):
    """A problem holds the tensors whose addresses its descriptors hold, whatever becomes of
    the parameters it was prepared with."""
    c = Case([50, 20], 3, BF, 64, H=2, G=2, spare=5, tree="tree", seed=25)
    p = jacap.AttentionParams(accumulate=True, live_lens=c.live, tree=c.tree,
                              row_weight=torch.ones((2, 3), device="cuda"))
    prob = jacap.prepare_attend(c.q, c.k, c.v, c.kd, c.vd, c.offsets, c.rows, p)
    wp = jacap.prepare_attn_weights(c.q, c.k, c.offsets, c.rows, p)
    live, tree, rw = p.live_lens.data_ptr(), p.tree.data_ptr(), p.row_weight.data_ptr()
    p.live_lens = p.tree = p.row_weight = None
    p.accumulate = False
    for x in (prob, wp):
        assert x.attn.live_lens == live == x.params.live_lens.data_ptr()
        assert x.attn.tree == tree == x.params.tree.data_ptr()
        assert x.attn.row_weight == rw == x.params.row_weight.data_ptr()
    with pytest.raises(ValueError):   # it still accumulates
        jacap.run_attend(prob, c.q, c.k, c.v, c.kd, c.vd)
    acc = c.acc.clone()
    jacap.run_attend(prob, c.q, c.k, c.v, c.kd, c.vd, acc=acc)
    check_attend(c, prob, acc, True, True)


def test_another_device_is_refused(jacap, monkeypatch):
    """A run with another device current, or on another device's stream, enqueues nothing."""
    c = Case([50, 20], 3, BF, 64, H=2, G=2, seed=26)
    p = jacap.AttentionParams(accumulate=True)
    prob = jacap.prepare_attend(c.q, c.k, c.v, c.kd, c.vd, c.offsets, c.rows, p)
    wp = jacap.prepare_attn_weights(c.q, c.k, c.offsets, c.rows, p)
    ev = jacap.prepare_evict_weighted(c.k, c.v, c.offsets, c.rows, 16)
    slots = jacap.alloc_slots(ev, c.rows)
    acc = c.acc.clone()
    prob.out.fill_(7.0)

    class Elsewhere:
        device_index, cuda_stream = 1, 0

    def refused(stream):
        for run in (lambda: jacap.run_attend(prob, c.q, c.k, c.v, c.kd, c.vd, acc=acc, stream=stream),
                    lambda: jacap.run_attn_weights(wp, c.q, c.k, acc, stream=stream),
                    lambda: jacap.run_evict_weighted(ev, acc, c.k, c.v, stream=stream),
                    lambda: jacap.run_evict_weighted_slots(ev, acc, slots, stream=stream)):
            with pytest.raises(ValueError):
                run()

    refused(Elsewhere)
    with monkeypatch.context() as m:
        m.setattr(torch.cuda, "current_device", lambda: 1)
        refused(None)
    torch.cuda.synchronize()
    assert torch.equal(acc, c.acc) and torch.equal(prob.out, torch.full_like(prob.out, 7.0))
    side = torch.cuda.Stream()
    jacap.run_attend(prob, c.q, c.k, c.v, c.kd, c.vd, acc=acc, stream=side)
    torch.cuda.synchronize()
    check_attend(c, prob, acc, True, True)


@pytest.mark.parametrize("S,G", [(1, 4), (9, 2), (40, 2)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_optional_outputs(jacap, S, G, accumulate):
    """lse and acc_draft may be null: the other outputs are the same."""
    c = Case([9000, 0, 300], S, BF, 64, H=2, G=G, holes=0.05, tree="tree" if S > 1 else None, seed=27)
    prob, acc = run_attend(jacap, c, True, accumulate, decay=0.5)
    want = prob.out.clone()
    prob.out.fill_(7.0)
    mine = c.acc.clone()
    jacap.attend(prob.cfg, prob.batch, prob.attn, c.q, c.k, c.v, c.kd, c.vd, prob.out, None, mine, None, prob.ws)
    assert torch.equal(prob.out, want)
    assert torch.equal(mine, acc if accumulate else c.acc)


@pytest.mark.parametrize("dtype,d", [(BF, 128), (F32, 64)])
@pytest.mark.parametrize("S", [1, 20, 40])
def test_strides_at_the_limit(jacap, dtype, d, S):
    """K and V rows 2^24 elements apart (offsets past 2^31 bytes), and heads that share them."""
    n, far = 37, 1 << 24
    c = Case([n], S, dtype, d, H=2, G=2, tree="tree" if S > 1 else None, seed=28)
    c.k, c.v = c.k[:, :1], c.v[:, :1]
    room = [torch.empty((n - 1) * far + d, dtype=dtype, device="cuda") for _ in range(2)]
    views = [t.as_strided((1, 2, n, d), (0, 0, far, 1)) for t in room]
    for view, x in zip(views, (c.k, c.v)):
        view[:, :1].copy_(x)
    c.k, c.v = views
    prob, acc = run_attend(jacap, c, True, True)
    check_attend(c, prob, acc, True, True)
    check_weights(jacap, c, True)


@pytest.mark.parametrize("S,w", [(1, 8), (40, 300)])
def test_accumulators_that_are_not_numbers(jacap, S, w):
    """A NaN entry hides nothing and stays NaN; decay 0 overwrites it."""
    c = Case([900, 31], S, BF, 64, H=2, G=4, holes=0.1, seed=29)
    c.acc[:, :, ::7] = math.nan
    prob, acc = run_attend(jacap, c, True, True, decay=0.5)
    check_attend(c, prob, acc, True, True, decay=0.5)
    prob, acc = run_attend(jacap, c, True, True, decay=0.0)
    odd = torch.isnan(c.acc)
    assert odd.any() and torch.isfinite(acc).all()
    c.acc = torch.where(odd, torch.ones_like(c.acc), c.acc)
    check_attend(c, prob, acc, True, True, decay=0.0)
    cw = Case([900, 31], w, BF, 64, H=2, G=4, holes=0.1, seed=29)
    cw.acc[:, :, ::7] = math.nan
    check_weights(jacap, cw, True, decay=0.5)


@pytest.mark.parametrize("S,G,w", [(1, 8, 64), (63, 4, 300), (20, 1, 2000)])
def test_runs_repeat_themselves(jacap, S, G, w):
    """The same bits from every run: joins of spans and chunks, sums of row parts."""
    c = Case([20000, 77, 1300], S, BF, 128, H=2, G=G, holes=0.02, tree="tree" if S > 1 else None, seed=30)
    cw = Case([20000, 77, 1300], w, BF, 128, H=2, G=G, holes=0.02, seed=30)
    wp = jacap.prepare_attn_weights(cw.q, cw.k, cw.offsets, cw.rows, jacap.AttentionParams())
    first = None
    for _ in range(4):
        prob, acc = run_attend(jacap, c, True, True)
        weigh = cw.acc.clone()
        jacap.run_attn_weights(wp, cw.q, cw.k, weigh)
        got = [t.clone() for t in (prob.out, prob.lse, prob.acc_draft, acc, wp.lse, weigh)]
        first = first or got
        assert all(torch.equal(x, y) for x, y in zip(first, got))

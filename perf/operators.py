"""Performance cases of the attention operators around an evicted cache:

* attend: attention of one new token, or of a tree of drafted tokens, over the
  cache (jacap.prepare_attend / run_attend), adding the cached tokens'
  attention weights to an accumulator;
* attn_weights: the accumulated attention weights of an observation window, of
  a whole prompt, or of the accepted rows of a verified tree
  (jacap.prepare_attn_weights / run_attn_weights);
* evict: eviction by the accumulated weights, compacting the cache or listing
  the slots to refill (jacap.prepare_evict_weighted / run_evict_weighted /
  run_evict_weighted_slots).

With own = False, run() computes the same outputs in elementary torch
operations in 32 bits.
"""

import math

import torch

own = False

DEFAULTS = {
    "op": "attend",         # attend | weights | evict | slots
    "layers": 1, "kv_heads": 8, "group": 4, "head_dim": 128, "dtype": "bf16",
    "lens": "",             # live sequence lengths, comma separated, or
    "seqs": 1, "lo": 0, "hi": 0, "lens_seed": 0,   # that many, drawn from lo..hi
    "spare": 0,             # > 0: every sequence owns (longest + spare) rows of the cache
    "rows": 1,              # query rows per head: drafted tokens, or the window
    "tree": False,          # attend: a random tree (else a chain)
    "acc": False,           # attend: accumulate the weights
    "decay": 0.0,           # what an accumulator's entry is multiplied by before the addition
    "holes": 0.0,           # fraction of empty slots (accumulator below zero)
    "causal": True,         # weights: the rows are the sequence's last positions
    "given": False,         # weights: the rows' lse is known, some rows have weight zero
    "budget": 512, "protect": 0,
    "token_major": False,   # K and V stored [L][T][H][d] and passed as views
}


def listed():
    return [
        # One decoded token of one layer over a short cache: all latency.
        {"name": "token_512", "op": "attend", "lens": "512"},
        # One decoded token of 16 ragged sequences (continuous batching), one
        # layer, adding to the accumulators that the next eviction ranks by.
        {"name": "token_ragged_16", "op": "attend", "seqs": 16, "lo": 4096, "hi": 32768,
         "lens_seed": 4, "acc": True, "decay": 1.0},
        # One decoded token over the longest context, refilled slots among it.
        {"name": "token_128k", "op": "attend", "lens": "131072", "acc": True, "holes": 0.01},
        # A tree of 63 drafted tokens verified over four caches kept at 16384
        # rows, each with room for the next 128.
        {"name": "tree_63_16k", "op": "attend", "lens": "16384,16383,16450,12001", "spare": 128,
         "rows": 63, "tree": True},
        # A small fp32 model's tree over very unequal, odd lengths.
        {"name": "tree_7_odd_fp32", "op": "attend", "lens": "0,1,17,255,256,257,1000,8193",
         "dtype": "fp32", "group": 2, "kv_heads": 4, "head_dim": 64, "rows": 7, "tree": True,
         "acc": True, "holes": 0.05},
        # One layer of an 8B model after an 8K prefill: the window's weights.
        {"name": "window_8k", "op": "weights", "lens": "8192", "rows": 32},
        # Four layers at 128K (one pipeline stage's group).
        {"name": "window_128k", "op": "weights", "layers": 4, "lens": "131072", "rows": 64},
        # Every query of an 8K prompt (weights accumulated over the prefill).
        {"name": "prompt_8k", "op": "weights", "lens": "8192", "rows": 8192},
        # The accepted rows of a verified tree of 31 tokens, fp32, lse known.
        {"name": "accepted_fp32", "op": "weights", "lens": "4096,1023,5001", "rows": 31,
         "dtype": "fp32", "group": 2, "head_dim": 64, "causal": False, "given": True,
         "decay": 0.98, "holes": 0.02},
        # A whole 8B model after a 32K prefill, evicted to 512 rows.
        {"name": "evict_32k", "op": "evict", "layers": 32, "lens": "32768", "budget": 512},
        # 16 decoding sequences at a reserved budget of 2048: 128 slots each.
        {"name": "slots_2k", "op": "slots", "layers": 32, "lens": ",".join(["2176"] * 16),
         "budget": 2048, "protect": 64},
    ]


# The most token entries (tokens x layers x KV heads) of a drawn case by kind.
_MOST = {"attend": 2_000_000, "weights": 2_000_000, "evict": 8_000_000, "slots": 8_000_000}


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "weights", "weights", "evict", "slots"])
    c = {"op": op, "head_dim": rng.choice([64, 128, 128]), "group": rng.choice([1, 2, 4, 4, 7, 8]),
         "kv_heads": rng.choice([1, 2, 4, 8]), "dtype": rng.choice(["bf16", "bf16", "bf16", "fp32"]),
         "token_major": rng.random() < 0.3, "layers": rng.choice([1, 1, 2, 3])}
    if rng.random() < 0.5:
        c["lens"] = str(_log_int(rng, 100, 131072))
    else:
        hi = _log_int(rng, 300, 32768)
        c.update(seqs=rng.randint(2, 16), lo=rng.randint(0, hi // 2), hi=hi,
                 lens_seed=rng.randrange(1 << 20))
    if rng.random() < 0.3:
        c["spare"] = rng.randint(1, 300)
    c["holes"] = rng.choice([0.0, 0.0, 0.02, 0.3])
    if op == "attend":
        c["rows"] = rng.choice([1, 1, 2, 5, rng.randint(2, 64), rng.randint(2, 64)])
        c["tree"] = c["rows"] > 1 and rng.random() < 0.7
        c["acc"] = rng.random() < 0.6
        c["decay"] = rng.choice([0.0, 0.9, 1.0])
    elif op == "weights":
        c["rows"] = rng.choice([16, 32, 64, rng.randint(1, 64), _log_int(rng, 64, 2048)])
        c["given"] = rng.random() < 0.3
        c["causal"] = not c["given"] and rng.random() < 0.8
        c["decay"] = rng.choice([0.0, 0.9, 1.0])
    else:
        c["layers"] = rng.randint(1, 32)
        c["budget"] = _log_int(rng, 16, 4096)
        c["protect"] = rng.choice([0, 0, 16, 64])
    lens = _lens(_full(c))
    entries = max(1, sum(lens)) * c["kv_heads"]
    c["layers"] = max(1, min(c["layers"], _MOST[op] // entries))
    if op == "weights":   # no more logits than the listed whole prompt
        most = (4 * 8 * 8192 * 8192 // 2) // (16 if c["dtype"] == "fp32" else 1)
        per_row = entries * c["layers"] * c["group"]
        c["rows"] = max(1, min(c["rows"], most // per_row))
    return c


def _full(case):
    c = dict(DEFAULTS)
    c.update({k: v for k, v in case.items() if k != "name"})
    return c


def _lens(c):
    if c["lens"]:
        return [int(x) for x in c["lens"].split(",")]
    gen = torch.Generator().manual_seed(int(c["lens_seed"]))
    return [int(x) for x in torch.randint(c["lo"], c["hi"] + 1, (c["seqs"],), generator=gen)]


def _starts(c, lens):
    """First cache row of every sequence, and the rows in all."""
    if c["spare"]:
        cap = max(lens) + c["spare"]
        return [b * cap for b in range(len(lens) + 1)]
    out = [0]
    for n in lens:
        out.append(out[-1] + n)
    return out


def _tree_words(rows, seqs, gen):
    """Ancestor masks of random trees: int64 [seqs][rows][words], bit j of a
    row set where the row sees drafted token j (its ancestors and itself)."""
    words = (rows + 63) // 64
    sees = torch.zeros((seqs, rows, rows), dtype=torch.bool)
    for b in range(seqs):
        for j in range(rows):
            p = int(torch.randint(-1, j, (1,), generator=gen)) if j else -1
            if p >= 0:
                sees[b, j] = sees[b, p]
            sees[b, j, j] = True
    bits = torch.zeros((seqs, rows, words * 64), dtype=torch.int64)
    bits[:, :, :rows] = sees.long()
    shift = torch.arange(64, dtype=torch.int64)
    return (bits.view(seqs, rows, words, 64) << shift).sum(-1)


class _State:
    pass


def _inputs(c, seed):
    """The cache, the query rows, the drafted tokens' keys and values, the
    accumulators: keys and queries share a centre, a few channels are outliers,
    token 0 is a sink, and some tokens are heavy hitters."""
    dev = "cuda"
    lens = _lens(c)
    starts = _starts(c, lens)
    L, H, G, d, S, B = c["layers"], c["kv_heads"], c["group"], c["head_dim"], c["rows"], len(lens)
    T = starts[-1]
    dt = torch.float32 if c["dtype"] == "fp32" else torch.bfloat16
    gen = torch.Generator(device=dev).manual_seed(int(seed) & ((1 << 62) - 1))
    host = torch.Generator().manual_seed(int(seed) & ((1 << 62) - 1))
    s = _State()
    s.case, s.lens, s.starts = c, lens, starts
    shape = (L, T, H, d) if c["token_major"] else (L, H, T, d)
    s.k, s.v = torch.zeros(shape, dtype=dt, device=dev), torch.zeros(shape, dtype=dt, device=dev)
    if c["token_major"]:
        s.k, s.v = s.k.transpose(1, 2), s.v.transpose(1, 2)
    centre = torch.randn((L, H, d), generator=gen, device=dev)
    attends = c["op"] in ("attend", "weights")
    for l in range(L):
        scale = torch.ones((2, H, 1, d), device=dev)
        ch = torch.rand((2, H, 1, d), generator=gen, device=dev).argsort(-1)[..., :4]
        scale.scatter_(3, ch, 6.0)
        for b, n in enumerate(lens):
            if n == 0:
                continue
            t = starts[b]
            k = torch.randn((H, n, d), generator=gen, device=dev)
            k *= scale[0]
            heavy = max(0, min(32, n - 1))
            if heavy:
                part = (n - 1) / heavy      # distinct positions in 1 .. n-1
                at = torch.rand((heavy,), generator=gen, device=dev) * math.floor(part)
                base = torch.tensor([1 + math.floor(i * part) for i in range(heavy)], device=dev)
                pos = (base + at.long()).clamp_(1, n - 1)
                k[:, pos] = 0.8 * centre[l][:, None] + 0.1 * torch.randn((H, heavy, d), generator=gen,
                                                                        device=dev)
            k[:, 0] = 1.2 * centre[l]
            s.k[l, :, t:t + n] = k.to(dt)
            v = torch.randn((H, n, d), generator=gen, device=dev)
            v *= scale[1]
            s.v[l, :, t:t + n] = v.to(dt)
    if attends:
        s.q = torch.empty((B, L, H * G, S, d), dtype=dt, device=dev)
        for b in range(B):
            q = torch.randn((L, H, G, S, d), generator=gen, device=dev) + centre[:, :, None, None]
            s.q[b] = q.reshape(L, H * G, S, d).to(dt)
    s.tree = None
    if c["op"] == "attend":
        s.kd = (torch.randn((B, L, H, S, d), generator=gen, device=dev) + 0.3 * centre[:, :, None]).to(dt)
        s.vd = torch.randn((B, L, H, S, d), generator=gen, device=dev).to(dt)
        if c["tree"]:
            s.tree = _tree_words(S, B, host).to(dev)
    # weights accumulated so far: a long tail over the tokens, empty slots below zero
    s.acc = None
    if c["op"] != "attend" or c["acc"] or c["holes"] > 0:
        s.acc = torch.rand((L, H, T), generator=gen, device=dev).pow_(8.0)
        if c["holes"] > 0:
            s.acc[torch.rand((L, H, T), generator=gen, device=dev) < c["holes"]] = -1.0
        if c["spare"]:
            for b, n in enumerate(lens):
                s.acc[:, :, starts[b] + n:starts[b + 1]] = -1.0
    s.row_weight = s.lse = None
    if c["given"]:
        s.row_weight = (torch.rand((B, S), generator=gen, device=dev) < 0.4).float()
        # what the verifying attention left: every row's log of its sum of exponentials
        s.lse = 9.0 + torch.rand((B, L, H * G, S), generator=gen, device=dev)
    s.offsets = torch.tensor(starts, dtype=torch.int32, device=dev)
    s.live = torch.tensor(lens, dtype=torch.int32, device=dev) if c["spare"] else None
    s.scale = 1.0 / math.sqrt(d)
    return s


def _restores(c):
    """Whether a pass reads the accumulators that it writes: it adds to them, or evicts by
    them (and marks what it evicts as empty slots)."""
    return c["op"] == "slots" or c["decay"] > 0 and (c["acc"] or c["op"] == "weights")


def _row_counts(s):
    return [b - a for a, b in zip(s.starts, s.starts[1:])]


def prepare(case, seed):
    s = _inputs(_full(case), seed)
    c = s.case
    B, L, H, d = len(s.lens), c["layers"], c["kv_heads"], c["head_dim"]
    dev = "cuda"
    if _restores(c):
        s.acc0 = s.acc.clone()
    cap = max(max(_row_counts(s)), 1)
    if own:
        from paper_2609_08131_amd import jacap
        if c["op"] == "attend":
            s.prob = jacap.prepare_attend(
                s.q, s.k, s.v, s.kd, s.vd, s.offsets, _row_counts(s),
                jacap.AttentionParams(scale=s.scale, accumulate=c["acc"], decay=c["decay"],
                                      live_lens=s.live, tree=s.tree))
        elif c["op"] == "weights":
            s.prob = jacap.prepare_attn_weights(
                s.q, s.k, s.offsets, _row_counts(s),
                jacap.AttentionParams(scale=s.scale, decay=c["decay"], causal=c["causal"],
                                      live_lens=s.live, row_weight=s.row_weight))
        else:
            s.prob = jacap.prepare_evict_weighted(
                s.k, s.v, s.offsets, _row_counts(s), budget=c["budget"],
                protect_last=c["protect"], live_lens=s.live)
            s.prob.k_out.zero_()
            s.prob.v_out.zero_()
            s.slots = torch.empty((B, L, H, max(1, cap - c["budget"])), dtype=torch.int32, device=dev)
    elif c["op"] == "slots":
        s.slots = torch.empty((B, L, H, max(1, cap - c["budget"])), dtype=torch.int32, device=dev)
    return s


def run(s):
    c = s.case
    if _restores(c):
        s.acc.copy_(s.acc0)   # one pass starts from the same accumulators as the last did
    return (_run_own if own else _run_plain)(s)


def _words(x):
    return x.view(torch.int32 if x.dtype == torch.float32 else torch.int16)


def _run_own(s):
    from paper_2609_08131_amd import jacap
    c, p = s.case, s.prob
    if c["op"] == "attend":
        jacap.run_attend(p, s.q, s.k, s.v, s.kd, s.vd, acc=s.acc)
        out = {"out": p.out, "lse": p.lse}
        if c["acc"]:
            out.update(acc=s.acc, acc_draft=p.acc_draft)
        return out
    if c["op"] == "weights":
        jacap.run_attn_weights(p, s.q, s.k, s.acc, lse=s.lse)
        return {"acc": s.acc} if c["given"] else {"acc": s.acc, "lse": p.lse}
    if c["op"] == "evict":
        jacap.run_evict_weighted(p, s.acc, s.k, s.v)
        return {"idx": p.idx, "k": _words(p.k_out), "v": _words(p.v_out), "acc": p.acc_out}
    jacap.run_evict_weighted_slots(p, s.acc, s.slots)
    return {"slots": s.slots, "acc": s.acc}


# ---------------------------------------------------------------------------
# Plain form: elementary torch operations, 32 bits
# ---------------------------------------------------------------------------
def _tree_sees(s, b):
    """bool [rows][rows]: which drafted tokens a row of sequence b sees."""
    S = s.case["rows"]
    j = torch.arange(S, device="cuda")
    if s.tree is None:
        return j[None, :] <= j[:, None]
    return (s.tree[b][:, j // 64] >> (j % 64) & 1) == 1


def _plain_attend(s):
    c = s.case
    L, H, G, S, d, B = c["layers"], c["kv_heads"], c["group"], c["rows"], c["head_dim"], len(s.lens)
    out = torch.empty_like(s.q)
    lse = torch.empty((B, L, H * G, S), dtype=torch.float32, device="cuda")
    acc_draft = torch.empty((B, L, H, S), dtype=torch.float32, device="cuda")
    for b, n in enumerate(s.lens):
        t = s.starts[b]
        sees = _tree_sees(s, b).repeat(G, 1)                       # [G S][S]
        for l in range(L):
            q = s.q[b, l].float().view(H, G * S, d)
            k, v = s.k[l, :, t:t + n].float(), s.v[l, :, t:t + n].float()
            kd, vd = s.kd[b, l].float(), s.vd[b, l].float()
            z = torch.matmul(q, k.transpose(1, 2).contiguous()) * s.scale
            zd = torch.matmul(q, kd.transpose(1, 2).contiguous()) * s.scale
            zd = zd.masked_fill(~sees, float("-inf"))
            if s.acc is not None:
                z = z.masked_fill((s.acc[l, :, t:t + n] < 0)[:, None], float("-inf"))
            z = torch.cat([z, zd], -1)
            top = z.amax(-1, keepdim=True)
            e = torch.exp(z - top)
            total = e.sum(-1, keepdim=True)
            p = e / total
            o = torch.matmul(p, torch.cat([v, vd], 1))
            out[b, l] = o.view(H * G, S, d).to(out.dtype)
            lse[b, l] = (top + torch.log(total)).view(H * G, S)
            if c["acc"]:
                w = p.sum(1)
                old = s.acc[l, :, t:t + n]
                kept = old * c["decay"] if c["decay"] > 0 else torch.zeros_like(old)
                s.acc[l, :, t:t + n] = torch.where(old < 0, old, kept + w[:, :n])
                acc_draft[b, l] = w[:, n:]
    res = {"out": out, "lse": lse}
    if c["acc"]:
        res.update(acc=s.acc, acc_draft=acc_draft)
    return res


def _plain_weights(s):
    c = s.case
    L, H, G, w, d, B = c["layers"], c["kv_heads"], c["group"], c["rows"], c["head_dim"], len(s.lens)
    lse = s.lse if c["given"] else torch.empty((B, L, H * G, w), dtype=torch.float32, device="cuda")
    for b, n in enumerate(s.lens):
        t = s.starts[b]
        # positions of the rows; rows before the sequence's start see nothing
        at = torch.arange(w, device="cuda") + (n - w)
        i = torch.arange(n, device="cuda")
        step = max(1, min(w, (1 << 27) // max(1, n * G)))
        for l in range(L):
            for h in range(H):
                k = s.k[l, h, t:t + n].float()
                kt = k.t().contiguous()
                old = s.acc[l, h, t:t + n]
                hidden = old < 0
                total = torch.zeros((n,), dtype=torch.float32, device="cuda")
                for p0 in range(0, w, step):
                    p1 = min(w, p0 + step)
                    q = s.q[b, l, h * G:(h + 1) * G, p0:p1].float()
                    z = torch.matmul(q.reshape(-1, d), kt).view(G, p1 - p0, n) * s.scale
                    z = z.masked_fill(hidden, float("-inf"))
                    if c["causal"]:
                        z = z.masked_fill(i[None, :] > at[p0:p1, None], float("-inf"))
                    if c["given"]:
                        ls = lse[b, l, h * G:(h + 1) * G, p0:p1]
                    elif n:
                        top = z.amax(-1)
                        ref = torch.where(top > float("-inf"), top, torch.zeros_like(top))
                        ls = ref + torch.log(torch.exp(z - ref[..., None]).sum(-1))
                        lse[b, l, h * G:(h + 1) * G, p0:p1] = ls
                    else:
                        lse[b, l, h * G:(h + 1) * G, p0:p1] = float("-inf")
                        continue
                    use = ls > float("-inf")
                    p = torch.exp(z - torch.where(use, ls, torch.zeros_like(ls))[..., None])
                    if s.row_weight is not None:
                        p = p * s.row_weight[b, p0:p1][None, :, None]
                    total += p.sum((0, 1))
                kept = old * c["decay"] if c["decay"] > 0 else torch.zeros_like(old)
                s.acc[l, h, t:t + n] = torch.where(hidden, old, kept + total)
    return {"acc": s.acc} if c["given"] else {"acc": s.acc, "lse": lse}


def _plain_ranked(s, b):
    """Positions of sequence b's kept tokens, bool [L][H][n]: the protected
    tail, and of the rest the largest weights, ties to the lower position."""
    c = s.case
    n, t = s.lens[b], s.starts[b]
    kk = min(c["budget"], n)
    tail = min(c["protect"], kk)
    a = s.acc[:, :, t:t + n]
    keep = torch.zeros(a.shape, dtype=torch.bool, device="cuda")
    keep[:, :, n - tail:] = True
    order = torch.sort(a[:, :, :n - tail], dim=-1, descending=True, stable=True).indices
    keep.scatter_(2, order[:, :, :kk - tail], True)
    return keep


def _plain_evict(s):
    c = s.case
    L, H, d, B, bud = c["layers"], c["kv_heads"], c["head_dim"], len(s.lens), c["budget"]
    idx = torch.full((B, L, H, bud), -1, dtype=torch.int32, device="cuda")
    k_out = torch.zeros((B, L, H, bud, d), dtype=s.k.dtype, device="cuda")
    v_out = torch.zeros_like(k_out)
    acc_out = torch.full((B, L, H, bud), -1.0, dtype=torch.float32, device="cuda")
    for b, n in enumerate(s.lens):
        kk, t = min(bud, n), s.starts[b]
        if kk == 0:
            continue
        at = _plain_ranked(s, b).nonzero()[:, 2].view(L, H, kk)
        idx[b, :, :, :kk] = at.int()
        rows = at[..., None].expand(L, H, kk, d)
        k_out[b, :, :, :kk] = s.k[:, :, t:t + n].gather(2, rows)
        v_out[b, :, :, :kk] = s.v[:, :, t:t + n].gather(2, rows)
        acc_out[b, :, :, :kk] = s.acc[:, :, t:t + n].gather(2, at)
    return {"idx": idx, "k": _words(k_out), "v": _words(v_out), "acc": acc_out}


def _plain_slots(s):
    c = s.case
    s.slots.fill_(-1)
    for b, n in enumerate(s.lens):
        gone = n - min(c["budget"], n)
        if gone == 0:
            continue
        t = s.starts[b]
        drop = ~_plain_ranked(s, b)
        at = drop.nonzero()[:, 2].view(c["layers"], c["kv_heads"], gone)
        s.slots[b, :, :, :gone] = at.int()
        a = s.acc[:, :, t:t + n]
        s.acc[:, :, t:t + n] = torch.where(drop, torch.full_like(a, -1.0), a)
    return {"slots": s.slots, "acc": s.acc}


def _run_plain(s):
    op = s.case["op"]
    if op == "attend":
        return _plain_attend(s)
    if op == "weights":
        return _plain_weights(s)
    return _plain_evict(s) if op == "evict" else _plain_slots(s)


def work(case):
    c = _full(case)
    lens = _lens(c)
    d, size, G, S = c["head_dim"], 4 if c["dtype"] == "fp32" else 2, c["group"], c["rows"]
    lh, B = c["layers"] * c["kv_heads"], len(lens)
    entries = sum(lens) * lh
    rows = B * lh * G * S
    live = entries * (1.0 - c["holes"])
    if c["op"] == "attend":
        nbytes = 2 * live * d * size + 2 * rows * d * size + rows * 4 + 2 * B * lh * S * d * size
        flops = 4 * d * G * S * live + 4 * d * rows * S // 2
        if c["acc"]:
            nbytes += (8 if c["decay"] > 0 else 4) * entries + 4 * B * lh * S
        elif c["holes"] > 0:
            nbytes += 4 * entries
        return {"bytes": int(nbytes), "flops": int(flops)}
    if c["op"] == "weights":
        nbytes = live * d * size + rows * d * size + rows * 4
        nbytes += (8 if c["decay"] > 0 else 4) * entries
        if c["causal"]:
            pairs = sum(sum(max(0, n - S + p + 1) for p in range(S)) for n in lens) * lh * G
            pairs *= 1.0 - c["holes"]
        else:
            pairs = live * G * S * (0.4 if c["given"] else 1.0)
        return {"bytes": int(nbytes), "flops": int(2 * d * pairs)}
    kept = sum(min(c["budget"], n) for n in lens) * lh
    units = B * lh
    if c["op"] == "evict":
        return {"bytes": int(4 * entries + 4 * kept * d * size + 8 * units * c["budget"] + 4 * kept),
                "flops": int(entries)}
    gone = entries - kept
    cap = max(1, max(_row_counts_of(c, lens)) - c["budget"])
    return {"bytes": int(4 * entries + 4 * gone + 4 * units * cap), "flops": int(entries)}


def _row_counts_of(c, lens):
    st = _starts(c, lens)
    return [b - a for a, b in zip(st, st[1:])]


# ---------------------------------------------------------------------------
# The definitions in 64 bits
# ---------------------------------------------------------------------------
def _exact_attend(s):
    c = s.case
    L, H, G, S, d, B = c["layers"], c["kv_heads"], c["group"], c["rows"], c["head_dim"], len(s.lens)
    f8 = dict(dtype=torch.float64, device="cuda")
    out = torch.zeros((B, L, H * G, S, d), **f8)
    lse = torch.zeros((B, L, H * G, S), **f8)
    acc_draft = torch.zeros((B, L, H, S), **f8)
    acc = s.acc.double() if s.acc is not None else None
    allowed = torch.zeros((B, S, S), dtype=torch.bool)
    if s.tree is None:
        allowed |= torch.tril(torch.ones((S, S), dtype=torch.bool))
    else:
        words = s.tree.cpu().tolist()
        for b in range(B):
            for r in range(S):
                for j in range(S):
                    allowed[b, r, j] = bool((words[b][r][j >> 6] >> (j & 63)) & 1)
    allowed = allowed.cuda()
    for b, n in enumerate(s.lens):
        lo = s.starts[b]
        for l in range(L):
            for h in range(H):
                keys = torch.cat([s.k[l, h, lo:lo + n], s.kd[b, l, h]]).double()
                vals = torch.cat([s.v[l, h, lo:lo + n], s.vd[b, l, h]]).double()
                vis = torch.ones((S, n + S), dtype=torch.bool, device="cuda")
                vis[:, n:] = allowed[b]
                if acc is not None:
                    vis[:, :n] &= ~(s.acc[l, h, lo:lo + n] < 0)
                given = torch.zeros((n + S,), **f8)
                for g in range(G):
                    z = (s.q[b, l, h * G + g].double() @ keys.t().contiguous()) / math.sqrt(d)
                    z[~vis] = -math.inf
                    ls = torch.logsumexp(z, 1)
                    p = torch.exp(z - ls[:, None])
                    out[b, l, h * G + g] = p @ vals
                    lse[b, l, h * G + g] = ls
                    given += p.sum(0)
                acc_draft[b, l, h] = given[n:]
                if c["acc"]:
                    a = acc[l, h, lo:lo + n]
                    live = a >= 0
                    a[live] = c["decay"] * a[live] + given[:n][live]
    res = {"out": out, "lse": lse}
    if c["acc"]:
        res.update(acc=acc, acc_draft=acc_draft)
    return res


def _exact_weights(s):
    c = s.case
    L, H, G, w, d, B = c["layers"], c["kv_heads"], c["group"], c["rows"], c["head_dim"], len(s.lens)
    acc = s.acc.double()
    lse = torch.full((B, L, H * G, w), -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(s.lens):
        if n == 0:
            continue
        lo = s.starts[b]
        for l in range(L):
            for h in range(H):
                keys = s.k[l, h, lo:lo + n].double().t().contiguous()
                a = acc[l, h, lo:lo + n]
                live = a >= 0
                got = torch.zeros((n,), dtype=torch.float64, device="cuda")
                size = max(1, (1 << 27) // n)
                for g in range(G):
                    for p0 in range(0, w, size):
                        p1 = min(w, p0 + size)
                        z = (s.q[b, l, h * G + g, p0:p1].double() @ keys) / math.sqrt(d)
                        z[:, ~live] = -math.inf
                        if c["causal"]:
                            row = torch.arange(n - w + p0, n - w + p1, device="cuda")
                            z[torch.arange(n, device="cuda")[None] > row[:, None]] = -math.inf
                        if c["given"]:
                            ls = s.lse[b, l, h * G + g, p0:p1].double()
                        else:
                            ls = torch.logsumexp(z, 1)
                            lse[b, l, h * G + g, p0:p1] = ls
                        seen = ls > -math.inf
                        p = torch.exp(z[seen] - ls[seen, None])
                        if s.row_weight is not None:
                            p = p * s.row_weight[b, p0:p1].double()[seen, None]
                        got += p.sum(0)
                a[live] = c["decay"] * a[live] + got[live]
    return {"acc": acc} if c["given"] else {"acc": acc, "lse": lse}


def _exact_evict(s):
    """The definition, unit by unit on the host: what has the most weight stays."""
    c = s.case
    L, H, B, bud, d = c["layers"], c["kv_heads"], len(s.lens), c["budget"], c["head_dim"]
    acc = s.acc.double().cpu()
    new = acc.clone()
    cap = max(1, max(_row_counts(s)) - bud)
    idx = torch.full((B, L, H, bud), -1, dtype=torch.int64)
    slots = torch.full((B, L, H, cap), -1, dtype=torch.int64)
    acc_out = torch.full((B, L, H, bud), -1.0, dtype=torch.float64)
    k_out = torch.zeros((B, L, H, bud, d), dtype=s.k.dtype, device="cuda")
    v_out = torch.zeros_like(k_out)
    evict = c["op"] == "evict"
    for b, n in enumerate(s.lens):
        lo, kk = s.starts[b], min(bud, n)
        tail = min(c["protect"], kk)
        for l in range(L):
            for h in range(H):
                a = acc[l, h, lo:lo + n]
                key = a.clone()
                key[n - tail:] = math.inf       # the tail stays whatever it weighs
                kept = torch.argsort(key, descending=True, stable=True)[:kk].sort().values
                gone = torch.ones((n,), dtype=torch.bool)
                gone[kept] = False
                drop = gone.nonzero()[:, 0]
                idx[b, l, h, :kk] = kept
                acc_out[b, l, h, :kk] = a[kept]
                slots[b, l, h, :len(drop)] = drop
                new[l, h, lo + drop] = -1.0
                if evict:
                    k_out[b, l, h, :kk] = s.k[l, h, lo + kept.cuda()]
                    v_out[b, l, h, :kk] = s.v[l, h, lo + kept.cuda()]
    if evict:
        return {"idx": idx.int().cuda(), "k": _words(k_out), "v": _words(v_out), "acc": acc_out.cuda()}
    return {"slots": slots.int().cuda(), "acc": new.cuda()}


def exact(case, seed):
    c = _full(case)
    s = _inputs(c, seed)
    if c["op"] in ("evict", "slots"):
        return _exact_evict(s)
    return _exact_attend(s) if c["op"] == "attend" else _exact_weights(s)

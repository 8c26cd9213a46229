"""jacap_verify against its definition in float64 (quant_ref.Verified): chains and trees,
with and without the draft's probabilities, greedy, any vocabulary and row alignment,
padding, rows that cannot be used. The kernel's exponentials are fp32 and the reference's
fp64: a test or draw within about 1e-7 of its border may differ, which none of the numbers
drawn here is (seeds are fixed)."""

import math

import pytest
import torch

from quant_ref import Verified

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def jacap():
    from paper_2609_08131_amd import jacap as j
    return j


class Batch:
    def __init__(self, B, S, V, dtype, tree=True, draft=False, seed=0, wide=0, peak=6.0):
        gen = torch.Generator().manual_seed(seed)
        z = 1.5 * torch.randn((B, S, V), generator=gen)
        z.scatter_(2, torch.randint(0, V, (B, S, 4), generator=gen), peak)
        self.parents = None
        if tree:
            p = torch.floor(torch.rand((B, S), generator=gen) * torch.arange(S)).int()
            p = torch.where(torch.rand((B, S), generator=gen) < 0.4, torch.zeros_like(p), p)  # many siblings
            p[:, 0] = -1
            self.parents = p.cuda()
        up = self.parents.cpu() if tree else (torch.arange(S) - 1).expand(B, S)
        up = up.clamp_min(0).long()
        q = torch.softmax(z + 0.8 * torch.randn((B, S, V), generator=gen), -1)
        at = torch.arange(B)[:, None]
        self.tokens = torch.multinomial(q[at, up].reshape(B * S, V), 1, generator=gen).view(B, S).int().cuda()
        self.uniform = torch.rand((B, S), generator=gen).cuda()
        base = torch.zeros((B, S, V + wide), dtype=dtype, device="cuda")
        self.logits = base[:, :, wide // 2:wide // 2 + V]     # rows of any alignment
        self.logits.copy_(z)
        self.draft = None
        if draft:
            base = torch.zeros((B, S, V + wide), device="cuda")
            self.draft = base[:, :, wide - wide // 2:wide - wide // 2 + V]
            self.draft.copy_(q)

    def run(self, jacap, T):
        prob = jacap.prepare_verify(self.logits, jacap.VerifyParams(T, self.parents), draft=self.draft)
        for x in (prob.path, prob.count, prob.next, prob.row_weight):
            x.fill_(77)
        jacap.run_verify(prob, self.logits, self.tokens, self.uniform if T else None, draft=self.draft)
        return prob

    def check(self, jacap, T):
        prob = self.run(jacap, T)
        B, S, V = self.logits.shape
        flag, accepted = False, 0
        for b in range(B):
            want = Verified(self.logits[b], self.tokens[b], self.uniform[b],
                            None if self.parents is None else self.parents[b].tolist(),
                            None if self.draft is None or T == 0 else self.draft[b], T)
            n = len(want.path)
            assert prob.path[b].tolist() == want.path + [-1] * (S - n), f"path of {b}"
            assert int(prob.count[b]) == n and int(prob.next[b]) == want.next, f"next of {b}"
            weight = torch.zeros(S)
            weight[want.path] = 1.0
            assert torch.equal(prob.row_weight[b].cpu(), weight)
            flag |= want.flag
            accepted += n - 1
        assert jacap.read_status(prob.ws) == (jacap.FLAG_NONFINITE if flag else 0)
        return prob, accepted


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T", [0.0, 0.7, 1.0])
@pytest.mark.parametrize("draft", [False, True])
@pytest.mark.parametrize("B,S,V,tree,wide", [(3, 1, 5, False, 0), (4, 5, 1000, False, 3), (5, 17, 8191, True, 1),
                                             (3, 64, 515, True, 9), (2, 130, 100, True, 0), (2, 9, 33000, True, 5)])
def test_verify(jacap, dtype, T, draft, B, S, V, tree, wide):
    print(f"[verify] {dtype} T{T} draft {draft} B{B} S{S} V{V}", flush=True)
    Batch(B, S, V, dtype, tree, draft, seed=B * S + V, wide=wide).check(jacap, T)


def test_accepts_and_rejects(jacap):
    """Inputs like those above lead to accepted and to rejected rows."""
    for draft in (False, True):
        _, n = Batch(16, 33, 300, F32, True, draft, seed=1).check(jacap, 1.0)
        assert 1 <= n < 16 * 32


@pytest.mark.parametrize("draft", [False, True])
def test_large_vocabulary(jacap, draft):
    Batch(2, 4, 256001, BF, False, draft, seed=3).check(jacap, 0.9)


def test_longest_chain(jacap):
    """512 rows, all accepted by the greedy rule, and by chance."""
    b = Batch(2, 512, 40, F32, tree=False, seed=5)
    best = b.logits.float().argmax(-1).int()
    b.tokens[:, 1:] = best[:, :-1]
    prob, n = b.check(jacap, 0.0)
    assert n == 2 * 511
    b.uniform[:, 1:] *= 1e-3
    prob, n = b.check(jacap, 1.0)
    assert n > 100


@pytest.mark.parametrize("draft", [False, True])
def test_many_siblings(jacap, draft):
    """All rows children of row 0, tokens twice among them, more than a wave's lanes."""
    b = Batch(3, 200, 60, F32, tree=True, draft=draft, seed=6)
    b.parents[:, 1:] = 0
    b.uniform[:, 1:] = 0.999 + 0.0009 * b.uniform[:, 1:]      # mostly rejected
    if not draft:
        b.tokens[:, 1:40] = torch.arange(39, dtype=torch.int32, device="cuda") // 3
    b.check(jacap, 1.3)


def test_padding_and_tokens_outside(jacap):
    """Parents and tokens that are none: not tested, nothing read outside the rows."""
    b = Batch(4, 12, 333, BF, seed=7)
    b.parents[0, 4:] = -1
    b.parents[1, 3] = 3
    b.parents[1, 5] = 9
    b.parents[1, 6] = 2 ** 31 - 1
    b.parents[2, :] = -2 ** 31
    b.tokens[2, 1:] = -1
    b.tokens[3, 1::2] = 333
    b.tokens[3, 2] = 2 ** 31 - 1
    b.tokens[:, 0] = -7
    for T in (0.0, 1.0):
        b.check(jacap, T)


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("T", [0.0, 1.0])
def test_rows_that_cannot_be_used(jacap, dtype, T):
    """NaN, infinities and rows of -inf: at the start, behind an accepted row, and where no walk
    comes; the other sequences are as ever."""
    b = Batch(7, 6, 9000, dtype, tree=False, seed=8)
    best = torch.nan_to_num(b.logits.float()).argmax(-1).int()
    b.tokens[:, 1:] = best[:, :-1]
    b.uniform[:, 1:] *= 1e-6             # accepted
    b.logits[0, 0, 8999] = math.nan
    b.logits[1, 2, 5] = math.inf
    b.logits[2, 0] = -math.inf
    b.logits[3, 3] = math.nan
    b.logits[4, 0, ::2] = -math.inf
    b.logits[4, 0, best[4, 0]] = 9.0
    b.logits[5, 5, 17] = math.nan
    b.tokens[5, 5] = (best[5, 4] + 1) % 9000
    b.uniform[5, 5] = 0.9999
    b.check(jacap, T)


def test_draft_that_is_not_a_number(jacap):
    """A NaN among the probabilities that a draw needs ends the sequence; an unneeded one does
    nothing."""
    b = Batch(3, 3, 400, F32, tree=False, draft=True, seed=9)
    b.uniform[:, 1] = 0.0
    b.uniform[0, 1] = 0.99999            # sequence 0 rejects row 1 and draws from what is left
    b.draft[:, 0, 7] = math.nan
    b.tokens[:, 1] = 11
    b.draft[:, 0, 11] = 0.9
    b.check(jacap, 1.0)


@pytest.mark.parametrize("u", [0.0, 1.0 - 2 ** -24, 1.0, 2.0])
def test_ends_of_the_draw(jacap, u):
    """The first and the last token of positive probability; numbers at and past 1."""
    b = Batch(3, 1, 20000, BF, tree=False, seed=10)
    b.logits[:, :, :3] = -math.inf
    b.logits[:, :, 19000:] = -math.inf
    b.uniform[:] = u
    prob, _ = b.check(jacap, 1.0)
    if u == 0.0 or u >= 1.0:
        assert prob.next.tolist() == [3 if u == 0.0 else 18999] * 3


def test_nothing_left(jacap):
    """The draft's probabilities above the target's everywhere, by more than rounding: the draw
    is of the target's own."""
    b = Batch(2, 2, 50, F32, tree=False, draft=True, seed=11)
    b.draft.copy_(torch.softmax(b.logits.double(), -1).float() * 1.01)
    b.uniform[:, 1] = 0.999
    prob, n = b.check(jacap, 1.0)
    assert n == 0


@pytest.mark.parametrize("draft", [False, True])
def test_distribution(jacap, draft):
    """4096 sequences of one distribution, numbers drawn: the first received tokens' shares
    are the target's, within 5 standard deviations (p (1 - p) / N each)."""
    N, V = 4096, 7
    gen = torch.Generator(device="cuda").manual_seed(12)
    z = torch.randn((1, 4, V), generator=gen, device="cuda")
    logits = z.expand(N, 4, V)            # sequences share their logits: a stride of 0
    q = torch.softmax(z[:, :1] + torch.randn((1, 1, V), generator=gen, device="cuda"), -1)
    parents = torch.tensor([-1, 0, 0, 0], dtype=torch.int32, device="cuda").expand(N, 4).contiguous()
    if draft:
        tokens = torch.multinomial(q[0, 0].expand(N, V), 4, replacement=True, generator=gen).int()
    else:
        tokens = torch.tensor([0, 2, 5, 1], dtype=torch.int32, device="cuda").expand(N, 4).contiguous()
    uniform = torch.rand((N, 4), generator=gen, device="cuda")
    prob = jacap.prepare_verify(logits, jacap.VerifyParams(1.0, parents),
                                draft=q.expand(N, 4, V) if draft else None)
    jacap.run_verify(prob, logits, tokens, uniform, draft=q.expand(N, 4, V) if draft else None)
    second = prob.path[:, 1].long()
    got = torch.where(second > 0, tokens.gather(1, second.clamp_min(0)[:, None])[:, 0], prob.next)
    p = torch.softmax(z[0, 0].double(), -1)
    share = torch.bincount(got.long(), minlength=V).double() / N
    assert bool(((share - p).abs() <= 5 * torch.sqrt(p * (1 - p) / N)).all())
    assert bool((second > 0).any()) and bool((second < 0).any())


@pytest.mark.parametrize("T,draft", [(0.0, False), (1.0, False), (1.0, True)])
def test_captured(jacap, T, draft):
    """Replayed with other inputs and eager work between: each replay is the eager result."""
    b = Batch(3, 9, 5000, BF, tree=True, draft=draft, seed=13)
    others = [Batch(3, 9, 5000, BF, tree=True, draft=draft, seed=s) for s in (14, 15, 16)]
    prob = jacap.prepare_verify(b.logits, jacap.VerifyParams(T, b.parents), draft=b.draft)
    go = lambda: jacap.run_verify(prob, b.logits, b.tokens, b.uniform, draft=b.draft)
    go()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for o in others:
        for name in ("logits", "tokens", "uniform", "parents") + (("draft",) if draft else ()):
            getattr(b, name).copy_(getattr(o, name))
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (prob.path, prob.count, prob.next, prob.row_weight)]
        want = o.check(jacap, T)[0]
        for x, y in zip(got, (want.path, want.count, want.next, want.row_weight)):
            assert torch.equal(x, y)


def test_refusals(jacap):
    b = Batch(2, 4, 50, F32, tree=True, seed=1)
    V = jacap.VerifyParams
    with pytest.raises(ValueError):
        jacap.prepare_verify(b.logits.half(), V())
    with pytest.raises(ValueError):
        jacap.prepare_verify(b.logits.transpose(1, 2), V())
    with pytest.raises(ValueError):
        jacap.prepare_verify(b.logits, V(), draft=b.logits[:, :2])
    with pytest.raises(ValueError):
        jacap.prepare_verify(b.logits, V(parents=b.parents.long()))
    with pytest.raises(jacap.JacapError):
        jacap.prepare_verify(b.logits, V(temperature=-1.0))
    prob = jacap.prepare_verify(b.logits, V(1.0, b.parents))
    with pytest.raises(ValueError):
        jacap.run_verify(prob, b.logits, b.tokens)
    with pytest.raises(ValueError):
        jacap.run_verify(prob, b.logits, b.tokens.long(), b.uniform)
    with pytest.raises(ValueError):
        jacap.run_verify(prob, b.logits, b.tokens, b.uniform, draft=b.logits)

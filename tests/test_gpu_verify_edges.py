"""jacap_verify where a row's numbers leave it little or nothing: a logit that is not a number at a
tested child's own token, and rejected children that are all, or all but one, of what the row can
give. The largest number below 1 accepts the last of them, as u N < w holds where w is all of N."""

import math

import pytest
import torch

from test_gpu_verify import BF, F32, Batch, jacap  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("draft", [False, True])
@pytest.mark.parametrize("odd", [math.nan, math.inf])
def test_a_childs_token_that_is_not_a_number(jacap, dtype, draft, odd):
    """The one logit that is not finite is that of a tested child, alone or beside a sibling, at row
    0 and behind an accepted row: the sequence ends there, whatever its children's tests leave out."""
    b = Batch(5, 4, 9000, dtype, tree=True, draft=draft, seed=21)
    b.parents.copy_(torch.tensor([[-1, 0, -1, -1], [-1, 0, 0, -1], [-1, 0, 0, 0], [-1, 0, 1, 1], [-1, 0, 0, 0]]))
    best = b.logits.float().argmax(-1).int()
    b.tokens[:, 1:] = torch.tensor([17, 4000, 8999], dtype=torch.int32)
    b.uniform[:, 1:] = 0.9
    b.tokens[3, 1] = best[3, 0]          # accepted: row 1 is the current one
    b.uniform[3, 1] = 0.0
    for at in ((0, 0, 17), (1, 0, 17), (2, 0, 4000), (3, 1, 8999)):
        b.logits[at] = odd
    prob, _ = b.check(jacap, 1.0)
    assert prob.next.tolist()[:4] == [-1] * 4 and prob.count.tolist()[:4] == [1, 1, 1, 2]
    assert int(prob.next[4]) >= 0


LAST = 1.0 - 2.0 ** -24      # the largest number below 1


def siblings(dtype, logits, tokens, uniform):
    """Sequences whose rows but the first are children of row 0: its logits [B][V], their tokens
    [B][S - 1] and the numbers [B][S]."""
    z, t = torch.as_tensor(logits, dtype=torch.float32), torch.as_tensor(tokens, dtype=torch.int32)
    B, V = z.shape
    b = Batch(B, t.shape[1] + 1, V, dtype, tree=True, seed=22)
    b.parents[:, 1:] = 0
    b.logits[:, 0] = z.to(dtype).cuda()
    b.tokens[:, 1:] = t.cuda()
    b.uniform[:] = torch.as_tensor(uniform, dtype=torch.float32).cuda()
    return b


def support(V, at, values):
    """Logits [B][V] of -inf but for values [B][n] at the tokens at [B][n]."""
    z = torch.full((len(values), V), -math.inf)
    return z.scatter_(1, torch.as_tensor(at), torch.as_tensor(values, dtype=torch.float32))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", [8, 20001])
def test_the_last_of_the_support(jacap, dtype, V):
    """Children that are all a row can give: after the others' rejection the last has all that is
    left, and any number below 1 accepts it."""
    second = torch.linspace(-9.0, -0.5, 200)
    z = support(V, [[0, 1]] * 200, torch.stack([torch.zeros(200), second], 1))
    b = siblings(dtype, z, [[0, 1]] * 200, [[0.5, 0.9999, LAST]] * 200)
    prob, _ = b.check(jacap, 1.0)
    assert prob.path.tolist() == [[0, 2, -1]] * 200
    # what the second adds to the first's 1 is of the size of fp32's last bit
    z = support(V, [[V - 2, V - 1]], [[0.0, -16.45]])
    prob, _ = siblings(dtype, z, [[V - 2, V - 1]], [[0.5, LAST, 0.9]]).check(jacap, 1.0)
    assert prob.path.tolist() == [[0, 2, -1]]


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("n,V", [(3, 40), (7, 30000), (100, 100), (100, 9000)])
def test_all_of_the_support_but_one(jacap, dtype, n, V):
    """n children for n tokens, in any order, some of them twice: each is rejected by the largest
    number, but the last one left."""
    gen = torch.Generator().manual_seed(n + V)
    B = 24
    at = torch.stack([torch.randperm(V, generator=gen)[:n] for _ in range(B)])
    z = support(V, at, -3.0 * torch.rand((B, n), generator=gen))
    order = torch.stack([torch.randperm(n, generator=gen) for _ in range(B)])
    tokens = at.gather(1, order)
    tokens = torch.cat([tokens[:, :2], tokens[:, :1], tokens[:, 2:]], 1)
    b = siblings(dtype, z, tokens, torch.full((B, n + 2), LAST))
    b.uniform[:, 0] = torch.rand(B, generator=gen).cuda()
    prob, _ = b.check(jacap, 1.0)
    assert prob.path[:, 1].tolist() == [n + 1] * B


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("V", [8, 40000])
def test_nothing_left_without_draft_probabilities(jacap, dtype, V):
    """Numbers of 1 and more reject all that a row can give: the draw is from the row's own
    weights, the rejected tokens' among them."""
    gen = torch.Generator().manual_seed(V)
    B, n = 32, 4
    at = torch.stack([torch.randperm(V, generator=gen)[:n] for _ in range(B)])
    z = support(V, at, -2.0 * torch.rand((B, n), generator=gen))
    b = siblings(dtype, z, at, [[0.5, 1.0, 2.0, 1.0, 1.5]] * B)
    b.uniform[:, 0] = torch.rand(B, generator=gen).cuda()
    prob, accepted = b.check(jacap, 1.0)
    assert accepted == 0 and all(int(x) in row for x, row in zip(prob.next, at.tolist()))
    assert len({row.index(int(x)) for x, row in zip(prob.next, at.tolist())}) > 1


@pytest.mark.parametrize("dtype", [BF, F32])
def test_the_last_of_the_support_behind_an_accepted_row(jacap, dtype):
    """The same two rows down a tree, between children of other rows."""
    b = Batch(6, 9, 5000, dtype, tree=True, seed=23)
    b.parents.copy_(torch.tensor([-1, 0, 0, 1, 1, 2, 3, 3, 3]))
    best = b.logits[:, :2].float().argmax(-1).int()
    b.tokens[:, 1], b.tokens[:, 3] = best[:, 0], best[:, 1]
    b.tokens[:, 2], b.tokens[:, 4] = 7, 9
    b.logits[:, 3] = support(5000, [[4, 4999, 17]] * 6, [[-0.4 * r, -0.1, -0.25] for r in range(6)]).to(dtype).cuda()
    b.tokens[:, 6:] = torch.tensor([4999, 17, 4], dtype=torch.int32)
    b.uniform[:] = LAST
    b.uniform[:, 1], b.uniform[:, 3] = 0.0, 0.0
    prob, _ = b.check(jacap, 1.0)
    assert prob.path.tolist() == [[0, 1, 3, 8] + [-1] * 5] * 6

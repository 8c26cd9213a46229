"""jacap_verify where a row's numbers leave it little or nothing: a logit that is not a number at a
tested child's own token."""

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

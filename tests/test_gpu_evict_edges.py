"""Edges of the eviction by accumulated weight and of the lists of evicted slots."""

import pytest
import torch

from test_gpu_evict_weighted import _cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def jacap():
    from paper_2609_08131_amd import jacap as j
    return j


@pytest.mark.parametrize("lens,budget,cap", [([459, 0, 3], 459, 1), ([459, 0, 3], 1000, 9),
                                             ([700] * 40, 700, 5000)])
def test_no_sequence_above_the_budget(jacap, lens, budget, cap):
    """Nothing is evicted: every list is -1 whatever its capacity, and the accumulators, NaN
    and empty slots among them, stay as they are; the same from scores."""
    L, H = 2, 2
    k, v, acc, offs, rows, live = _cache(lens, L, H, 64, torch.bfloat16, 5)
    prob = jacap.prepare_evict_weighted(k, v, offs, rows, budget, 4, live)
    slots = torch.full((len(lens), L, H, cap), 7, dtype=torch.int32, device="cuda")
    before = acc.clone()
    jacap.run_evict_weighted_slots(prob, acc, slots)
    assert torch.equal(slots, torch.full_like(slots, -1))
    assert torch.equal(acc.view(torch.int32), before.view(torch.int32))
    ws = torch.empty(jacap.workspace_size(prob.cfg, prob.batch), dtype=torch.uint8, device="cuda")
    slots.fill_(7)
    jacap.select_evicted(prob.cfg, prob.batch, acc, slots, ws)
    assert torch.equal(slots, torch.full_like(slots, -1))

"""jacap_quantize given lengths that contradict the sequences' rows: what such a sequence holds stays."""

import pytest
import torch

from test_gpu_quant import BF, F32, check_quantized, empty_cache, jacap, wide_case  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d,block", [(BF, 128, 32), (F32, 64, 128)])
@pytest.mark.parametrize("hides", [False, True])
@pytest.mark.parametrize("bad", [-1, -2 ** 31, 385, 2 ** 31 - 1])
def test_a_length_that_is_not_of_the_rows(jacap, dtype, d, block, hides, bad):
    """Written again in place with one wrong length on the device: that sequence keeps its codes and
    scales, the others get theirs."""
    lens = [300, 384, 17, 0]
    rows, starts, k, v = wide_case(dtype, d, block, lens, seed=block)
    assert rows[1] == 384
    cache = empty_cache(jacap, *k.shape[:4], block, False)
    off = torch.tensor(starts, dtype=torch.int32, device="cuda")
    live = torch.tensor(lens, dtype=torch.int32, device="cuda")
    prob = jacap.prepare_quantize(k, v, cache, off, rows, live_lens=live)
    acc = torch.ones(k.shape[:3], device="cuda") if hides else None
    jacap.run_quantize(prob, k, v, cache, acc=acc)
    check_quantized(cache, (k, v), starts, lens, block)
    old = [x.clone() for x in (cache.k.view(torch.uint8), cache.v.view(torch.uint8), cache.scales)]
    live[1] = bad
    k.mul_(8.0)
    v.mul_(8.0)
    jacap.run_quantize(prob, k, v, cache, acc=acc)
    a, e = starts[1], starts[2]
    now = [cache.k.view(torch.uint8), cache.v.view(torch.uint8), cache.scales]
    for i, (x, y) in enumerate(zip(now, old)):
        part = slice(a, e) if i < 2 else slice(a // block, e // block)
        assert torch.equal(x[:, :, part], y[:, :, part])
        x[:, :, part] = 0x2A if i < 2 else 2.0 ** -100     # as check_quantized wants an empty sequence
    check_quantized(cache, (k, v), starts, [300, 0, 17, 0], block)

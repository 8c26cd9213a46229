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

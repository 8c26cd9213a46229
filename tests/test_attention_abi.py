"""Host-side checks of the attention entry points (no GPU, nothing launched):
the descriptor's layout, and the arguments that are refused."""

import ctypes
import os
import subprocess
import tempfile

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
jacap = pytest.importorskip("paper_2609_08131_amd.jacap")
P = ctypes.c_void_p
GOOD = 0x100000


def test_struct_layout_matches_header():
    fields = [n for n, _ in jacap.Attention._fields_]
    prog = '#include <stdio.h>\n#include <stddef.h>\n#include "jacap.h"\nint main(void) {\n' + \
        'printf("size %zu\\n", sizeof(jacap_attention));\n' + \
        "".join(f'printf("{f} %zu\\n", offsetof(jacap_attention, {f}));\n' for f in fields) + "return 0; }\n"
    with tempfile.TemporaryDirectory() as d:
        src, exe = os.path.join(d, "t.c"), os.path.join(d, "t")
        open(src, "w").write(prog)
        subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), src, "-o", exe], check=True)
        out = dict(x.split() for x in subprocess.run([exe], capture_output=True, text=True,
                                                    check=True).stdout.splitlines())
    assert int(out["size"]) == ctypes.sizeof(jacap.Attention)
    for f in fields:
        assert int(out[f]) == getattr(jacap.Attention, f).offset, f


def cfg(**kw):
    base = dict(num_layers=1, num_kv_heads=1, num_q_heads=4, head_dim=64, window=5, budget_k=8,
                temperature=10.0, ridge=1.0, cov_mode=0, dtype=1)
    base.update(kw)
    return jacap.Config(**base)


def batch(**kw):
    b = jacap.Batch()
    b.num_seqs, b.max_seq_len, b.total_tokens = 1, 100, 100
    b.seq_offsets = 0x1000
    b.k_stride_layer = b.v_stride_layer = b.k_stride_head = b.v_stride_head = 6400
    b.k_stride_token = b.v_stride_token = 64
    b.q_stride_seq = b.q_stride_layer = 2048
    b.q_stride_head, b.q_stride_pos = 320, 64
    b.out_stride_seq, b.out_stride_layer, b.out_stride_head, b.out_stride_row = 512, 512, 512, 64
    for k, v in kw.items():
        setattr(b, k, v)
    return b


def attn(**kw):
    a = jacap.Attention()
    a.scale, a.decay = 0.125, 1.0
    for x in ("dk", "dv"):
        for n, s in (("seq", 320), ("layer", 320), ("head", 320), ("row", 64)):
            setattr(a, f"{x}_stride_{n}", s)
    a.o_stride_seq = a.o_stride_layer = 1280
    a.o_stride_head, a.o_stride_pos = 320, 64
    a.a_stride_seq = a.a_stride_layer = a.a_stride_head = 8
    for k, v in kw.items():
        setattr(a, k, v)
    return a


SIZES = ("jacap_attend_workspace_size", "jacap_attn_weights_workspace_size",
         "jacap_evict_weighted_workspace_size")


def size(fn, c, b, a):
    n = ctypes.c_size_t(0)
    code = getattr(jacap._lib, fn)(ctypes.byref(c), ctypes.byref(b), ctypes.byref(a), ctypes.byref(n))
    return code, n.value


@pytest.mark.parametrize("fn", SIZES)
def test_sizes_and_refusals(fn):
    code, n = size(fn, cfg(), batch(), attn())
    assert code == jacap.OK and n >= 256 and n % 256 == 0
    bad = jacap.ERR_INVALID_ARG
    for a in (attn(scale=0.0), attn(scale=-1.0), attn(scale=float("nan")), attn(scale=float("inf")),
              attn(decay=-0.5), attn(decay=1.01), attn(decay=float("nan")), attn(accumulate=2),
              attn(causal=-1), attn(live_lens=0x1002), attn(row_weight=0x1001), attn(tree=0x1004)):
        assert size(fn, cfg(), batch(), a)[0] == bad
    assert size(fn, cfg(head_dim=96), batch(), attn())[0] == jacap.ERR_UNSUPPORTED
    assert size(fn, cfg(dtype=2), batch(), attn())[0] == jacap.ERR_UNSUPPORTED
    assert size(fn, cfg(window=0), batch(), attn())[0] == bad
    assert size(fn, cfg(), batch(k_stride_token=60), attn())[0] == bad
    lib = getattr(jacap._lib, fn)
    assert lib(ctypes.byref(cfg()), ctypes.byref(batch()), None, ctypes.byref(ctypes.c_size_t())) == bad
    assert lib(ctypes.byref(cfg()), ctypes.byref(batch()), ctypes.byref(attn()), None) == bad
    assert lib(None, ctypes.byref(batch()), ctypes.byref(attn()), ctypes.byref(ctypes.c_size_t())) == bad


def test_attend_limits():
    f = SIZES[0]
    assert size(f, cfg(window=512), batch(), attn())[0] == jacap.OK
    assert size(f, cfg(window=513), batch(), attn())[0] == jacap.ERR_UNSUPPORTED
    for name in ("dk_stride_row", "dv_stride_row", "o_stride_pos"):
        assert size(f, cfg(), batch(), attn(**{name: 56}))[0] == jacap.ERR_INVALID_ARG
        assert size(f, cfg(), batch(), attn(**{name: 68}))[0] == jacap.ERR_INVALID_ARG
        assert size(f, cfg(), batch(), attn(**{name: -64}))[0] == jacap.ERR_INVALID_ARG
    assert size(f, cfg(), batch(), attn(dk_stride_row=(1 << 24) + 8))[0] == jacap.ERR_UNSUPPORTED
    # the grid: units x chunks x row blocks
    big = batch(num_seqs=65535, max_seq_len=1 << 24, total_tokens=1 << 24)
    assert size(f, cfg(window=512, num_q_heads=8), big, attn())[0] == jacap.ERR_UNSUPPORTED
    # few rows keep their logits when they accumulate: 4 bytes a row and token
    long = batch(max_seq_len=100000, total_tokens=100000)
    plain, keep = size(f, cfg(window=4), long, attn())[1], size(f, cfg(window=4), long, attn(accumulate=1))[1]
    assert keep >= plain + 4 * 16 * 100000


def test_entry_points_reject_bad_pointers():
    c, b, a = cfg(), batch(), attn(accumulate=1)
    n = size(SIZES[0], c, b, a)[1]
    bad, lib = jacap.ERR_INVALID_ARG, jacap._lib

    def attend(i=None, value=None, ws=P(GOOD), nbytes=n):
        args = [P(GOOD)] * 9                # q k v kd vd out lse acc acc_draft
        if i is not None:
            args[i] = value
        return lib.jacap_attend(ctypes.byref(c), ctypes.byref(b), ctypes.byref(a), *args, ws, nbytes, None)

    for i in range(6):
        assert attend(i, None) == bad
        assert attend(i, P(GOOD + 8)) == bad
    for i in (6, 7, 8):
        assert attend(i, P(GOOD + 2)) == bad
    assert attend(7, None) == bad            # accumulating needs the accumulators
    assert attend(ws=None) == bad and attend(ws=P(GOOD + 128)) == bad
    assert attend(nbytes=n - 1) == jacap.ERR_WORKSPACE

    n = size(SIZES[1], c, b, a)[1]

    def weights(i=None, value=None, ws=P(GOOD), nbytes=n):
        args = [P(GOOD), P(GOOD), None, P(GOOD), P(GOOD)]   # q k lse_in lse_out acc
        if i is not None:
            args[i] = value
        return lib.jacap_attn_weights(ctypes.byref(c), ctypes.byref(b), ctypes.byref(a), *args, ws, nbytes, None)

    for i in (0, 1, 4):
        assert weights(i, None) == bad
    assert weights(2, P(GOOD)) == bad        # lse_in and lse_out together
    assert weights(2, P(GOOD + 1)) == bad and weights(3, P(GOOD + 2)) == bad
    assert weights(ws=None) == bad and weights(nbytes=n - 256) == jacap.ERR_WORKSPACE

    def evict(i=None, value=None, a_=None):
        args = [P(GOOD)] * 7                # acc k v idx k_out v_out acc_out
        if i is not None:
            args[i] = value
        return lib.jacap_evict_weighted(ctypes.byref(c), ctypes.byref(b), ctypes.byref(a_ or a), *args, None)

    for i in range(7):
        assert evict(i, None) == bad
    for i in range(1, 6):
        assert evict(i, P(GOOD + 4)) == bad
    assert evict(a_=attn(a_stride_head=-8)) == bad

    n = size(SIZES[2], c, b, a)[1]
    slots = lambda acc=P(GOOD), s=P(GOOD), cap=92, ws=P(GOOD), nbytes=n: lib.jacap_evict_weighted_slots(
        ctypes.byref(c), ctypes.byref(b), ctypes.byref(a), acc, s, ctypes.c_int32(cap), ws, nbytes, None)
    assert slots(cap=91) == bad and slots(acc=None) == bad and slots(s=None) == bad
    assert slots(s=P(GOOD + 4)) == bad and slots(ws=None) == bad
    assert slots(nbytes=n - 256) == jacap.ERR_WORKSPACE

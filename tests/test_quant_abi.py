"""Host-side checks of the 8-bit cache's and the verification's entry points (no GPU, nothing
launched): the descriptors' layouts, and the arguments that are refused."""

import ctypes
import os
import subprocess
import tempfile

import pytest

from test_attention_abi import GOOD, P, attn, batch, cfg

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
jacap = pytest.importorskip("paper_2609_08131_amd.jacap")
BAD, UNSUP = jacap.ERR_INVALID_ARG, jacap.ERR_UNSUPPORTED
ref = ctypes.byref


def test_struct_layouts_match_header():
    for name, cls in (("jacap_quant", jacap.Quant), ("jacap_verification", jacap.Verification)):
        fields = [n for n, _ in cls._fields_]
        prog = '#include <stdio.h>\n#include <stddef.h>\n#include "jacap.h"\nint main(void) {\n' + \
            f'printf("size %zu\\n", sizeof({name}));\n' + \
            "".join(f'printf("{f} %zu\\n", offsetof({name}, {f}));\n' for f in fields) + "return 0; }\n"
        with tempfile.TemporaryDirectory() as d:
            src, exe = os.path.join(d, "t.c"), os.path.join(d, "t")
            open(src, "w").write(prog)
            subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), src, "-o", exe], check=True)
            out = dict(x.split() for x in subprocess.run([exe], capture_output=True, text=True,
                                                        check=True).stdout.splitlines())
        assert int(out["size"]) == ctypes.sizeof(cls)
        for f in fields:
            assert int(out[f]) == getattr(cls, f).offset, f


def qbatch(**kw):
    return batch(**{**dict(max_seq_len=96, total_tokens=96), **kw})


def quant(**kw):
    q = jacap.Quant(32, 0, 6144, 6144, 64, 6144, 6144, 64)
    for k, v in kw.items():
        setattr(q, k, v)
    return q


def size(c, b, a, q):
    n = ctypes.c_size_t(0)
    return jacap._lib.jacap_attend_quant_workspace_size(ref(c), ref(b), ref(a), ref(q), ref(n)), n.value


def calls(c, b, a, q, n=1 << 40):
    """Every entry point's code for these descriptors (null data: refused before any launch)."""
    g = P(GOOD + 8)     # misaligned: what is not refused by the descriptors is by this
    lib = jacap._lib
    return (size(c, b, a, q)[0],
            lib.jacap_attend_quant(ref(c), ref(b), ref(a), ref(q), *[g] * 10, P(GOOD), n, None),
            lib.jacap_quantize(ref(c), ref(b), ref(a), ref(q), g, g, None, g, g, g, None),
            lib.jacap_append_quant(ref(c), ref(b), ref(a), ref(q), g, g, g, None, None, None, 0, g, g, g, None,
                                   None, None, None, None),
            lib.jacap_attn_weights_quant(ref(c), ref(b), ref(a), ref(q), g, g, g, g, g, None, None))


def test_descriptors():
    code, n = size(cfg(), qbatch(), attn(), quant())
    assert code == jacap.OK and n >= 256 and n % 256 == 0
    for q, want in ((quant(block=8), UNSUP), (quant(block=48), UNSUP), (quant(block=256), UNSUP),
                    (quant(block=0), UNSUP), (quant(reserved=1), BAD), (quant(k_stride_token=72), BAD),
                    (quant(k_stride_token=48), BAD), (quant(v_stride_head=-16), BAD), (quant(v_stride_layer=8), BAD),
                    (quant(k_stride_token=(1 << 24) + 16), UNSUP), (quant(v_stride_token=(1 << 24) + 16), UNSUP)):
        assert set(calls(cfg(), qbatch(), attn(), q)) == {want}
    assert set(calls(cfg(), qbatch(total_tokens=100, max_seq_len=100), attn(), quant())) == {BAD}
    assert set(calls(cfg(head_dim=96), qbatch(), attn(), quant(k_stride_token=96, v_stride_token=96))) == {UNSUP}
    assert set(calls(cfg(dtype=2), qbatch(), attn(), quant())) == {UNSUP}
    assert set(calls(cfg(), qbatch(), attn(scale=0.0), quant())) == {BAD}
    # the batch's own K and V strides are those of the wide cache, which only one call has
    odd = qbatch(k_stride_token=60, v_stride_head=4)
    assert size(cfg(), odd, attn(), quant())[0] == jacap.OK
    got = calls(cfg(), odd, attn(), quant())
    assert got[2] == BAD
    lib = jacap._lib
    assert lib.jacap_attend_quant_workspace_size(ref(cfg()), ref(qbatch()), ref(attn()), None, ref(ctypes.c_size_t())) == BAD
    assert lib.jacap_attend_quant_workspace_size(ref(cfg()), ref(qbatch()), ref(attn()), ref(quant()), None) == BAD
    assert lib.jacap_attend_quant_workspace_size(None, ref(qbatch()), ref(attn()), ref(quant()), ref(ctypes.c_size_t())) == BAD


def test_limits():
    assert size(cfg(window=512), qbatch(), attn(), quant())[0] == jacap.OK
    assert size(cfg(window=513), qbatch(), attn(), quant())[0] == UNSUP
    big = qbatch(num_seqs=60000, max_seq_len=1 << 24, total_tokens=1 << 24)
    assert size(cfg(window=512, num_q_heads=8), big, attn(), quant())[0] == UNSUP
    g = P(GOOD)
    w = lambda c, a: jacap._lib.jacap_attn_weights_quant(ref(c), ref(qbatch()), ref(a), ref(quant()), None, g, g, g, g,
                                                        None, None)
    assert w(cfg(), attn(causal=1)) == UNSUP and w(cfg(window=513), attn()) == UNSUP and w(cfg(), attn()) == BAD
    # no workspace for the sums of more rows than keep their logits
    long = qbatch(max_seq_len=96000, total_tokens=96000)
    assert size(cfg(window=30), long, attn(accumulate=1), quant())[1] == size(cfg(window=30), long, attn(), quant())[1]


def test_pointers():
    c, b, a, q = cfg(), qbatch(), attn(accumulate=1), quant()
    n = size(c, b, a, q)[1]
    lib = jacap._lib

    def attend(i=None, value=None, ws=P(GOOD), nbytes=n):
        args = [P(GOOD)] * 10      # q kq vq scales kd vd out lse acc acc_draft
        if i is not None:
            args[i] = value
        return lib.jacap_attend_quant(ref(c), ref(b), ref(a), ref(q), *args, ws, nbytes, None)

    for i in range(7):
        assert attend(i, None) == BAD
        assert attend(i, P(GOOD + 4)) == BAD
    for i in (7, 8, 9):
        assert attend(i, P(GOOD + 2)) == BAD
    assert attend(8, None) == BAD
    assert attend(ws=None) == BAD and attend(ws=P(GOOD + 128)) == BAD
    assert attend(nbytes=n - 1) == jacap.ERR_WORKSPACE

    def quantize(i, value):
        args = [P(GOOD)] * 6       # k v acc kq vq scales
        args[i] = value
        return lib.jacap_quantize(ref(c), ref(b), ref(a), ref(q), *args, None)

    for i in (0, 1, 3, 4, 5):
        assert quantize(i, None) == BAD and quantize(i, P(GOOD + 4)) == BAD
    assert quantize(2, P(GOOD + 2)) == BAD

    def append(i, value, cap=4):
        args = [P(GOOD)] * 6 + [cap] + [P(GOOD)] * 7   # kd vd start count rows slots cap kq vq scales acc draft out status
        args[i] = value
        return lib.jacap_append_quant(ref(c), ref(b), ref(a), ref(q), *args, None)

    for i in (0, 1, 7, 8, 9):
        assert append(i, None) == BAD and append(i, P(GOOD + 4)) == BAD
    for i in (2, 3, 4, 5, 10, 11, 12, 13):
        assert append(i, P(GOOD + 2)) == BAD
    assert append(6, -1) == BAD
    assert lib.jacap_append_quant(ref(c), ref(b), ref(a), ref(q), P(GOOD), P(GOOD), None, None, None, None, 0, P(GOOD),
                                  P(GOOD), P(GOOD), None, None, None, None, None) == BAD   # neither start nor slots

    def weights(i, value):
        args = [P(GOOD)] * 6       # q kq scales lse acc status
        args[i] = value
        return lib.jacap_attn_weights_quant(ref(c), ref(b), ref(a), ref(q), *args, None)

    for i in range(5):
        assert weights(i, None) == BAD
    for i in range(6):
        assert weights(i, P(GOOD + 2)) == BAD


def ver(**kw):
    v = jacap.Verification(2, 5, 1000, 1, 1.0, 0, 5000, 1000, 5000, 1000)
    for k, x in kw.items():
        setattr(v, k, x)
    return v


def vsize(v):
    n = ctypes.c_size_t(0)
    return jacap._lib.jacap_verify_workspace_size(ref(v), ref(n)), n.value


def test_verification():
    code, n = vsize(ver())
    assert code == jacap.OK and n >= 256 and n % 256 == 0
    nan, inf = float("nan"), float("inf")
    for v in (ver(num_seqs=0), ver(rows=0), ver(vocab=0), ver(temperature=-1.0), ver(temperature=nan),
              ver(temperature=inf), ver(temperature=1e-44), ver(reserved=1), ver(l_stride_seq=-1), ver(l_stride_row=-1),
              ver(q_stride_seq=-1), ver(q_stride_row=-1), ver(parents=0x1002)):
        assert vsize(v)[0] == BAD
    for v in (ver(dtype=2), ver(rows=513), ver(vocab=(1 << 24) + 1), ver(num_seqs=1 << 24, rows=512)):
        assert vsize(v)[0] == UNSUP
    for v in (ver(temperature=0.0), ver(vocab=1 << 24), ver(rows=512), ver(l_stride_row=0, l_stride_seq=3)):
        assert vsize(v)[0] == jacap.OK
    lib = jacap._lib
    assert lib.jacap_verify_workspace_size(None, ref(ctypes.c_size_t())) == BAD
    assert lib.jacap_verify_workspace_size(ref(ver()), None) == BAD

    def call(i=None, value=None, v=ver(), ws=P(GOOD), nbytes=n):
        args = [P(GOOD)] * 8       # logits tokens uniform draft path count next row_weight
        if i is not None:
            args[i] = value
        return lib.jacap_verify(ref(v), *args, ws, nbytes, None)

    for i in (0, 1, 2, 4, 5, 6):
        assert call(i, None) == BAD
    for i in range(1, 8):
        assert call(i, P(GOOD + 2)) == BAD
    assert call(0, P(GOOD + 1)) == BAD
    assert call(0, P(GOOD + 2), v=ver(dtype=0)) == BAD
    assert call(ws=None) == BAD and call(ws=P(GOOD + 8)) == BAD
    assert call(nbytes=n - 1) == jacap.ERR_WORKSPACE

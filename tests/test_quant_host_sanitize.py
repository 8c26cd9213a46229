"""The host layers of the 8-bit cache and of the verification of drafted tokens (argument
validation, workspace layouts and grids of quant_host.hip and verify_host.hip) built for the
CPU with AddressSanitizer and UndefinedBehaviorSanitizer and driven
(tests/sanitize/quant_driver.cpp) against host-only stand-ins for the launchers. No GPU is
used: only host code is instrumented."""

import os
import subprocess

import pytest

from test_attention_host_sanitize import CLANG, CSRC, HIPCC, ROOT, SAN


@pytest.mark.skipif(not (os.path.exists(HIPCC) and os.path.exists(CLANG)), reason="no ROCm toolchain")
def test_quant_and_verify_host_layers_under_asan_ubsan(tmp_path):
    flags = ["-O1", "-g", "-std=c++17", "--offload-host-only", "-x", "hip",
             "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
             "-Xarch_host", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer",
             f"-I{os.path.join(ROOT, 'include')}", f"-I{CSRC}", f"-I{SAN}"]
    objs = []
    for src in [os.path.join(CSRC, f) for f in ("jacap_host.hip", "attention_host.hip", "quant_host.hip",
                                                "verify_host.hip")] + \
            [os.path.join(SAN, f) for f in ("launch_stubs.cpp", "attention_stubs.cpp", "quant_driver.cpp")]:
        obj = str(tmp_path / (os.path.basename(src) + ".o"))
        r = subprocess.run([HIPCC, *flags, "-c", src, "-o", obj], capture_output=True, text=True)
        assert r.returncode == 0, r.stdout + r.stderr
        objs.append(obj)
    exe = str(tmp_path / "quant_check")
    r = subprocess.run([CLANG, "-fsanitize=address,undefined", "-fno-sanitize-recover=all", *objs, "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stdout + r.stderr
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "ok under the sanitizers" in r.stdout
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr

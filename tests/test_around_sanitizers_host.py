"""Host sanitizer run (no GPU needed) of the operators around the attention: their
entry points' argument checks and workspace sizes, built with AddressSanitizer and
UndefinedBehaviorSanitizer and driven by tests/sanitize/around_check.cpp."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_33591_amd", "csrc")
BUILD = os.path.join(ROOT, "paper_2609_33591_amd", "_build")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
# the device code's objects, as build() leaves them (not sanitized)
OBJS = [os.path.join(BUILD, n) for n in ("kia_fwd.o", "kia_bwd.o", "kia_bf16.o", "kia_around_1.o",
                                         "kia_around_2.o", "kia_window.o", "kia_cached.o")]


def run(cmd, **kw):
    res = subprocess.run(cmd, capture_output=True, text=True, **kw)
    assert res.returncode == 0, f"{' '.join(cmd)}\n{res.stdout}\n{res.stderr[-4000:]}"
    return res


def test_host_code_under_address_and_undefined_sanitizers(tmp_path):
    if not os.path.exists(HIPCC) or not all(os.path.exists(o) for o in OBJS):
        pytest.skip("hipcc or the kernel objects of build() are missing")
    comp = [HIPCC, "-O1", "-g", "-std=c++17", "--offload-arch=gfx950", "-munsafe-fp-atomics",
            "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
            "-Xarch_host", "-fno-omit-frame-pointer", "-I" + os.path.join(ROOT, "include"),
            "-I" + CSRC]
    own = []
    for src in (os.path.join(CSRC, "kia_around_abi.hip"), os.path.join(CSRC, "kia_abi.hip"),
                os.path.join(ROOT, "tests", "sanitize", "around_check.cpp")):
        own.append(str(tmp_path / (os.path.basename(src) + ".o")))
        run([*comp, "-c", src, "-o", own[-1]])
    exe = str(tmp_path / "around_check")
    run([HIPCC, "--offload-arch=gfx950", "-fsanitize=address", "-fsanitize=undefined",
         "-fno-gpu-sanitize", *own, *OBJS, "-o", exe])
    res = run([exe], env=dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0",
                              UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1"))
    assert "around host sanitizer run: ok" in res.stdout
    assert "runtime error" not in res.stderr and "AddressSanitizer" not in res.stderr

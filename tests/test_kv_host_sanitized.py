"""The attention block's host code (csrc/mdbf_kv.hip, csrc/mdbf_kv_attn.hip: checks, the choice of kernel, workspace sizes, grids) compiled without its
kernels, with AddressSanitizer and UndefinedBehaviorSanitizer, linked into a standalone driver (tests/host_kv_driver.cpp) whose
HIP entry points go nowhere, and run with sizes up to 2^31 - 1.  No GPU, no HIP runtime, no Python in the sanitized process."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2512_24545_amd", "csrc")


def test_host_code_of_the_attention_block_under_sanitizers(tmp_path):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    clang = "/opt/rocm/lib/llvm/bin/clang++"
    if not (os.path.exists(hipcc) and os.path.exists(clang)):
        pytest.skip("no ROCm toolchain")
    include = ["-I", os.path.join(ROOT, "include"), "-I", CSRC]
    objs = []
    for name in ("mdbf_kv", "mdbf_kv_attn"):
        objs.append(str(tmp_path / (name + ".o")))
        subprocess.run([hipcc, "-O1", "-g", "-std=c++17", "-fPIC", "--offload-arch=gfx950", "--cuda-host-only", "-w", "-Xarch_host", "-fsanitize=address",
                        "-Xarch_host", "-fsanitize=undefined", *include, "-c", os.path.join(CSRC, name + ".hip"), "-o", objs[-1]],
                       check=True, capture_output=True)
    exe = str(tmp_path / "kv_driver")
    # (the kernels' binaries are what stays unresolved)
    subprocess.run([clang, "-O1", "-g", "-std=c++17", "-fsanitize=address,undefined", "-fno-omit-frame-pointer", *include,
                    os.path.join(ROOT, "tests", "host_kv_driver.cpp"), *objs, "-Wl,--unresolved-symbols=ignore-in-object-files", "-o", exe],
                   check=True, capture_output=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    report = r.stdout[-3000:] + r.stderr[-6000:]
    assert r.returncode == 0, report
    assert "AddressSanitizer" not in r.stderr and "runtime error" not in r.stderr, report
    assert r.stdout.strip().endswith("ok"), report

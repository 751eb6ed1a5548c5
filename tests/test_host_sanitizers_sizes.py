"""Host code of the paged-cache operators at their largest sizes under UndefinedBehaviorSanitizer, without a GPU (none is visible to the
program, which ends if one is): tests/host_sanitize_sizes.c against the sources with the sanitizer on the host side only."""
import os
import subprocess

import pytest

from paper_2406_17276_amd import build as B

SAN = ["-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=undefined"]
STUB = "namespace ot { void set_last_hip_error(int) {} }\n"


@pytest.mark.timeout(900)
def test_no_host_arithmetic_overflows_at_the_largest_sizes(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    clang = os.path.join(rocm, "lib", "llvm", "bin", "clang")
    if not (os.path.exists(hipcc) and os.path.exists(clang)):
        pytest.skip("no ROCm compiler")
    (tmp_path / "stub.hip").write_text(STUB)
    procs, objs = [], []
    for src in [os.path.join(B.CSRC, "qk_rope.hip"), os.path.join(B.CSRC, "paged_append.hip"), str(tmp_path / "stub.hip")]:
        objs.append(str(tmp_path / (os.path.basename(src) + ".o")))
        flags = [f for f in B.FLAGS if f != "-O3"] + ["-O1", "-Xarch_device", "-O0"] + SAN
        procs.append(subprocess.Popen([hipcc] + flags + ["-c", src, "-o", objs[-1]], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True))
    for pr in procs:
        out, _ = pr.communicate()
        assert pr.returncode == 0, out[-3000:]
    exe, lib_dir = str(tmp_path / "host_sanitize_sizes"), os.path.join(rocm, "lib")
    main = str(tmp_path / "main.o")
    subprocess.run([clang, "-std=c11", "-O1", "-D__HIP_PLATFORM_AMD__", "-I" + os.path.join(B.ROOT, "include"), "-I" + os.path.join(rocm, "include"), "-c",
                    os.path.join(B.ROOT, "tests", "host_sanitize_sizes.c"), "-o", main], check=True)
    subprocess.run([clang + "++", "-fsanitize=undefined", main] + objs + ["-o", exe, "-L" + lib_dir, "-lamdhip64", "-Wl,-rpath," + lib_dir], check=True)
    env = dict(os.environ, HIP_VISIBLE_DEVICES="-1", ROCR_VISIBLE_DEVICES="-1", UBSAN_OPTIONS="print_stacktrace=1")
    run = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=env, timeout=300)
    if run.returncode == 2:
        pytest.skip("a GPU is visible")
    assert "runtime error" not in run.stdout, run.stdout[-4000:]
    assert run.returncode == 0 and run.stdout.strip().splitlines()[-1] == "ok", run.stdout[-4000:]

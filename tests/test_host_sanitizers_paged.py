"""The host code of the operators around a paged cache under AddressSanitizer + UndefinedBehaviorSanitizer, without a GPU: their
sources once more with the sanitizers on the host side only, and tests/host_sanitize_paged.c against them."""
import os
import subprocess

import pytest

from paper_2406_17276_amd import build as B

SAN = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-omit-frame-pointer"]
SOURCES = ["api.hip", "row_scan.hip", "tree_build.hip", "build_fused.hip", "tree_select.hip", "tree_expand.hip", "qk_rope.hip", "paged_append.hip", "paged_attn.hip"]


@pytest.mark.timeout(900)
def test_host_paths_are_clean_under_asan_and_ubsan(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    clang = os.path.join(rocm, "lib", "llvm", "bin", "clang")
    if not (os.path.exists(hipcc) and os.path.exists(clang)):
        pytest.skip("no ROCm compiler")
    procs, objs = [], []
    for src in SOURCES:
        obj = str(tmp_path / src.replace(".hip", ".o"))
        objs.append(obj)
        flags = [f for f in B.FLAGS if f != "-O3"] + ["-O1", "-Xarch_device", "-O3", "-Xarch_device", "-O0"] + SAN
        procs.append(subprocess.Popen([hipcc] + flags + B.EXTRA_FLAGS.get(src, []) + ["-c", os.path.join(B.CSRC, src), "-o", obj],
                                      stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True))
    for pr in procs:
        out, _ = pr.communicate()
        assert pr.returncode == 0, out[-3000:]
    lib = str(tmp_path / "libopttree_san.so")
    subprocess.run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", "-fsanitize=address,undefined", "-o", lib] + objs, check=True)
    exe = str(tmp_path / "host_sanitize_paged")
    lib_dir = os.path.join(rocm, "lib")
    subprocess.run([clang, "-std=c11", "-O1", "-g", "-fsanitize=address,undefined", "-fno-omit-frame-pointer", "-D__HIP_PLATFORM_AMD__",
                    "-I" + os.path.join(B.ROOT, "include"), os.path.join(B.ROOT, "tests", "host_sanitize_paged.c"), "-o", exe, "-L" + str(tmp_path),
                    "-lopttree_san", "-L" + lib_dir, "-lamdhip64", "-Wl,-rpath," + str(tmp_path), "-Wl,-rpath," + lib_dir], check=True)
    env = dict(os.environ, ASAN_OPTIONS="verify_asan_link_order=0:detect_leaks=0", UBSAN_OPTIONS="print_stacktrace=1")
    run = subprocess.run([exe], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, env=env, timeout=600)
    assert "runtime error" not in run.stdout and "AddressSanitizer" not in run.stdout, run.stdout[-4000:]
    assert run.returncode == 0 and run.stdout.strip().splitlines()[-1].startswith("ok "), run.stdout[-4000:]

"""The launch plans of tree attention under AddressSanitizer and UndefinedBehaviorSanitizer, and every launch that they make against what the kernels
assume of it: each work item once, pieces that have keys, partial results inside the workspace and where the merge looks for them.

The planning stands beside the kernels' launches in csrc/cs_tree.hip, which is compiled here for the host alone; tests/host_sanitize/tree_driver.cpp is the
runtime that it launches on.  No GPU is needed."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2410_01228_amd", "csrc")
HERE = os.path.join(ROOT, "tests", "host_sanitize")
CLANG = "/opt/rocm/lib/llvm/bin/clang++"


@pytest.mark.skipif(shutil.which("hipcc") is None or not os.path.exists(CLANG), reason="no ROCm toolchain")
def test_tree_plans_and_their_launches(tmp_path):
    san = ["-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-fno-omit-frame-pointer", "-O1", "-g", "-std=c++17"]
    inc = ["-I", os.path.join(ROOT, "include"), "-I", CSRC, "-I", HERE]
    objs = []
    for src in (os.path.join(CSRC, "cs_tree.hip"), os.path.join(CSRC, "cs_api.hip"), os.path.join(HERE, "stubs.hip"), os.path.join(HERE, "tree_driver.cpp")):
        objs.append(str(tmp_path / (os.path.basename(src) + ".o")))
        subprocess.run(["hipcc", "--offload-arch=gfx950", "--cuda-host-only", "-fPIC", *san, *inc, "-x", "hip", "-c", src, "-o", objs[-1]], check=True, stdout=subprocess.DEVNULL,
                       stderr=subprocess.DEVNULL)
    # the device code that the host part would register is not there
    undefined = subprocess.run(["nm", "-u", objs[0]], check=True, capture_output=True, text=True).stdout
    binary = ["-Wl,--defsym=%s=0" % s for s in re.findall(r"__hip_fatbin\w*", undefined)]
    exe = str(tmp_path / "driver")
    subprocess.run([CLANG, "-fsanitize=address,undefined", "-no-pie", *objs, *binary, "-L/opt/rocm/lib", "-lamdhip64", "-Wl,-rpath,/opt/rocm/lib", "-o", exe], check=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    run = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert run.returncode == 0, run.stdout[-2000:] + run.stderr[-4000:]
    assert run.stdout.startswith("ok ") and "runtime error" not in run.stderr and "AddressSanitizer" not in run.stderr, run.stdout + run.stderr[-4000:]

"""Every plan of the biased attention's host code against what the kernels take
from it (tests/asan/plan_check.cpp), under AddressSanitizer and
UndefinedBehaviorSanitizer, built as in test_asan_host.  No GPU is used."""
import os
import subprocess

import pytest

from test_asan_host import CLANGXX, HERE, HIPCC, ROCM, ROOT, _run


def test_partitions_reach_every_visible_token(tmp_path):
    if not (os.path.exists(HIPCC) and os.path.exists(CLANGXX)):
        pytest.skip("ROCm compilers not found")
    csrc = os.path.join(ROOT, "paper_2510_14126_amd", "csrc")
    inc = ["-I", os.path.join(ROOT, "include"), "-I", csrc]
    host_hip = [HIPCC, "-x", "hip", "--offload-host-only", "--offload-arch=gfx950", "-O1", "-g", "-std=c++17",
                "-fno-omit-frame-pointer", "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
                "-Xarch_host", "-fno-sanitize-recover=all", *inc]
    objs = []
    for src in (os.path.join(csrc, "api.cpp"), os.path.join(csrc, "api_ops.cpp"),
                os.path.join(HERE, "asan", "launch_stubs.cpp"), os.path.join(HERE, "asan", "plan_check.cpp")):
        objs.append(os.path.basename(src).replace(".cpp", ".o"))
        _run(host_hip + ["-c", src, "-o", objs[-1]], tmp_path)
    lib = os.path.join(ROCM, "lib")
    _run([CLANGXX, "-fsanitize=address,undefined", "-fno-sanitize-recover=all", *objs, "-L", lib, "-lamdhip64",
          f"-Wl,-rpath,{lib}", "-o", "plan_check"], tmp_path)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([str(tmp_path / "plan_check")], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0, r.stdout + r.stderr
    assert "plans hold" in r.stdout
    assert "Sanitizer" not in r.stderr, r.stderr

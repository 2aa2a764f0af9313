"""Host code of the streamed layer's entry points under AddressSanitizer and UndefinedBehaviorSanitizer, over arguments of any size, without the HIP
runtime (tests/hostglue/check_stream.cpp has stubs for it): no GPU is needed, and none is used where there is one."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2509_07120_amd", "csrc")


def test_arguments_of_any_size(tmp_path):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    sanitize = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=undefined"]
    flags = [hipcc, "--offload-arch=gfx950", "--cuda-host-only", "-O1", "-g", "-std=c++17", *sanitize, "-fno-omit-frame-pointer",
             "-Wno-unused-command-line-argument", "-I", os.path.join(ROOT, "include"), "-I", CSRC]
    sources = [os.path.join(CSRC, f + ".hip") for f in ("norm_rope", "window", "window_bwd", "paged")]
    sources.append(os.path.join(ROOT, "tests", "hostglue", "check_stream.cpp"))
    jobs = []
    for s in sources:
        o = str(tmp_path / (os.path.basename(s) + ".o"))
        jobs.append((o, subprocess.Popen(flags + (["-x", "hip"] if s.endswith(".cpp") else []) + ["-c", s, "-o", o], stderr=subprocess.PIPE, text=True)))
    for o, job in jobs:
        err = job.communicate()[1]
        assert job.returncode == 0, err[-3000:]
    exe = str(tmp_path / "check_stream")  # (the images for the GPU are not built; nobody reads them)
    link = subprocess.run([hipcc, *sanitize, "-Wl,--unresolved-symbols=ignore-all", *[o for o, _ in jobs], "-o", exe], capture_output=True, text=True)
    assert link.returncode == 0, link.stderr[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    run = subprocess.run([exe, "2000"], capture_output=True, text=True, env=env, timeout=300)
    assert run.returncode == 0, (run.stdout[-2000:], run.stderr[-4000:])
    assert " 0 failed checks" in run.stdout and "runtime error" not in run.stderr, run.stdout

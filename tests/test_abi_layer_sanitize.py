"""The layer operators' host code under AddressSanitizer and UndefinedBehaviorSanitizer: their sources are rebuilt
with both sanitizers on the host code only (device code unchanged), side by side, and
tests/sanitize/abi_layer_sanitize.c, linked against them, calls every workspace-size function at extreme sizes and
the entry points with arguments that the host rejects before any HIP call. No GPU is used."""

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
SOURCES = ["layer_api", "causal_conv", "selective_scan", "residual_norm", "part_sums"]


def test_layer_host_code_clean_under_sanitizers(tmp_path):
    hipcc = os.path.join(ROCM, "bin", "hipcc")
    clang = os.path.join(ROCM, "llvm", "bin", "clang++")
    if not (os.path.exists(hipcc) and os.path.exists(clang)):
        pytest.skip("ROCm compilers not installed")
    flags = ["-O1", "-g", "-std=c++17", "--offload-arch=gfx950", "-fPIC", "-fvisibility=hidden",
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
             "-Xarch_host", "-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "include")]
    jobs = []
    for name in SOURCES:
        src = os.path.join(ROOT, "paper_2508_01073_amd", "csrc", name + ".hip")
        log = open(tmp_path / (name + ".log"), "w+")
        jobs.append((subprocess.Popen([hipcc, *flags, "-c", src, "-o", str(tmp_path / (name + ".o"))], stdout=log,
                                      stderr=subprocess.STDOUT), log))
    for job, log in jobs:
        code = job.wait(timeout=900)
        log.seek(0)
        assert code == 0, log.read()[-4000:]
    objects = [str(tmp_path / (name + ".o")) for name in SOURCES]
    main = str(tmp_path / "main.o")
    sanitize = ["-fsanitize=address,undefined", "-fno-sanitize-recover=all"]
    for step in ([shutil.which("clang", path=os.path.dirname(clang)) or clang, "-std=c99", "-Wall", "-Wextra", "-Werror",
                  "-g", *sanitize, "-I", os.path.join(ROOT, "include"), "-c",
                  os.path.join(ROOT, "tests", "sanitize", "abi_layer_sanitize.c"), "-o", main],
                 [clang, *sanitize, main, *objects, "-L", os.path.join(ROCM, "lib"), "-lamdhip64",
                  f"-Wl,-rpath,{os.path.join(ROCM, 'lib')}", "-o", str(tmp_path / "abi_layer")]):
        done = subprocess.run(step, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
        assert done.returncode == 0, done.stdout[-4000:]
    # leaks are not checked: the HIP runtime keeps its own allocations until exit
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:verify_asan_link_order=0", UBSAN_OPTIONS="print_stacktrace=1")
    run = subprocess.run([str(tmp_path / "abi_layer")], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True,
                         timeout=300, env=env)
    assert run.returncode == 0, run.stdout[-4000:]
    assert "abi layer sanitize: ok" in run.stdout

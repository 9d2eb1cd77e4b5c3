"""AddressSanitizer + UndefinedBehaviorSanitizer on the host code of the attention operators (validation, plans, workspace
sizes; no kernel is launched).  Needs no GPU.  Sanitizers run on host code only."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2405_03133_amd", "csrc")
FILES = ("attn_api", "kv_plan", "paged_attn", "qk_rope", "qk_rope_bwd", "profile")


@pytest.mark.timeout(900)
def test_attention_host_layer_under_asan_ubsan(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    flags = ["--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fno-gpu-rdc",
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-Wno-unused-command-line-argument",
             "-w", "-I", os.path.join(ROOT, "include"), "-I", CSRC, "-Xarch_host", "-fsanitize=address",
             "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=undefined"]
    jobs = [(os.path.join(CSRC, f + ".hip"), str(tmp_path / (f + ".o"))) for f in FILES]
    jobs.append((os.path.join(ROOT, "tests", "host_sanitize", "attn_driver.cpp"), str(tmp_path / "driver.o")))
    procs = [subprocess.Popen([hipcc] + flags + (["-x", "hip"] if src.endswith(".cpp") else []) + ["-c", src, "-o", obj],
                              stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True) for src, obj in jobs]
    for (src, _), proc in zip(jobs, procs):
        out, _ = proc.communicate()
        assert proc.returncode == 0, (src, out[-4000:])
    exe = str(tmp_path / "driver")
    link = subprocess.run([hipcc, "--offload-arch=gfx950", "-fno-gpu-rdc", "-fsanitize=address", "-fsanitize=undefined",
                           "-fno-gpu-sanitize"] + [obj for _, obj in jobs] + ["-o", exe], stdout=subprocess.PIPE,
                          stderr=subprocess.STDOUT, text=True)
    assert link.returncode == 0, link.stdout[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:verify_asan_link_order=0:abort_on_error=0",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    run = subprocess.run([exe], env=env, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    print(run.stdout[-4000:])
    assert run.returncode == 0 and "attention abi sanitizer run: ok" in run.stdout, run.stdout[-4000:]
    for marker in ("AddressSanitizer", "runtime error", "FAILED"):
        assert marker not in run.stdout, run.stdout[-4000:]

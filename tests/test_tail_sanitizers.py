"""The trained tail's host code under AddressSanitizer and UBSan: argument checks, tile
rules and the workspace's layout from one row to the largest sizes, with stand-ins for
the kernel launchers that check each scratch region's place."""

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SAN = os.path.join(ROOT, "tests", "sanitize")
CSRC = os.path.join(ROOT, "paper_2210_08650_amd", "csrc")
ENV = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:halt_on_error=1",
           UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")


def _run(cmd, **kw):
    r = subprocess.run(cmd, capture_output=True, text=True, **kw)
    assert r.returncode == 0, f"{' '.join(cmd[:3])} ...: rc {r.returncode}\n{r.stdout[-3000:]}\n{r.stderr[-3000:]}"
    return r


def test_tail_host_code_under_asan_ubsan(tmp_path):
    hipcc = next((c for c in ("/opt/rocm/bin/hipcc", shutil.which("hipcc") or "") if c and os.path.exists(c)), None)
    if not hipcc:
        pytest.skip("hipcc not found")
    sanitize = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined"]
    flags = ["-x", "hip", "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-I", os.path.join(ROOT, "include"),
             "-I", CSRC] + sanitize + ["-Xarch_host", "-fno-omit-frame-pointer", "-Wno-unused-result"]
    objs = []
    for src in (os.path.join(CSRC, "api.cpp"), os.path.join(CSRC, "split.cpp"), os.path.join(CSRC, "tail.cpp"),
                os.path.join(SAN, "stubs.cpp"), os.path.join(SAN, "tail_driver.cpp")):
        o = str(tmp_path / (os.path.basename(src) + ".o"))
        _run([hipcc] + flags + ["-c", src, "-o", o])
        objs.append(o)
    exe = str(tmp_path / "tail_driver")
    _run([hipcc, "--offload-arch=gfx950"] + sanitize + objs + ["-o", exe])
    r = _run([exe], env=ENV, timeout=300)
    assert r.stdout.startswith("OK "), r.stdout
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr, r.stderr[-3000:]

"""The trained block's host code under AddressSanitizer and UBSan: argument checks, split
rules and the workspace's layout from no token to the largest sizes, with stand-ins for
the kernel launchers that check each scratch region's place."""
import os
import shutil

import pytest

from tests.test_tail_sanitizers import CSRC, ENV, ROOT, SAN, _run


def test_block_host_code_under_asan_ubsan(tmp_path):
    hipcc = next((c for c in ("/opt/rocm/bin/hipcc", shutil.which("hipcc") or "") if c and os.path.exists(c)), None)
    if not hipcc:
        pytest.skip("hipcc not found")
    sanitize = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined"]
    flags = ["-x", "hip", "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-I", os.path.join(ROOT, "include"),
             "-I", CSRC] + sanitize + ["-Xarch_host", "-fno-omit-frame-pointer", "-Wno-unused-result"]
    objs = []
    for src in (os.path.join(CSRC, "api.cpp"), os.path.join(CSRC, "split.cpp"), os.path.join(CSRC, "block.cpp"),
                os.path.join(SAN, "stubs.cpp"), os.path.join(SAN, "block_driver.cpp")):
        o = str(tmp_path / (os.path.basename(src) + ".o"))
        _run([hipcc] + flags + ["-c", src, "-o", o])
        objs.append(o)
    exe = str(tmp_path / "block_driver")
    _run([hipcc, "--offload-arch=gfx950"] + sanitize + objs + ["-o", exe])
    r = _run([exe], env=ENV, timeout=300)
    assert r.stdout.startswith("OK "), r.stdout
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr, r.stderr[-3000:]

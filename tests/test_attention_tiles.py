"""The cross attention's walk over tiles of keys, on the host under AddressSanitizer and UBSan."""
import os
import shutil

import pytest

from tests.test_tail_sanitizers import CSRC, ENV, ROOT, SAN, _run


def test_a_tile_has_the_bits_of_its_own_keys(tmp_path):
    hipcc = next((c for c in ("/opt/rocm/bin/hipcc", shutil.which("hipcc") or "") if c and os.path.exists(c)), None)
    if not hipcc:
        pytest.skip("hipcc not found")
    sanitize = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined"]
    exe, obj = str(tmp_path / "attend_driver"), str(tmp_path / "attend_driver.o")
    _run([hipcc, "-x", "hip", "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-I", os.path.join(ROOT, "include"), "-I", CSRC] + sanitize +
         ["-Xarch_host", "-fno-omit-frame-pointer", "-Wno-unused-result", "-c", os.path.join(SAN, "attend_driver.cpp"), "-o", obj])
    _run([hipcc, "--offload-arch=gfx950"] + sanitize + [obj, "-o", exe])
    r = _run([exe], env=ENV, timeout=120)
    assert r.stdout.startswith("OK "), r.stdout
    assert "runtime error" not in r.stderr and "AddressSanitizer" not in r.stderr, r.stderr[-3000:]

"""The calls that fill caches and those of 4-bit caches from C: struct layouts as the Python
binding declares them, refusals (no GPU needed)."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2605_31457_amd import vp

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2605_31457_amd")


@pytest.mark.skipif(shutil.which("gcc") is None, reason="gcc not available")
def test_c_client(tmp_path):
    if not os.path.exists(os.path.join(PKG, "libvisionpulse.so")):
        pytest.skip("library not built")
    exe = tmp_path / "kv4_smoke"
    r = subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"),
                        os.path.join(ROOT, "tests", "c", "kv4_smoke.c"), "-L", PKG, "-lvisionpulse", f"-Wl,-rpath,{PKG}",
                        "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "all checks passed" in r.stdout, r.stdout + r.stderr
    size, off = ctypes.sizeof, lambda t, f: getattr(t, f).offset
    assert (f"vp_rope {size(vp.vp_rope)} {off(vp.vp_rope, 'pos')} {off(vp.vp_rope, 'section')}, "
            f"vp_tokens {size(vp.vp_tokens)} {off(vp.vp_tokens, 'n_tokens')}, "
            f"vp_kv4 {size(vp.vp_kv4)} {off(vp.vp_kv4, 'scale_stride_h')}\n") in r.stdout

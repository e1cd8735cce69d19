"""The way of a batch with a window or over 4-bit pools, as the host chooses it: what a bound on the lengths changes the device would find by itself,
so rows do not depend on the bound (no GPU)."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2602_11530_amd", "csrc")


def test_the_bound_decides_nothing_that_the_device_would_not(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    exe = str(tmp_path / "span_route_check")
    subprocess.check_call([hipcc, "-O1", "-std=c++17", "--offload-arch=gfx950", "-x", "hip", "-I", CSRC,
                           os.path.join(ROOT, "tests", "span_route_check.cpp"), os.path.join(CSRC, "pkv_api_span.hip"), "-o", exe],
                          stderr=subprocess.DEVNULL)
    out = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and "wrong=0" in out.stdout, out.stdout

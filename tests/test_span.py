"""The units and tokens that a window and sinks leave of a request, against the definition (no GPU)."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_units_and_tokens(tmp_path):
    hipcc = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
    exe = str(tmp_path / "span_check")
    subprocess.check_call([hipcc, "-O1", "-std=c++17", "--offload-arch=gfx950", "-x", "hip", "-I",
                           os.path.join(ROOT, "paper_2602_11530_amd", "csrc"), os.path.join(ROOT, "tests", "span_check.cpp"), "-o", exe],
                          stderr=subprocess.DEVNULL)
    out = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert out.returncode == 0 and "wrong=0" in out.stdout, out.stdout

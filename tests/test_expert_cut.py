"""The cut of the experts' factors, counted on the CPU (expert_cut_check.cpp)."""
import os
import subprocess

HERE = os.path.dirname(os.path.abspath(__file__))


def test_ranges_and_scratch_cover_whatever_rows_the_experts_get(tmp_path):
    exe = str(tmp_path / "expert_cut_check")
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "-x", "hip", "--offload-arch=gfx950", "--offload-host-only", "-std=c++17", "-O2",
                    "-I", os.path.join(HERE, "..", "include"), os.path.join(HERE, "expert_cut_check.cpp"), "-o", exe], check=True, capture_output=True)
    done = subprocess.run([exe], capture_output=True, text=True)
    assert done.returncode == 0 and done.stdout == "120000 cuts, 0 faults\n", done.stdout

"""What an epilogue's results may not lie over, decided before any device call (the driver's handle and addresses are made up)."""
import os
import shutil
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_results_over_a_handles_arrays_are_refused(tmp_path):
    from paper_2007_13055_amd import binding
    if not os.path.exists(binding.library_path()):
        from paper_2007_13055_amd import build
        build.build()
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    exe = str(tmp_path / "host_epilogue_driver")
    subprocess.run([hipcc, "--offload-arch=gfx950", "-O1", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                    "-Wno-unused-command-line-argument", "-I", os.path.join(ROOT, "include"),
                    "-I", os.path.join(ROOT, "paper_2007_13055_amd", "csrc"), os.path.join(ROOT, "tests", "host_epilogue_driver.cpp"),
                    "-L", os.path.dirname(binding.library_path()), "-l:libbsr_spmm.so", "-Wl,-rpath," + os.path.dirname(binding.library_path()), "-o", exe],
                   check=True, capture_output=True, timeout=600)
    out = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert out.returncode == 0, out.stdout + out.stderr
    assert "all refused" in out.stdout

"""Numbers of rows beyond what offsets hold are refused whatever their size (no GPU)."""
import os
import shutil
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_rows_beyond_64_bits(tmp_path):
    from paper_2007_13055_amd import binding
    if not os.path.exists(binding.library_path()):
        from paper_2007_13055_amd import build
        build.build()
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    exe, folder = str(tmp_path / "host_rows_driver"), os.path.dirname(binding.library_path())
    subprocess.run([hipcc, "--offload-arch=gfx950", "-O1", "-std=c++17", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                    "-Wno-unused-command-line-argument", "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2007_13055_amd", "csrc"),
                    os.path.join(ROOT, "tests", "host_rows_driver.cpp"), "-L", folder, "-l:libbsr_spmm.so", "-Wl,-rpath," + folder, "-o", exe],
                   check=True, capture_output=True, timeout=600)
    out = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert out.returncode == 0 and "all refused" in out.stdout, out.stdout + out.stderr

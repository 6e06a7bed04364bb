"""What transfers along rows may read, on the host: tests/host/windows.hip compiled against the headers the kernels use."""
import os
import subprocess

from paper_2608_15592_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))


def test_windows_of_the_stages(tmp_path):
    exe = str(tmp_path / "windows")
    cmd = [build.hipcc(), f"--offload-arch={build.ARCH}", "-O1", "-std=c++17", f"-I{build.INCLUDE}", f"-I{build.CSRC}",
           os.path.join(HERE, "host", "windows.hip"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout + r.stderr

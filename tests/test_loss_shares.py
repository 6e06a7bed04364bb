"""How dX's vocabulary rows are shared out, on the host: tests/host/loss_shares.hip compiled against the header the
kernels use."""
import os
import subprocess

from paper_2608_15592_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))


def test_shares_of_the_vocabulary(tmp_path):
    exe = str(tmp_path / "loss_shares")
    cmd = [build.hipcc(), f"--offload-arch={build.ARCH}", "-O1", "-std=c++17", f"-I{build.INCLUDE}", f"-I{build.CSRC}",
           os.path.join(HERE, "host", "loss_shares.hip"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout + r.stderr

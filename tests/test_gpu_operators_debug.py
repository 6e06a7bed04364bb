"""The library's debug mode (ESTP_DEBUG_CHECKS=1) in the calls on a cache: lens and cu_q are checked on the host
before any kernel reads them.  The mode is read once per process, so it runs in a child process, which confirms
first that the mode is on."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = r"""
import sys, torch
sys.path.insert(0, ROOT)
import paper_2608_15592_amd as estp
if estp.load().estp_debug_checks() != 1:
    print("debug checks are off"); sys.exit(3)
i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
Q = torch.randn(6, 4, 32, device="cuda")
K, V = (torch.randn(3, 2, 64, 32, device="cuda") for _ in range(2))
acc, pos = torch.zeros(3, 2, 64, device="cuda"), torch.zeros(3, 2, 64, dtype=torch.int32, device="cuda")
attend = lambda lens, cu: estp.tree_attention(Q, K, V, lens, cu, 3, 60, acc=acc)
O, lse = attend(i32(50, 0, 57), i32(0, 2, 2, 5))  # a sequence without rows, a row behind the last
credit = lambda lens, cu: estp.tree_importance(Q, K, lse, lens, cu, 3, 60, acc)
credit(i32(50, 0, 57), i32(0, 2, 2, 5))
good_l, good_c = (50, 40, 57), (0, 2, 5, 6)
bad = [(good_l, (1, 2, 5, 6)), (good_l, (0, 4, 5, 6)), (good_l, (0, 2, 1, 4)), (good_l, (0, 3, 6, 8)),
       ((50, -1, 57), good_c), ((59, 40, 57), good_c), ((50, 40, 2**31 - 1), good_c)]
for call in (attend, credit):
    for lens, cu in bad:
        try:
            call(i32(*lens), i32(*cu))
        except estp.EstpError as e:
            assert e.status == 1 and "debug check" in str(e), str(e)
            continue
        print(f"NOT refused: {lens} {cu}"); sys.exit(4)
seen = i32(60, 60, 60)
estp.cache_evict(K, V, acc, pos, i32(64, 0, 30), seen, 32)
for lens in ((65, 0, 30), (64, -1, 30)):
    try:
        estp.cache_evict(K, V, acc, pos, i32(*lens), seen, 32)
    except estp.EstpError as e:
        assert e.status == 1 and "debug check" in str(e), str(e)
        continue
    print(f"NOT refused: {lens}"); sys.exit(4)
torch.cuda.synchronize()
print("child ok")
"""


def test_debug_checks_refuse_malformed_lengths():
    env = dict(os.environ, ESTP_DEBUG_CHECKS="1")
    r = subprocess.run([sys.executable, "-c", CHILD.replace("ROOT", repr(ROOT))], cwd=ROOT, env=env,
                       capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "child ok" in r.stdout, r.stdout[-3000:] + r.stderr[-3000:]

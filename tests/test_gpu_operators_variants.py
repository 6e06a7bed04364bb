"""The kernels that a rule on sizes chooses only for larger calls, on the GPU against the fp64 oracle: cases on both
sides of each rule."""
import numpy as np
import pytest
import torch

import paper_2608_15592_amd as estp
from tests._util import dev, host
from tests.test_gpu_token_loss import _check_backward, _check_forward, _inputs
from tests.test_gpu_tree_attention import Case

pytestmark = pytest.mark.gpu


# fp32 tiles are 32, 64 or 128 tokens wide: by the token count, and 32 while 128-wide ones are fewer than 192 (V up to
# 24448 for one tile of tokens).  dW's tiles are 128 vocabulary rows wide from 192 tiles of 128 x 128 on, else 32.
F32 = [
    (32, 40, 24577), (33, 40, 24577), (50, 160, 24577), (64, 264, 24577),  # 32, then 64 wide
    (65, 40, 24577), (65, 40, 24448),                                      # 128 and 32 wide
    (129, 392, 16411),                                                     # 128 wide, dW of 4 column blocks, one ragged
    (300, 136, 8300),                                                      # 128 wide (3 x 65 tiles), dW 32 wide (2 x 65)
    (20, 520, 5000), (20, 512, 6100),                                      # dW: 5 x 40 tiles, and 4 x 48, the fewest
]


@pytest.mark.parametrize("n,d,V", F32)
def test_f32_tiles_of_every_width(n, d, V):
    X, W, t, g = _inputs(n + d + V, n, d, V, "f32", ignored=0.15)
    _check_backward(X, W, t, g, "f32", _check_forward(X, W, t, "f32"))


@pytest.mark.parametrize("n,d,V", [(384, 96, 1500), (385, 96, 1500), (700, 96, 5000), (700, 32, 66000),
                                   (2048, 160, 3001), (2049, 160, 3001), (2048, 128, 3001)])
def test_bf16_forward_on_both_sides_of_its_rules(n, d, V):
    # 128- and 256-token tiles at 384, the entropy kernels past 2048 tokens; depths of an odd and an even number of 32
    X, W, t, _ = _inputs(n + d, n, d, V, "bf16", ignored=0.1)
    _check_forward(X, W, t, "bf16")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,Hq", [(1, 4), (5, 4), (33, 2)])
def test_join_of_very_many_segments(dtype, T, Hq):
    # one KV head: all workgroups share its keys, and sixteen waves a row join what they leave, with the account or not
    c = Case(31, [70_000], [T], Hq, 1, 128, dtype)
    ref, acc = c.oracle(), dev(c.acc)
    O, lse = c.attend(acc=acc)
    c.check(O, lse, acc, ref)
    O2, lse2 = c.attend()
    assert torch.equal(O, O2) and torch.equal(lse, lse2)


def test_f32_loss_of_a_wide_call_repeats():
    X, W, t, g = _inputs(50, 50, 160, 24577, "f32", ignored=0.15)
    Xd, Wd, td, gd = dev(X), dev(W), dev(t), dev(g)
    lse = estp.token_loss(Xd, Wd, td)[1]
    first = estp.token_loss_backward(Xd, Wd, td, lse, gd)
    ws = torch.full((estp.load().estp_token_loss_backward_workspace_size(50, 160, 24577, 1),), 255, dtype=torch.uint8,
                    device="cuda")
    again = estp.token_loss_backward(Xd, Wd, td, lse, gd, workspace=ws)
    assert all(torch.equal(a, b) for a, b in zip(first, again))
    np.testing.assert_array_equal(host(lse), host(estp.token_loss(Xd, Wd, td)[1]))

"""The account that a prompt starts with, for every KV head of its own: importance of one KV head at a time."""
import numpy as np
import pytest

import oracle
import paper_2608_15592_amd as estp
from oracle import operators as OP
from synth import inputs as I
from tests._util import dev, host

pytestmark = pytest.mark.gpu

S_RTOL = 1e-3  # of the parity tests


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,dh", [(8, 2, 64), (6, 3, 128), (4, 4, 32)])
def test_a_prompts_account_head_by_head(Hq, Hkv, dh, dtype):
    g, n, G = np.random.default_rng(Hq + dh), [50, 13], Hq // Hkv
    cu = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
    Q, K = (g.standard_normal((cu[-1], h, dh)).astype(np.float32) for h in (Hq, Hkv))
    if dtype == "bf16":
        Q, K = I.f32_to_bf16_bits(Q), I.f32_to_bf16_bits(K)
    for h in range(Hkv):
        S = host(estp.attn_importance(dev(Q[:, h * G:(h + 1) * G]), dev(K[:, h:h + 1]), dev(cu), max(n)))
        for b, N in enumerate(n):
            at = slice(cu[b], cu[b + 1])
            # the weights that N drafted tokens in a chain give each other, which is the prompt
            k = np.ascontiguousarray(K[at, h:h + 1].transpose(1, 0, 2))[None]
            want = OP.tree_attention(Q[at, h * G:(h + 1) * G], k, k, [0], [0, N], dtype=dtype)["got"][0, 0]
            np.testing.assert_allclose(S[at] * N * G, want, rtol=S_RTOL)
    # and the average over all heads, which is one account for them all
    S = host(estp.attn_importance(dev(Q), dev(K), dev(cu), max(n)))
    ref = oracle.attn_importance(Q[None], K[None], cu)
    np.testing.assert_allclose(S, ref, rtol=S_RTOL)

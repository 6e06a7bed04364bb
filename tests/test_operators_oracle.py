"""The oracle of the loss, tree-attention and eviction calls, pinned by closed forms, by differences of the
loss and by pure-Python loops (CPU)."""
import math

import numpy as np
import pytest

import oracle
from oracle import operators as OP


def _head(seed, n, d, V):
    g = np.random.default_rng(seed)
    return g.standard_normal((n, d)), 0.3 * g.standard_normal((V, d)), g.integers(0, V, n), g.uniform(0.5, 2.0, n)


def test_loss_of_uniform_logits_is_ln_v():
    X, W = np.ones((3, 8)), np.tile(np.arange(8.0), (11, 1))
    loss, lse = OP.token_loss(X, W, [0, 5, 10])
    np.testing.assert_allclose(loss, math.log(11), rtol=1e-14)
    np.testing.assert_allclose(lse, 28.0 + math.log(11), rtol=1e-14)


def test_mean_loss_over_the_distribution_is_the_entropy():
    # sum_t P(t) loss(t) = H
    X, W, _, _ = _head(0, 1, 16, 9)
    losses = np.array([OP.token_loss(X, W, [t])[0][0] for t in range(9)])
    assert abs((np.exp(-losses) * losses).sum() - oracle.token_entropy(X, W)[0]) < 1e-13
    assert abs(np.exp(-losses).sum() - 1.0) < 1e-13


def test_ignored_tokens_have_no_loss_and_no_gradient():
    X, W, t, g = _head(1, 5, 8, 7)
    t[[1, 3]] = [-100, 7]
    loss, _ = OP.token_loss(X, W, t)
    assert loss[1] == loss[3] == 0.0 and (loss[[0, 2, 4]] > 0).all()
    dX, dW, _, _ = OP.token_loss_grads(X, W, t, g, "f32")
    live = [0, 2, 4]
    assert not dX[[1, 3]].any()
    np.testing.assert_allclose(dW, OP.token_loss_grads(X[live], W, t[live], g[live], "f32")[1], rtol=1e-13)


@pytest.mark.parametrize("n,d,V", [(1, 8, 1), (4, 8, 5), (3, 16, 12)])
def test_gradients_are_the_losses_differences(n, d, V):
    X, W, t, g = _head(2, n, d, V)
    dX, dW, bX, bW = OP.token_loss_grads(X, W, t, g, "f32")
    h = 1e-5
    for A, dA in ((X, dX), (W, dW)):
        for at in np.random.default_rng(3).integers(0, A.size, 25):
            i = np.unravel_index(at, A.shape)
            keep = A[i]
            A[i] = keep + h
            up = (g * OP.token_loss(X, W, t)[0]).sum()
            A[i] = keep - h
            down = (g * OP.token_loss(X, W, t)[0]).sum()
            A[i] = keep
            assert abs((up - down) / (2 * h) - dA[i]) < 1e-7
    assert (bX >= 0).all() and (bW >= 0).all()


def test_gradient_rows_sum_to_zero_over_the_vocabulary():
    # sum_v G_iv = 0, so equal weight rows leave no gradient in X
    X, W, t, g = _head(4, 6, 8, 9)
    W[:] = W[0]
    assert np.abs(OP.token_loss_grads(X, W, t, g, "f32")[0]).max() < 1e-14


def _cache(seed, B, T, lens, Hq, Hkv, dh, cap):
    g = np.random.default_rng(seed)
    cu = np.concatenate([[0], np.cumsum(T)])
    return (g.standard_normal((cu[-1], Hq, dh)), g.standard_normal((B, Hkv, cap, dh)),
            g.standard_normal((B, Hkv, cap, dh)), lens, cu)


def test_tree_attention_against_loops():
    B, T, lens, Hq, Hkv, dh, cap = 2, [3, 2], [4, 0], 4, 2, 8, 9
    Q, K, V, lens, cu = _cache(5, B, T, lens, Hq, Hkv, dh, cap)
    mask = [1, 0b11, 0b101, 0b1, 0b10]
    r = OP.tree_attention(Q, K, V, lens, cu, mask)
    got = np.zeros((B, Hkv, cap))
    for b in range(B):
        for t in range(T[b]):
            i = cu[b] + t
            for h in range(Hq):
                w = {}
                for j in range(lens[b] + T[b]):
                    if j < lens[b] or mask[i] >> (j - lens[b]) & 1:
                        w[j] = math.exp(sum(Q[i, h, c] * K[b, h // 2, j, c] for c in range(dh)) / math.sqrt(dh))
                z = sum(w.values())
                for j, x in w.items():
                    got[b, h // 2, j] += x / z
                np.testing.assert_allclose(r["O"][i, h], sum(x / z * V[b, h // 2, j] for j, x in w.items()), rtol=1e-12)
                assert abs(r["lse"][h, i] - math.log(z)) < 1e-12
    np.testing.assert_allclose(r["got"], got, rtol=1e-12, atol=1e-15)


def test_a_chain_over_an_empty_cache_is_causal_attention():
    # every row of the causal attention sums to 1, and the account is N S (Hq / Hkv) of the importance
    N, Hq, Hkv, dh = 7, 4, 2, 8
    Q, K, V, lens, cu = _cache(6, 1, [N], [0], Hq, Hkv, dh, N)
    r = OP.tree_attention(Q, K, V, lens, cu)
    S = oracle.attn_importance(Q[None], K.transpose(0, 2, 1, 3), np.array([0, N]))
    np.testing.assert_allclose(r["got"].sum(axis=(0, 1)), N * Hq * S, rtol=1e-12)
    lse = oracle.attn_row_lse(Q[None], K.transpose(0, 2, 1, 3), np.array([0, N]))
    np.testing.assert_allclose(r["lse"], lse.reshape(Hq, N), rtol=1e-12)


def test_a_row_that_sees_nothing_is_empty():
    Q, K, V, lens, cu = _cache(7, 1, [2], [0], 2, 1, 8, 2)
    r = OP.tree_attention(Q, K, V, lens, cu, [0, 0b10])
    assert not r["O"][0].any() and np.isneginf(r["lse"][:, 0]).all()
    np.testing.assert_allclose(r["O"][1], V[0, 0, 1][None].repeat(2, 0))
    np.testing.assert_allclose(r["got"][0, 0], [0.0, 2.0])


def test_row_weights_choose_rows():
    Q, K, V, lens, cu = _cache(8, 1, [3], [5], 2, 2, 8, 8)
    each = [OP.tree_attention(Q, K, V, lens, cu, row_weight=w)["got"] for w in np.eye(3)]
    np.testing.assert_allclose(sum(each), OP.tree_attention(Q, K, V, lens, cu)["got"], rtol=1e-13)
    assert not each[0][0, 0, 6:].any()  # the first row of a chain sees the later drafted tokens not at all


def test_eviction_by_hand():
    acc = np.array([[[5.0, 0.0, 3.0, np.nan, 3.0, 9.0, 1.0, -np.inf]]])
    pos = np.arange(8)[None, None]
    idx, lens = OP.cache_evict(acc, pos, [8], [8], 4)
    assert idx.tolist() == [[[0, 4, 2, 5]]] and lens.tolist() == [4]  # 9, 5, 3, 3: holes 1 and 3 take 4 and 5
    idx, _ = OP.cache_evict(acc, pos, [8], [8], 3)
    assert idx.tolist() == [[[0, 5, 2]]]                              # of the equals, the lower slot
    idx, _ = OP.cache_evict(acc, pos, [8], [8], 4, recent=2, sink=1)
    assert idx.tolist() == [[[0, 5, 6, 7]]]                           # 0, 6 and 7 are guarded, then 9
    idx, lens = OP.cache_evict(acc, pos, [3], [3], 4)
    assert idx.tolist() == [[[0, 1, 2, -1]]] and lens.tolist() == [3]
    idx, _ = OP.cache_evict(acc, pos, [8], [8], 7)
    assert 3 not in idx[0, 0]                                         # NaN goes before -inf
    np.testing.assert_array_equal(OP.evicted(pos, np.array([[[0, 5, 2]]]), [8], -1), [[[0, 5, 2, -1, -1, -1, -1, -1]]])

"""Workspaces of the loss, tree-attention and eviction calls: one that is sized for a program's largest call serves its
smaller ones."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2608_15592_amd as estp

FAKE = ctypes.c_void_p(1 << 20)
OTHER = ctypes.c_void_p(1 << 21)
WS = ctypes.c_void_p(1 << 24)


def _never_less(size, values):
    """size(x) over ascending x."""
    sizes = np.array([size(x) for x in values])
    assert (sizes > 0).all()
    falls = np.flatnonzero(np.diff(sizes) < 0)
    assert len(falls) == 0, [(values[i], sizes[i], values[i + 1], sizes[i + 1]) for i in falls[:3]]


@pytest.mark.parametrize("cap", [4096, 16384, 16400, 20000, 65536, 131072, 1 << 20])
def test_eviction_workspaces_grow_with_the_call(cap):
    size = estp.load().estp_cache_evict_workspace_size
    for keep in (1, 2048, cap):
        _never_less(lambda b: size(b, 1, cap, min(keep, cap)), range(1, 700))
        _never_less(lambda h: size(3, h, cap, min(keep, cap)), range(1, 200))
    for groups in (1, 16, 30, 31, 170, 171, 256, 300):
        _never_less(lambda k: size(groups, 1, cap, k), sorted({*range(1, cap + 1, cap // 300 + 1), 4095, 4096} & {*range(cap + 1)}))


def test_eviction_workspaces_grow_with_the_capacity():
    size = estp.load().estp_cache_evict_workspace_size
    for groups in (1, 16, 170, 300):
        _never_less(lambda c: size(groups, 1, c, 1024), [*range(1024, 20000, 61), *range(20000, 200000, 997)])


TOKENS = [*range(1, 2200), 2500, 4095, 4096, 4097, 8191, 8192, 8193, 16384, 16385, 65536, 100000, 1 << 20, 1 << 22]
HEADS = [(2048, 128256), (4096, 128256), (1536, 151936), (1024, 16384), (96, 5000), (64, 1000), (32, 24449), (32, 1)]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("d,V", HEADS)
def test_loss_workspaces_grow_with_the_tokens(d, V, dtype):
    _never_less(lambda n: estp.load().estp_token_loss_workspace_size(n, d, V, dtype), TOKENS)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("d,V", HEADS)
def test_gradient_workspaces_grow_with_the_tokens(d, V, dtype):
    _never_less(lambda n: estp.load().estp_token_loss_backward_workspace_size(n, d, V, dtype), TOKENS)


@pytest.mark.parametrize("B,max_q,Hq,Hkv,max_kv,dh", [(32, 1, 32, 8, 32768, 128), (8, 1, 32, 8, 131072, 128),
                                                      (8, 4, 32, 8, 131072, 128), (1, 16, 8, 8, 100_003, 128)])
def test_kept_scores_take_the_room_of_the_rows_there_are(B, max_q, Hq, Hkv, max_kv, dh):
    # fp32 scores of every row; besides them 25 MB at most: the partial results of 1024 + B Hkv segments of 16 rows
    size = estp.load().estp_tree_attention_workspace_size(B, max_q, B * max_q, Hq, Hkv, max_kv, dh, 0)
    scores = 4 * B * max_q * Hq * (-(-max_kv // 32) * 32)
    assert scores < size < scores + 25e6


@pytest.mark.skipif(torch.cuda.is_available(), reason="fake pointers")
@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("dh", [32, 64, 128])
@pytest.mark.parametrize("G", [1, 4, 6])
@pytest.mark.parametrize("acc", [FAKE, None])
def test_a_tree_workspace_serves_every_smaller_call(dh, G, dtype, acc):
    lib = estp.load()

    def size(B, max_q, max_kv):
        return lib.estp_tree_attention_workspace_size(B, max_q, B * max_q, 8 * G, 8, max_kv, dh, dtype)

    def taken(wsb, B, max_q, max_kv):  # whatever follows the checks fails without a GPU
        status = lib.estp_tree_attention(FAKE, FAKE, OTHER, FAKE, FAKE, None, B, max_q, B * max_q, 8 * G, 8, 1 << 18,
                                         max_kv, dh, 0.125, dtype, FAKE, FAKE, acc, WS, wsb, None)
        assert status in (3, 4)
        return status != 3

    largest = [(B, q, kv) for B in (1, 8, 40) for q in (1, 2, 3, 5, 9, 16, 17, 40, 64) for kv in (70, 5000, 131072)]
    for call in largest:
        for larger in largest:
            if all(a <= b for a, b in zip(call, larger)):
                assert taken(size(*larger), *call), (call, larger)


@pytest.mark.skipif(torch.cuda.is_available(), reason="fake pointers")
def test_scores_are_asked_for_where_they_are_kept():
    # without the account, or of a call that keeps no scores, the least a call takes is the partial results
    lib = estp.load()
    full = lib.estp_tree_attention_workspace_size(8, 1, 8, 32, 8, 131072, 128, 0)
    wide = lib.estp_tree_attention_workspace_size(8, 16, 128, 32, 8, 131072, 128, 0)
    assert wide < full // 4
    for acc in (FAKE, None):
        for wsb, ok in ((full, True), (wide, True), (full - 1, True), (4096, False)):
            status = lib.estp_tree_attention(FAKE, FAKE, OTHER, FAKE, FAKE, None, 8, 1, 8, 32, 8, 131072, 131072, 128,
                                             0.125, 0, FAKE, FAKE, acc, WS, wsb, None)
            assert status == (4 if ok else 3)

"""Refusals of the loss, tree-attention and eviction calls: on the host, before any device work."""
import ctypes

import pytest
import torch

import paper_2608_15592_amd as estp

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="host-validation cases use fake pointers")

FAKE = ctypes.c_void_p(1 << 20)
OTHER = ctypes.c_void_p(1 << 21)
ODD = ctypes.c_void_p((1 << 20) + 2)
HALF = ctypes.c_void_p((1 << 20) + 4)  # 4-byte aligned only
WS = ctypes.c_void_p(1 << 24)


def _caller(fn, names, base):
    def call(**kw):
        a = dict(zip(names, base))
        assert set(kw) <= set(names)
        a.update(kw)
        status = fn(*[a[n] for n in names])
        assert status == 0 or estp.load().estp_last_error()
        return status
    return call


def test_token_loss_validation():
    lib = estp.load()
    ws = lib.estp_token_loss_workspace_size(100, 64, 1000, 0)
    assert ws == lib.estp_token_entropy_workspace_size(100, 64, 1000, 0) > 0
    call = _caller(lib.estp_token_loss, "X W t n d V dtype loss lse H arg ws wsb stream".split(),
                   (FAKE, FAKE, FAKE, 100, 64, 1000, 0, FAKE, FAKE, None, None, WS, ws, None))
    for name in ("X", "W", "t", "loss", "lse", "ws"):
        assert call(**{name: None}) == 1, name
    for name in ("X", "W", "t", "loss", "lse", "H", "arg", "ws"):
        assert call(**{name: ODD}) == 1, name
    assert call(n=0) == call(V=0) == call(d=60) == call(dtype=2) == 1
    assert call(d=40) == 2
    assert call(d=40, dtype=1, wsb=0) == 3
    assert call(wsb=ws - 1) == 3
    assert lib.estp_token_loss_workspace_size(0, 64, 1000, 0) == 0
    assert call(V=(1 << 31) - 65536, wsb=1 << 62) == 2
    # more tokens than one launch holds: refused before any kernel, with room enough
    for dtype in (0, 1):
        assert call(n=(1 << 26) + 1, V=3, dtype=dtype, wsb=1 << 62) == 2


def test_token_loss_backward_validation():
    lib = estp.load()
    ws = lib.estp_token_loss_backward_workspace_size(100, 64, 1000, 0)
    assert ws > 0
    call = _caller(lib.estp_token_loss_backward, "X W t lse grad n d V dtype dX dW ws wsb stream".split(),
                   (FAKE, FAKE, FAKE, FAKE, None, 100, 64, 1000, 0, FAKE, FAKE, WS, ws, None))
    for name in ("X", "W", "t", "lse", "ws"):
        assert call(**{name: None}) == 1, name
    for name in ("X", "W", "t", "lse", "grad", "dX", "dW", "ws"):
        assert call(**{name: ODD}) == 1, name
    assert call(dX=HALF) == call(dW=HALF) == 1
    assert call(dX=None, dW=None) == 1
    assert call(n=0) == call(V=0) == call(d=60) == call(dtype=2) == 1
    assert call(d=40) == call(n=(1 << 22) + 1) == 2
    assert call(d=1 << 15, n=(1 << 21) + 1, dtype=1, wsb=1 << 62) == 2
    assert call(V=(1 << 31) - 65536, wsb=1 << 62) == 2
    assert call(wsb=ws - 1) == 3
    for bad in ((0, 64, 1000), (100, 0, 1000), (100, 64, 0)):
        assert lib.estp_token_loss_backward_workspace_size(*bad, 0) == 0


TREE = "Q K V lens cu mask B max_q n_q Hq Hkv cap max_kv dh scale dtype O lse acc ws wsb stream".split()
CREDIT = "Q K lse lens cu mask w B max_q n_q Hq Hkv cap max_kv dh scale dtype acc stream".split()


def _tree_refusals(call):
    for name in ("Q", "K", "lens", "cu"):
        assert call(**{name: None}) == 1, name
    for name in ("Q", "K", "lens", "cu", "mask", "acc", "lse"):
        assert call(**{name: ODD}) == 1, name
    assert call(mask=HALF) == call(Q=HALF) == call(K=HALF) == 1
    assert call(B=0) == call(n_q=0) == call(Hq=0) == call(Hkv=0) == call(max_q=0) == 1
    assert call(Hq=5) == 1
    assert call(max_q=13) == 1           # more than n_q
    assert call(max_q=5) == 1            # two sequences of at most 5 rows hold no 12
    assert call(max_kv=0) == call(max_kv=101) == call(cap=0) == call(cap=(1 << 31)) == 1
    assert call(scale=0.0) == call(scale=float("nan")) == call(scale=float("inf")) == call(scale=-1.0) == 1
    assert call(dtype=2) == 1
    assert call(dh=96) == 2
    assert call(n_q=130, max_q=65) == 2  # more drafted tokens than mask bits
    assert call(Hq=2 * 65536) == 2


def test_tree_attention_validation():
    lib = estp.load()
    ws = lib.estp_tree_attention_workspace_size(2, 7, 12, 4, 2, 90, 64, 0)
    assert ws > 0
    call = _caller(lib.estp_tree_attention, TREE, (FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 2, 7, 12, 4, 2, 100, 90, 64,
                                                   0.125, 0, FAKE, FAKE, FAKE, WS, ws, None))
    _tree_refusals(call)
    assert call(V=None) == call(O=None) == call(ws=None) == 1
    assert call(V=HALF) == call(O=HALF) == call(ws=HALF) == 1
    assert call(wsb=ws - 1) == 3
    for bad in ((0, 7, 12, 4, 2, 90, 64), (2, 0, 12, 4, 2, 90, 64), (2, 7, 0, 4, 2, 90, 64), (2, 7, 12, 5, 2, 90, 64),
                (2, 7, 12, 4, 0, 90, 64), (2, 7, 12, 4, 2, 0, 64)):
        assert lib.estp_tree_attention_workspace_size(*bad, 0) == 0


def test_tree_importance_validation():
    lib = estp.load()
    call = _caller(lib.estp_tree_importance, CREDIT, (FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 2, 7, 12, 4, 2, 100,
                                                      90, 64, 0.125, 0, FAKE, None))
    _tree_refusals(call)
    assert call(lse=None) == call(acc=None) == call(w=ODD) == 1


def test_cache_evict_validation():
    lib = estp.load()
    ws = lib.estp_cache_evict_workspace_size(2, 4, 100, 50)
    assert ws > 0 and lib.estp_cache_evict_workspace_size(0, 4, 100, 50) == 0
    assert lib.estp_cache_evict_workspace_size(2, 4, 49, 50) == lib.estp_cache_evict_workspace_size(2, 4, 1 << 31, 50) == 0
    assert lib.estp_cache_evict_workspace_size(2, 4, 1 << 20, 50) > ws
    names = "K V acc pos lens seen B Hkv cap dh dtype keep recent sink acc_out pos_out lens_out idx ws wsb stream".split()
    call = _caller(lib.estp_cache_evict, names, (FAKE, OTHER, FAKE, FAKE, FAKE, FAKE, 2, 4, 100, 64, 0, 50, 8, 4, FAKE,
                                                 FAKE, FAKE, FAKE, WS, ws, None))
    for name in ("K", "V", "acc", "pos", "lens", "seen", "acc_out", "pos_out", "lens_out", "idx", "ws"):
        assert call(**{name: None}) == 1, name
        assert call(**{name: ODD}) == 1, name
    assert call(K=HALF) == call(V=HALF) == call(ws=HALF) == 1
    assert call(V=FAKE) == 1  # one memory for both
    assert call(B=0) == call(Hkv=0) == call(cap=0) == call(cap=1 << 31) == call(dtype=2) == 1
    assert call(keep=0) == call(keep=101) == call(recent=-1) == call(sink=-1) == call(recent=47) == 1
    assert call(dh=96) == call(B=20000) == 2
    assert call(wsb=ws - 1) == 3


def test_binding_refuses_host_tensors():
    X, W, t = torch.zeros(3, 32), torch.zeros(5, 32), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="X must be a device tensor"):
        estp.token_loss(X, W, t)
    with pytest.raises(ValueError, match="X must be a device tensor"):
        estp.token_loss_backward(X, W, t, torch.zeros(3))
    C = torch.zeros(1, 2, 8, 32)
    for call in (lambda: estp.tree_attention(torch.zeros(1, 2, 32), C, C, t[:1], t[:2], 1, 8),
                 lambda: estp.tree_importance(torch.zeros(1, 2, 32), C, torch.zeros(2, 1), t[:1], t[:2], 1, 8, C[..., 0])):
        with pytest.raises(ValueError, match="Q must be a device tensor"):
            call()
    with pytest.raises(ValueError, match="K must be a device tensor"):
        estp.cache_evict(C, C, C[..., 0], t, t, t, 4)

"""The fp64 oracle of the log-probability calls pinned against hand-computed values, differences and its own symmetries;
their refusals on the host; their workspaces."""
import os
import subprocess

import numpy as np
import pytest
import torch

import paper_2608_15592_amd as estp
from oracle import head as HD
from oracle import operators as OP
from paper_2608_15592_amd import build
from tests.test_operators_abi import FAKE, HALF, ODD, WS, _caller
from tests.test_operators_workspace import HEADS, TOKENS, _never_less


def test_logprobs_of_a_known_distribution():
    W = np.log(np.array([[0.5], [0.25], [0.125], [0.125]]))
    r = HD.token_logprobs(np.ones((1, 1)), W, [1], 4)
    np.testing.assert_allclose(r["logprob"], [np.log(0.25)], rtol=1e-14)
    np.testing.assert_allclose(r["H"], [1.75 * np.log(2)], rtol=1e-14)
    assert r["top_id"].tolist() == [[0, 1, 2, 3]]  # equal ones by index
    hot = HD.token_logprobs(np.ones((1, 1)), W, [1], 1, temperature=0.5)  # squares: 16, 4, 1, 1 of 22
    np.testing.assert_allclose(hot["logprob"], [np.log(4 / 22)], rtol=1e-14)


def test_distillation_of_a_known_distribution():
    W = np.log(np.array([[0.5], [0.25], [0.125], [0.125]]))
    x = np.ones((1, 1))
    own = HD.distill(x, W, [[2, 0, 1, 3]], np.log([[0.125, 0.5, 0.25, 0.125]]), grad=[1.0])
    np.testing.assert_allclose(own["loss"], 0, atol=1e-15)
    np.testing.assert_allclose(own["dW"], 0, atol=1e-15)
    one = HD.distill(x, W, [[1, -1, 4]], [[-3.0, 0.0, 0.0]])  # one held entry, renormalised: -log q
    np.testing.assert_allclose(one["loss"], [np.log(4)], rtol=1e-14)
    part = HD.distill(x, W, [[1]], [[np.log(0.5)]], renormalise=False)
    np.testing.assert_allclose(part["loss"], [0.5 * np.log(2)], rtol=1e-14)
    none = HD.distill(x, W, [[-1, 2]], [[0.0, -np.inf]], grad=[1.0])
    assert none["loss"][0] == 0 and not none["dX"].any() and not none["dW"].any()


@pytest.mark.parametrize("renormalise", [True, False])
def test_gradients_against_differences(renormalise):
    g = np.random.default_rng(2)
    X, W, w = g.standard_normal((3, 4)), g.standard_normal((9, 4)), g.standard_normal(3)
    ids = np.array([[1, 1, 5], [-1, 9, 0], [8, 2, 2]])
    logp = np.log(g.dirichlet(np.ones(3), 3) * 0.9)
    f = lambda: (w * HD.distill(X, W, ids, logp, 1.7, renormalise)["loss"]).sum()  # noqa: E731
    r = HD.distill(X, W, ids, logp, 1.7, renormalise, w)
    for A, dA in ((X, r["dX"]), (W, r["dW"])):
        for at in np.ndindex(A.shape):
            a, h = A[at], 1e-5
            A[at] = a + h
            up = f()
            A[at] = a - h
            down = f()
            A[at] = a
            assert abs((up - down) / (2 * h) - dA[at]) < 1e-8


def test_one_entry_is_the_loss_of_its_token():
    g = np.random.default_rng(3)
    X, W, w = g.standard_normal((5, 6)), g.standard_normal((11, 6)), g.standard_normal(5)
    t = np.array([3, -1, 10, 11, 0])
    r = HD.distill(X, W, t[:, None], np.zeros((5, 1)), grad=w)
    loss, lse = OP.token_loss(X, W, t)
    np.testing.assert_allclose(r["loss"], loss, rtol=1e-13)
    dX, dW = OP.token_loss_grads(X, W, t, w, "f32")[:2]
    np.testing.assert_allclose(r["dX"], dX, rtol=1e-12, atol=1e-15)
    np.testing.assert_allclose(r["dW"], dW, rtol=1e-12, atol=1e-15)


fakes = pytest.mark.skipif(torch.cuda.is_available(), reason="host-validation cases use fake pointers")


def _head_refusals(call, ws):
    for name in ("X", "W", "ws"):
        assert call(**{name: None}) == call(**{name: ODD}) == 1, name
    assert call(n=0) == call(V=0) == call(d=60) == call(dtype=2) == 1
    assert call(d=40) == 2
    for temperature in (0.0, -1.0, 1e-4, 1001.0, float("nan"), float("inf")):
        assert call(T=temperature) == 1
    assert call(wsb=ws - 1) == 3


@fakes
def test_token_logprobs_validation():
    lib = estp.load()
    ws = lib.estp_token_logprobs_workspace_size(100, 64, 1000, 20, 0)
    assert ws > 0
    call = _caller(lib.estp_token_logprobs, "X W t n d V k T dtype lp lse H id top ws wsb stream".split(),
                   (FAKE, FAKE, FAKE, 100, 64, 1000, 20, 1.0, 0, FAKE, FAKE, FAKE, FAKE, FAKE, WS, ws, None))
    _head_refusals(call, ws)
    for name in ("t", "lp", "lse", "H", "id", "top"):
        assert call(**{name: ODD}) == 1, name
    for name in ("t", "lp", "id", "top"):
        assert call(**{name: None}) == 1, name
    assert call(k=-1) == call(k=129) == call(V=19) == 1
    assert call(k=0, t=None, lp=None, lse=None, H=None) == 1
    assert call(V=(1 << 24) + 1, wsb=1 << 62) == 2
    for bad in ((0, 64, 1000, 20), (100, 0, 1000, 20), (100, 64, 0, 20), (100, 64, 1000, -1), (100, 64, 1000, 129)):
        assert lib.estp_token_logprobs_workspace_size(*bad, 0) == 0


@fakes
def test_distill_validation():
    lib = estp.load()
    ws = lib.estp_distill_loss_workspace_size(100, 64, 1000, 0)
    assert ws > 0
    call = _caller(lib.estp_distill_loss, "X W ids logp n d V K T norm dtype loss lse logq ws wsb stream".split(),
                   (FAKE, FAKE, FAKE, FAKE, 100, 64, 1000, 20, 1.0, 1, 0, FAKE, FAKE, FAKE, WS, ws, None))
    _head_refusals(call, ws)
    for name in ("ids", "logp", "loss", "lse", "logq"):
        assert call(**{name: None}) == call(**{name: ODD}) == 1, name
    assert call(K=0) == call(K=129) == 1
    assert call(n=(1 << 22) + 1) == call(V=(1 << 31) - 65536, wsb=1 << 62) == 2


@fakes
def test_distill_backward_validation():
    lib = estp.load()
    ws = lib.estp_distill_loss_backward_workspace_size(100, 64, 1000, 0)
    assert ws > 0
    call = _caller(lib.estp_distill_loss_backward,
                   "X W ids logp lse logq grad n d V K T norm dtype dX dW ws wsb stream".split(),
                   (FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None, 100, 64, 1000, 20, 1.0, 1, 0, FAKE, FAKE, WS, ws, None))
    _head_refusals(call, ws)
    for name in ("ids", "logp", "lse", "logq"):
        assert call(**{name: None}) == call(**{name: ODD}) == 1, name
    assert call(grad=ODD) == call(dX=HALF) == call(dW=HALF) == call(dX=None, dW=None) == 1
    assert call(K=0) == call(K=129) == 1
    assert call(n=(1 << 22) + 1) == call(d=1 << 15, n=(1 << 21) + 1, dtype=1, wsb=1 << 62) == 2


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("d,V", HEADS)
def test_workspaces_grow_with_the_tokens(d, V, dtype):
    lib = estp.load()
    _never_less(lambda n: lib.estp_distill_loss_workspace_size(n, d, V, dtype), TOKENS)
    _never_less(lambda n: lib.estp_distill_loss_backward_workspace_size(n, d, V, dtype), TOKENS)
    for k in (0, 1, 128):
        _never_less(lambda n: lib.estp_token_logprobs_workspace_size(n, d, V, k, dtype), TOKENS)
    for n in (1, 100, 5000):
        _never_less(lambda k: lib.estp_token_logprobs_workspace_size(n, d, V, k, dtype), range(129))


def test_plans_of_log_probability_calls(tmp_path):
    exe = str(tmp_path / "logprob_plan")
    here = os.path.dirname(os.path.abspath(__file__))
    cmd = [build.hipcc(), f"--offload-arch={build.ARCH}", "-O1", "-std=c++17", f"-I{build.INCLUDE}", f"-I{build.CSRC}",
           os.path.join(here, "host", "logprob_plan.hip"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stdout + r.stderr


def test_launches_of_a_teachers_entries(tmp_path):
    exe = str(tmp_path / "pick_threads")
    here = os.path.dirname(os.path.abspath(__file__))
    cmd = [build.hipcc(), f"--offload-arch={build.ARCH}", "-O1", "-std=c++17", f"-I{build.INCLUDE}", f"-I{build.CSRC}",
           os.path.join(here, "host", "pick_threads.hip"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-3000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stdout + r.stderr

"""LM-head loss and its gradients on the GPU against the fp64 oracle, element by element, at the bounds the
oracle derives (oracle/operators.py)."""
import numpy as np
import pytest
import torch

import paper_2608_15592_amd as estp
from oracle import operators as OP
from synth import inputs as I
from tests._util import dev, host

pytestmark = pytest.mark.gpu


def _bits(a, dtype):
    a = np.ascontiguousarray(a, dtype=np.float32)
    return I.f32_to_bf16_bits(a) if dtype == "bf16" else a


def _wide(t):
    return host(t.float()).astype(np.float64)


def _inputs(seed, n, d, V, dtype, ignored=0.0, lean=6.0):
    g = np.random.default_rng(seed)
    W = _bits(g.standard_normal((V, d)) * 0.05, dtype)
    t = g.integers(0, V, n).astype(np.int32)
    X = g.standard_normal((n, d))
    X += lean * g.uniform(size=(n, 1)) * OP.widen(W)[t] / (0.0025 * d)
    t[g.uniform(size=n) < ignored] = g.choice([-100, -1, V, 2**31 - 1])
    return _bits(X, dtype), W, t, (g.standard_normal(n) / n).astype(np.float32)


SHAPES = [(1, 32, 1), (1, 64, 7), (3, 32, 257), (64, 96, 1000), (65, 64, 256), (127, 160, 4099), (257, 128, 513),
          (300, 224, 5000), (1030, 64, 3001)]


def _check_forward(X, W, t, dtype):
    loss, lse = estp.token_loss(dev(X), dev(W), dev(t))
    ref_loss, ref_lse = OP.token_loss(X, W, t)
    b = OP.lse_bound(X, W, ref_lse)
    assert (np.abs(_wide(lse) - ref_lse) <= b).all()
    # the target's logit, and one rounding of the difference
    b = b + OP.logit_bound(X, W) + 2 * OP.U * (np.abs(ref_lse) + np.abs(ref_loss))
    assert (np.abs(_wide(loss) - ref_loss) <= b).all()
    assert (host(loss) >= 0).all() and (host(loss)[(t < 0) | (t >= len(W))] == 0).all()
    return lse


def _check_backward(X, W, t, g, dtype, lse, **kw):
    dX, dW = estp.token_loss_backward(dev(X), dev(W), dev(t), lse, None if g is None else dev(g), **kw)
    ref = OP.token_loss_grads(X, W, t, np.ones(len(X)) if g is None else g, dtype)
    for got, want, bound, name in ((dX, ref[0], ref[2], "dX"), (dW, ref[1], ref[3], "dW")):
        if got is not None:
            over = np.abs(_wide(got) - want) - bound
            assert (over <= 0).all(), f"{name}: {over.max()} over the bound at {np.unravel_index(over.argmax(), over.shape)}"
    return dX, dW


@pytest.mark.parametrize("n,d,V", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_loss_and_gradients(n, d, V, dtype):
    X, W, t, g = _inputs(n + V, n, d, V, dtype, ignored=0.2 if n > 3 else 0.0)
    lse = _check_forward(X, W, t, dtype)
    _check_backward(X, W, t, g, dtype, lse)


@pytest.mark.parametrize("n,d,V", [(5, 8, 3), (70, 40, 300), (130, 72, 1003)])
def test_f32_widths(n, d, V):
    X, W, t, g = _inputs(n, n, d, V, "f32")
    _check_backward(X, W, t, g, "f32", _check_forward(X, W, t, "f32"))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_several_vocabulary_pieces(dtype):
    # enough tokens that the vocabulary is cut into pieces, the last of them short
    n = 17000 if dtype == "bf16" else 9000
    X, W, t, g = _inputs(5, n, 32, 17001, dtype)
    _check_backward(X, W, t, g, dtype, _check_forward(X, W, t, dtype))


@pytest.mark.parametrize("n", [5, 128, 129])
def test_weights_larger_than_the_last_cache(n):
    # 270 MB of W and dW
    X, W, t, g = _inputs(n, n, 4096, 33001, "bf16", ignored=0.1)
    _check_backward(X, W, t, g, "bf16", _check_forward(X, W, t, "bf16"))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_default_weights_and_single_outputs(dtype):
    X, W, t, g = _inputs(6, 90, 64, 700, dtype, ignored=0.3)
    lse = estp.token_loss(dev(X), dev(W), dev(t))[1]
    dX, dW = _check_backward(X, W, t, None, dtype, lse)
    only_x = _check_backward(X, W, t, None, dtype, lse, want_dW=False)
    only_w = _check_backward(X, W, t, None, dtype, lse, want_dX=False)
    assert only_x[1] is None and only_w[0] is None
    assert torch.equal(only_x[0], dX) and torch.equal(only_w[1], dW)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_all_tokens_ignored(dtype):
    X, W, t, g = _inputs(7, 70, 64, 300, dtype)
    t[:] = -100
    loss, lse = estp.token_loss(dev(X), dev(W), dev(t))
    dX, dW = (torch.full_like(dev(a), float("nan")) for a in (X, W))
    estp.token_loss_backward(dev(X), dev(W), dev(t), lse, dev(g), dX=dX, dW=dW)
    assert not loss.any() and not dX.any() and not dW.any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ignored_rows_may_hold_anything(dtype):
    X, W, t, g = _inputs(8, 200, 64, 900, dtype, ignored=0.4)
    lse = _check_forward(X, W, t, dtype)
    clean = estp.token_loss_backward(dev(X), dev(W), dev(t), lse, dev(g))
    Xd, gd, off = dev(X), dev(g), dev((t < 0) | (t >= 900))
    Xd[off] = float("nan")
    Xd[off.nonzero()[0, 0]] = float("inf")
    gd[off] = float("nan")
    loss, lse = estp.token_loss(Xd, dev(W), dev(t))
    assert torch.equal(loss[off], torch.zeros_like(loss[off]))
    for got, want in zip(estp.token_loss_backward(Xd, dev(W), dev(t), lse, gd), clean):
        assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_entropy_and_mode_are_those_of_token_entropy(dtype):
    X, W, t, _ = _inputs(9, 333, 128, 5000, dtype)
    H, am, H2, am2 = (torch.empty(333, dtype=k, device="cuda") for k in (torch.float32, torch.int32) * 2)
    estp.token_entropy(dev(X), dev(W), H=H, vocab_argmax=am)
    estp.token_loss(dev(X), dev(W), dev(t), H=H2, vocab_argmax=am2)
    assert torch.equal(H, H2) and torch.equal(am, am2)


def test_gradient_against_differences_of_the_loss():
    # the fp32 kernels' own losses: central differences of step h err by O(h^2) and by the losses' rounding / h
    X, W, t, g = _inputs(10, 20, 32, 50, "f32")
    Xd, Wd, td, gd = dev(X), dev(W), dev(t), dev(g)
    dX, dW = estp.token_loss_backward(Xd, Wd, td, estp.token_loss(Xd, Wd, td)[1], gd)
    total = lambda: float((estp.token_loss(Xd, Wd, td)[0].double() * gd.double()).sum())  # noqa: E731
    h = 2.0 ** -6
    noise = float(gd.double().abs().sum()) * (2 * float(OP.lse_bound(X, W, OP.token_loss(X, W, t)[1]).max())) / h
    for A, dA in ((Xd, dX), (Wd, dW)):
        for at in np.random.default_rng(3).integers(0, A.numel(), 12).tolist():
            a = A.view(-1)[at].item()
            A.view(-1)[at] = a + h
            up = total()
            A.view(-1)[at] = a - h
            down = total()
            A.view(-1)[at] = a
            # third derivatives of a log-sum-exp in one coordinate are at most the cube of its other factor
            third = float((gd.abs().double()).sum()) * max(np.abs(X).max(), np.abs(W).max()) ** 3
            assert abs((up - down) / (2 * h) - dA.view(-1)[at].item()) <= noise + third * h * h / 6 + 1e-6


def test_non_finite_logits_stay_in_their_row():
    X, W, t, g = _inputs(11, 64, 64, 300, "bf16")
    Xd = dev(X)
    Xd[5] = float("nan")
    lse = estp.token_loss(Xd, dev(W), dev(t))[1]
    dX, dW = estp.token_loss_backward(Xd, dev(W), dev(t), lse, dev(g))
    assert torch.isnan(lse[5]) and torch.isnan(dX[5]).all() and torch.isnan(dW).all()
    keep = torch.arange(64, device="cuda") != 5
    assert torch.isfinite(lse[keep]).all() and torch.isfinite(dX[keep]).all()


def test_repeats_streams_and_smaller_calls_on_one_workspace():
    X, W, t, g = _inputs(12, 700, 128, 3000, "bf16", ignored=0.1)
    Xd, Wd, td, gd = dev(X), dev(W), dev(t), dev(g)
    ws = torch.empty(estp.load().estp_token_loss_backward_workspace_size(700, 128, 3000, 0), dtype=torch.uint8,
                     device="cuda")
    lse = estp.token_loss(Xd, Wd, td)[1]
    first = estp.token_loss_backward(Xd, Wd, td, lse, gd, workspace=ws)
    ws.fill_(255)  # NaN wherever a kernel reads what the call has not written
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = estp.token_loss_backward(Xd, Wd, td, lse, gd, workspace=ws, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(first, again):
        assert torch.equal(a, b)
    m = 65  # a call on fewer tokens
    X, t, g = X[:m], t[:m], g[:m]
    _check_backward(X, W, t, g, "bf16", lse[:m].contiguous())


def test_replayed_in_a_graph():
    X, W, t, g = _inputs(13, 300, 64, 2000, "bf16", ignored=0.2)
    Xd, Wd, td, gd = dev(X), dev(W), dev(t), dev(g)
    lib = estp.load()
    ws = [torch.empty(f(300, 64, 2000, 0), dtype=torch.uint8, device="cuda")
          for f in (lib.estp_token_loss_workspace_size, lib.estp_token_loss_backward_workspace_size)]
    loss, lse = (torch.empty(300, device="cuda") for _ in range(2))
    dX, dW = torch.empty_like(Xd), torch.empty_like(Wd)

    def step():
        estp.token_loss(Xd, Wd, td, loss=loss, lse=lse, workspace=ws[0])
        estp.token_loss_backward(Xd, Wd, td, lse, gd, dX=dX, dW=dW, workspace=ws[1])

    step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for rep in range(3):
        if rep == 1:  # other live tokens: the graph's own work follows the data
            td.copy_(dev(np.where(t < 0, 7, np.where(t % 3 == 0, -100, t)).astype(np.int32)))
        want = estp.token_loss(Xd, Wd, td)
        want += estp.token_loss_backward(Xd, Wd, td, want[1], gd)
        for a in (loss, lse, dX, dW):
            a.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip((loss, lse, dX, dW), want):
            assert torch.equal(a, b), rep


def test_weights_past_32_bit_offsets():
    # W and dW of 2.46e9 elements: byte offsets pass 2^32, element offsets 2^31.  Rows far apart are given, the
    # rest of W is 0, so the logits are 0 there and the distribution is known
    n, d, V = 4, 4096, 600_000
    g = np.random.default_rng(14)
    X = _bits(g.standard_normal((n, d)), "bf16")
    at = np.array([0, 255, 131_071, 300_001, 524_288, 599_999])
    rows = _bits(0.05 * g.standard_normal((len(at), d)), "bf16")
    W = torch.zeros(V, d, dtype=torch.bfloat16, device="cuda")
    W[dev(at)] = dev(rows)
    t = np.array([0, 300_001, 599_999, 524_288], dtype=np.int32)
    loss, lse = estp.token_loss(dev(X), W, dev(t))
    z = OP.widen(X) @ OP.widen(rows).T
    ref = np.log(np.exp(z).sum(axis=1) + V - len(at))
    zt = z[np.arange(n), [0, 3, 5, 4]]
    bound = OP.lse_bound(X, rows, ref) + 4 * OP.U * (V // 256) * (1 + np.abs(ref))
    assert (np.abs(_wide(lse) - ref) <= bound).all() and (np.abs(_wide(loss) - (ref - zt)) <= 2 * bound).all()
    dX, dW = estp.token_loss_backward(dev(X), W, dev(t), lse)
    P = np.exp(z - ref[:, None])
    G = P.copy()
    G[np.arange(n), [0, 3, 5, 4]] -= 1.0
    r = 2.0 ** -8 * 1.05
    assert (np.abs(_wide(dX) - G @ OP.widen(rows)) <= r * (np.abs(G @ OP.widen(rows)) + np.abs(G) @ np.abs(OP.widen(rows)))
            + 1e-6).all()
    want = G.T @ OP.widen(X)
    assert (np.abs(_wide(dW[dev(at)]) - want) <= r * (np.abs(want) + np.abs(G).T @ np.abs(OP.widen(X))) + 1e-9).all()
    other = np.array([1, 256, 262_144, 524_287, 599_998])  # p = exp(-lse), no target
    want = np.exp(-ref) @ OP.widen(X)
    bound = r * (np.abs(want) + np.exp(-ref) @ np.abs(OP.widen(X)))
    assert (np.abs(_wide(dW[dev(other)]) - want) <= bound).all()


def test_binding_refuses_mis_sized_tensors():
    X, W = torch.zeros(4, 64, device="cuda"), torch.zeros(9, 64, device="cuda")
    t, f = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(4, device="cuda")
    with pytest.raises(ValueError, match="targets must hold 4"):
        estp.token_loss(X, W, t[:3])
    with pytest.raises(TypeError, match="targets must be"):
        estp.token_loss(X, W, t.long())
    with pytest.raises(ValueError, match="disagree on d"):
        estp.token_loss(X, W[:, :32].contiguous(), t)
    with pytest.raises(TypeError, match="W must be"):
        estp.token_loss(X, W.bfloat16(), t)
    for name in ("loss", "lse", "H", "vocab_argmax"):
        with pytest.raises((ValueError, TypeError), match=name):
            estp.token_loss(X, W, t, **{name: f[:3]})
    with pytest.raises(ValueError, match="X must be contiguous"):
        estp.token_loss(torch.zeros(64, 4, device="cuda").t(), W, t)
    with pytest.raises(ValueError, match="lse must hold 4"):
        estp.token_loss_backward(X, W, t, f[:2])
    with pytest.raises(ValueError, match="grad must hold 4"):
        estp.token_loss_backward(X, W, t, f, f[:2])
    with pytest.raises(ValueError, match="dW must hold 576"):
        estp.token_loss_backward(X, W, t, f, dW=X)
    with pytest.raises(estp.EstpError, match="both null"):
        estp.token_loss_backward(X, W, t, f, want_dX=False, want_dW=False)
    with pytest.raises(estp.EstpError, match="workspace"):
        estp.token_loss_backward(X, W, t, f, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [3, 70, 2100])
def test_a_nan_weight_row_reaches_every_loss(dtype, n):
    X, W, t, g = _inputs(15, n, 64, 700, dtype)
    for row in (0, 300, 699):
        Wd = dev(W)
        Wd[row, 5] = float("nan")
        loss, lse = estp.token_loss(dev(X), Wd, dev(t))
        assert torch.isnan(loss).all() and torch.isnan(lse).all(), row


def test_few_live_tokens_among_very_many():
    # fp32, 600 001 tokens of which 90 are live: more shares of the vocabulary than workgroups for them
    n, d, V = 600_001, 256, 8192
    X, W, t, g = _inputs(15, 90, d, V, "f32")
    at = np.sort(np.random.default_rng(15).choice(n, 90, replace=False))
    Xd = torch.full((n, d), float("nan"), device="cuda")
    td = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    lse, gd = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    place = torch.from_numpy(at).cuda()
    Xd[place], td[place], gd[place] = dev(X), dev(t), dev(g)
    lse[place] = estp.token_loss(dev(X), dev(W), dev(t))[1]
    dX, dW = estp.token_loss_backward(Xd, dev(W), td, lse, gd)
    rX, rW, bX, bW = OP.token_loss_grads(X, W, t, g, "f32")
    assert (np.abs(_wide(dX[place]) - rX) <= bX).all() and (np.abs(_wide(dW) - rW) <= bW).all()
    dX[place] = 0
    assert not dX.any()

"""Distillation losses and gradients on the GPU against the fp64 oracle (oracle/head.py), element by element, at the
bounds it derives."""
import numpy as np
import pytest
import torch

import paper_2608_15592_amd as estp
from oracle import head as HD
from oracle import operators as OP
from tests._util import dev, host
from tests.test_gpu_operators_workspace import Guarded
from tests.test_gpu_token_loss import _inputs, _wide

pytestmark = pytest.mark.gpu


def _case(seed, n, d, V, K, dtype, ignored=0.2, repeats=False):
    """Inputs of a step: some rows without entries, some with fewer than K, ids out of range, weights of 0."""
    X, W, t, grad = _inputs(seed, n, d, V, dtype)
    g = np.random.default_rng(seed + 1)
    ids = (t[:, None] + np.arange(K) * g.integers(1, max(2, V // K), (n, 1))) % V
    if repeats:
        ids = g.integers(0, min(V, 5), (n, K))
    logp = np.sort(g.standard_normal((n, K)) * 2 - 4, axis=1)[:, ::-1].astype(np.float32)
    logp -= np.log(np.exp(logp.astype(np.float64)).sum(axis=1, keepdims=True) * g.uniform(1.0, 1.5, (n, 1))).astype(np.float32)
    ids = np.where(g.uniform(size=(n, K)) < 0.1, g.choice([-1, -100, V, 2**31 - 1], (n, K)), ids)
    logp[g.uniform(size=(n, K)) < 0.05] = -np.inf
    out = g.uniform(size=n) < ignored
    ids[out & (g.uniform(size=n) < 0.7)] = -1
    logp[out] = -np.inf
    return X, W, ids.astype(np.int32), logp, grad


def _check(case, dtype, temperature=1.0, renormalise=True, grads=True, **kw):
    X, W, ids, logp, grad = case
    Xd, Wd, idd, lpd, gd = map(dev, case)
    how = {"temperature": temperature, "renormalise": renormalise}
    out = dict(zip(("loss", "lse", "logq"), estp.distill_loss(Xd, Wd, idd, lpd, **how)))
    if grads:
        out["dX"], out["dW"] = estp.distill_loss_backward(Xd, Wd, idd, lpd, out["lse"], out["logq"], gd, **how, **kw)
    ref = HD.distill(X, W, ids, logp, temperature, renormalise, grad if grads else None, dtype)
    for name, a in out.items():
        if a is not None:
            over = np.abs(_wide(a) - ref[name]) - ref[name + "_bound"]
            assert (over <= 0).all(), f"{name}: {over.max()} over the bound at {np.unravel_index(over.argmax(), over.shape)}"
    return out


SHAPES = [(1, 32, 1, 1), (1, 64, 7, 3), (3, 32, 257, 128), (64, 96, 1000, 20), (65, 64, 256, 65), (127, 160, 4099, 5),
          (257, 128, 513, 33), (300, 224, 5000, 64), (1030, 64, 3001, 16)]


@pytest.mark.parametrize("n,d,V,K", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("renormalise", [True, False])
def test_loss_and_gradients(n, d, V, K, dtype, renormalise):
    _check(_case(n + V, n, d, V, K, dtype, ignored=0.2 if n > 3 else 0.0), dtype, 1.0, renormalise)


@pytest.mark.parametrize("temperature", [0.5, 3.0, 20.0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [30, 150])
def test_temperatures(temperature, dtype, n):
    _check(_case(n, n, 96, 2000, 12, dtype), dtype, temperature)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [20, 200])
@pytest.mark.parametrize("renormalise", [True, False])
def test_one_token_in_several_entries(dtype, n, renormalise):
    _check(_case(n, n, 64, 400, 40, dtype, repeats=True), dtype, 1.0, renormalise)


@pytest.mark.parametrize("n,d,V", [(5, 8, 30), (70, 40, 300), (130, 72, 1003)])
def test_f32_widths(n, d, V):
    _check(_case(n, n, d, V, 9, "f32"), "f32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_several_vocabulary_pieces(dtype):
    n = 17000 if dtype == "bf16" else 9000
    _check(_case(5, n, 32, 17001, 6, dtype, ignored=0.9), dtype, 2.0)


@pytest.mark.parametrize("n,d,V", [(1, 1024, 5000), (17, 1024, 77), (64, 1024, 4100), (33, 1536, 4097), (20, 2048, 16400),
                                   (50, 2048, 4099), (32, 2560, 4500), (40, 2560, 4500), (16, 3584, 4111),
                                   (1, 4096, 4600), (32, 4096, 4097), (33, 4096, 4097)])
def test_few_tokens(n, d, V):
    # whose part of the depth stays in registers, where they fit
    _check(_case(n + d, n, d, V, 10, "bf16"), "bf16", 1.2)


@pytest.mark.parametrize("n,d,V,K", [(1, 128, 98400, 2), (16, 264, 98500, 9), (30, 520, 50000, 9), (64, 264, 61000, 5),
                                     (65, 72, 50001, 7), (90, 256, 50000, 20), (96, 136, 49153, 4), (100, 72, 140001, 3), (90, 64, 270001, 5), (200, 512, 17003, 128),
                                     (500, 256, 8300, 9), (9000, 64, 8200, 4)])
def test_f32_from_parts(n, d, V, K):
    # products formed from parts in bf16
    _check(_case(n + d, n, d, V, K, "f32", ignored=0.2 if n < 1000 else 0.9), "f32", 1.3)


@pytest.mark.parametrize("n", [2049, 2500, 3400, 4400])
def test_many_tokens_forward(n):
    _check(_case(n, n, 64, 6000, 4, "bf16"), "bf16", 1.5, grads=False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_entry_of_full_weight_is_the_loss_of_that_token(dtype):
    X, W, t, g = _inputs(31, 150, 64, 900, dtype, ignored=0.2)
    Xd, Wd, td, gd = dev(X), dev(W), dev(t), dev(g)
    loss, lse = estp.token_loss(Xd, Wd, td)
    ids, logp = td[:, None].contiguous(), torch.zeros(150, 1, device="cuda")
    for renormalise in (True, False):
        got, lse2, logq = estp.distill_loss(Xd, Wd, ids, logp, renormalise=renormalise)
        b = OP.lse_bound(X, W, _wide(lse)) + OP.logit_bound(X, W)
        assert torch.equal(lse, lse2) and (np.abs(_wide(got) - _wide(loss)) <= 2 * b).all()
        dX, dW = estp.distill_loss_backward(Xd, Wd, ids, logp, lse2, logq, gd, renormalise=renormalise)
        ref = OP.token_loss_grads(X, W, t, g, dtype)
        assert (np.abs(_wide(dX) - ref[0]) <= 2 * ref[2]).all() and (np.abs(_wide(dW) - ref[1]) <= 2 * ref[3]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_default_weights_and_single_outputs(dtype):
    X, W, ids, logp, _ = _case(6, 90, 64, 700, 8, dtype, ignored=0.3)
    case = (X, W, ids, logp, np.ones(90, np.float32))
    out = _check(case, dtype)
    args = [dev(a) for a in case[:4]] + [out["lse"], out["logq"]]
    both = estp.distill_loss_backward(*args)
    only_x, only_w = estp.distill_loss_backward(*args, want_dW=False), estp.distill_loss_backward(*args, want_dX=False)
    assert only_x[1] is None and only_w[0] is None
    assert torch.equal(both[0], out["dX"]) and torch.equal(both[1], out["dW"])
    assert torch.equal(only_x[0], both[0]) and torch.equal(only_w[1], both[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("renormalise", [True, False])
def test_all_rows_ignored(dtype, renormalise):
    X, W, ids, logp, g = _case(7, 70, 64, 300, 5, dtype)
    ids[::2], logp[1::2] = -1, -np.inf
    how = {"renormalise": renormalise}
    args = [dev(a) for a in (X, W, ids, logp)]
    loss, lse, logq = estp.distill_loss(*args, **how)
    dX, dW = (torch.full_like(a, float("nan")) for a in args[:2])
    estp.distill_loss_backward(*args, lse, logq, dev(g), dX=dX, dW=dW, **how)
    assert not loss.any() and not dX.any() and not dW.any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [50, 1200])
def test_ignored_rows_and_entries_may_hold_anything(dtype, n):
    case = _case(8, n, 64, 900, 10, dtype, ignored=0.4)
    out = _check(case, dtype)
    X, W, ids, logp, g = map(dev, case)
    held = (ids >= 0) & (ids < 900)
    logp[~held] = float("nan")
    off = ~(held & (logp > -float("inf"))).any(dim=1)
    X[off], g[off] = float("nan"), float("nan")
    loss, lse, logq = estp.distill_loss(X, W, ids, logp)
    assert torch.equal(loss, out["loss"]) and not logq[~held].any()
    lse[off], logq[off] = float("nan"), float("nan")
    logq[~held] = float("nan")
    dX, dW = estp.distill_loss_backward(X, W, ids, logp, lse, logq, g)
    assert torch.equal(dX, out["dX"]) and torch.equal(dW, out["dW"])


def test_non_finite_values_stay_in_their_row():
    case = _case(11, 64, 64, 300, 6, "bf16", ignored=0.0)
    X, W, ids, logp, g = map(dev, case)
    ids[5, 0], logp[5, 0] = 7, float("nan")
    X[9] = float("inf")
    loss, lse, logq = estp.distill_loss(X, W, ids, logp)
    dX, _ = estp.distill_loss_backward(X, W, ids, logp, lse, logq, g)
    bad = torch.zeros(64, dtype=torch.bool, device="cuda")
    bad[5] = bad[9] = True
    assert torch.isnan(loss[bad]).all() and torch.isnan(dX[bad]).all()
    assert torch.isfinite(loss[~bad]).all() and torch.isfinite(dX[~bad]).all()


def test_f32_from_parts_with_infinite_numbers():
    # one live row of X holds an infinite number, two gradients are infinite: dW is infinite or NaN in what they reach, as
    # products of 64 bits are, and the rest is as it was without them
    n, d, V = 70, 64, 50000
    X, W, ids, logp, g = _case(21, n, d, V, 6, "f32")
    clean = _check((X, W, ids, logp, g), "f32")
    args = [dev(a) for a in (W, ids, logp)] + [clean["lse"], clean["logq"]]
    Xd, gd = dev(X), dev(g)
    live = (((ids >= 0) & (ids < V)) & (logp > -np.inf)).any(axis=1).nonzero()[0]
    gd[int(live[3])] = float("inf")
    got = estp.distill_loss_backward(Xd, *args, gd, want_dX=False)[1]
    # that row's factor (p sum_w - w) is nowhere 0 here, so that every number of dW has a product of infinity in it
    assert not torch.isfinite(got).any()
    x = Xd[int(live[3])]
    rows = torch.randperm(V, generator=torch.Generator().manual_seed(3))[:500].cuda()
    others = sorted(set(range(V)) - set(ids[int(live[3])].tolist()))
    rows = rows[torch.isin(rows, torch.tensor(others, device="cuda"))]
    assert torch.equal(got[rows], torch.sign(x).expand(len(rows), d) * float("inf"))


@pytest.mark.parametrize("renormalise", [True, False])
def test_gradient_against_differences_of_the_loss(renormalise):
    # central differences of the fp32 kernels' own losses: off by O(h^2) and by the losses' rounding / h
    X, W, ids, logp, g = _case(10, 20, 32, 50, 6, "f32")
    how = {"renormalise": renormalise, "temperature": 2.0}
    Xd, Wd, idd, lpd, gd = dev(X), dev(W), dev(ids), dev(logp), dev(g)
    lse, logq = estp.distill_loss(Xd, Wd, idd, lpd, **how)[1:]
    dX, dW = estp.distill_loss_backward(Xd, Wd, idd, lpd, lse, logq, gd, **how)
    total = lambda: float((estp.distill_loss(Xd, Wd, idd, lpd, **how)[0].double() * gd.double()).sum())  # noqa: E731
    h = 2.0 ** -6
    noise = float((np.abs(g) * HD.distill(X, W, ids, logp, 2.0, renormalise)["loss_bound"]).sum()) / h
    for A, dA in ((Xd, dX), (Wd, dW)):
        for at in np.random.default_rng(3).integers(0, A.numel(), 12).tolist():
            a = A.view(-1)[at].item()
            A.view(-1)[at] = a + h
            up = total()
            A.view(-1)[at] = a - h
            down = total()
            A.view(-1)[at] = a
            # third derivatives of a log-sum-exp in one coordinate are at most the cube of its other factor
            third = float(gd.abs().double().sum()) * (max(np.abs(X).max(), np.abs(W).max()) / 2) ** 3
            assert abs((up - down) / (2 * h) - dA.view(-1)[at].item()) <= noise + third * h * h / 6 + 1e-6


def test_repeats_streams_and_smaller_calls_on_one_workspace():
    case = _case(12, 700, 128, 3000, 24, "bf16")
    X, W, ids, logp, g = map(dev, case)
    lib = estp.load()
    ws = [Guarded(f(700, 128, 3000, 0)) for f in (lib.estp_distill_loss_workspace_size,
                                                  lib.estp_distill_loss_backward_workspace_size)]
    first = estp.distill_loss(X, W, ids, logp)
    first += estp.distill_loss_backward(X, W, ids, logp, *first[1:], g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = estp.distill_loss(X, W, ids, logp, workspace=ws[0].ws, stream=side)
    again += estp.distill_loss_backward(X, W, ids, logp, *again[1:], g, workspace=ws[1].ws, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(first, again):
        assert torch.equal(a, b)
    for m in (1, 64, 65, 385):
        few = [a[:m].contiguous() for a in (X, ids, logp, g)]
        want = estp.distill_loss(few[0], W, few[1], few[2])
        want += estp.distill_loss_backward(few[0], W, few[1], few[2], *want[1:], few[3])
        got = estp.distill_loss(few[0], W, few[1], few[2], workspace=ws[0].ws)
        got += estp.distill_loss_backward(few[0], W, few[1], few[2], *got[1:], few[3], workspace=ws[1].ws)
        assert all(torch.equal(a, b) for a, b in zip(want, got)), m
    for w in ws:
        w.check()


@pytest.mark.parametrize("n,larger", [(30, 31), (64, 65), (96, 97), (90, 129), (200, 1000), (1, 90)])
def test_f32_on_a_larger_calls_workspace(n, larger):
    d, V = 256, 98400
    X, W, ids, logp, g = map(dev, _case(n, n, d, V, 6, "f32"))
    lib = estp.load()
    ws = [Guarded(f(larger, d, V, 1)) for f in (lib.estp_distill_loss_workspace_size,
                                                lib.estp_distill_loss_backward_workspace_size)]
    want = estp.distill_loss(X, W, ids, logp)
    want += estp.distill_loss_backward(X, W, ids, logp, *want[1:], g)
    got = estp.distill_loss(X, W, ids, logp, workspace=ws[0].ws)
    got += estp.distill_loss_backward(X, W, ids, logp, *got[1:], g, workspace=ws[1].ws)
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    for w in ws:
        w.check()


def test_a_teachers_record_trains_a_student_in_a_graph():
    """As used together: the teacher's alternatives, the student's loss and gradients on them, captured and replayed."""
    n, V, K, T = 300, 2000, 16, 2.0
    Xt, Wt, t, g = _inputs(40, n, 96, V, "bf16")
    Xs, Ws, _, _ = _inputs(41, n, 64, V, "bf16")
    Xt, Wt, Xs, Ws, g = map(dev, (Xt, Wt, Xs, Ws, g))
    lib = estp.load()
    wss = [torch.empty(b, dtype=torch.uint8, device="cuda") for b in (
        lib.estp_token_logprobs_workspace_size(n, 96, V, K, 0), lib.estp_distill_loss_workspace_size(n, 64, V, 0),
        lib.estp_distill_loss_backward_workspace_size(n, 64, V, 0))]

    def step(out, ws=(None,) * 3):
        _, _, _, ids, logp = estp.token_logprobs(Xt, Wt, None, K, temperature=T, workspace=ws[0],
                                                 **{k: out.get(k) for k in ("lse", "H", "top_id", "top_logprob")})
        loss, lse, logq = estp.distill_loss(Xs, Ws, ids, logp, T, False, workspace=ws[1],
                                            **{k: out.get("s_" + k) for k in ("loss", "lse", "logq")})
        dX, dW = estp.distill_loss_backward(Xs, Ws, ids, logp, lse, logq, g, T, False, workspace=ws[2],
                                            **{k: out.get(k) for k in ("dX", "dW")})
        return ids, logp, loss, lse, logq, dX, dW

    f32 = lambda *s: torch.empty(s, device="cuda")  # noqa: E731
    out = {"lse": f32(n), "H": f32(n), "top_id": torch.empty(n, K, dtype=torch.int32, device="cuda"),
           "top_logprob": f32(n, K), "s_loss": f32(n), "s_lse": f32(n), "s_logq": f32(n, K), "dX": torch.empty_like(Xs),
           "dW": torch.empty_like(Ws)}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(out, wss)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step(out, wss)
    for rep in range(3):
        if rep:
            Xt.copy_(dev(_inputs(50 + rep, n, 96, V, "bf16")[0]))
            Ws.sub_(0.1 * out["dW"])
        want = step({})
        for a in out.values():
            a.fill_(-1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(captured, want):
            assert torch.equal(a, b), rep
        ids, logp = host(want[0]), host(want[1])
        ref = HD.distill(host(Xs.float()), host(Ws.float()), ids, logp, T, False, host(g), "bf16")
        for name, a in zip(("loss", "lse", "logq", "dX", "dW"), want[2:]):
            assert (np.abs(_wide(a) - ref[name]) <= ref[name + "_bound"]).all(), (rep, name)


def test_weights_past_32_bit_offsets():
    # rows far apart are given, the rest of W is 0
    n, d, V = 4, 4096, 600_000
    g = np.random.default_rng(14)
    from tests.test_gpu_token_loss import _bits
    X = _bits(g.standard_normal((n, d)), "bf16")
    at = np.array([0, 255, 131_071, 300_001, 524_288, 599_999])
    rows = _bits(0.05 * g.standard_normal((len(at), d)), "bf16")
    W = torch.zeros(V, d, dtype=torch.bfloat16, device="cuda")
    W[dev(at)] = dev(rows)
    z = OP.widen(X) @ OP.widen(rows).T
    ref = np.log(np.exp(z).sum(axis=1) + V - len(at))
    bound = OP.lse_bound(X, rows, ref) + 4 * OP.U * (V // 256) * (1 + np.abs(ref))
    logprob, lse, H, ids, top = estp.token_logprobs(dev(X), W, dev(np.full(n, 599_999, np.int32)), len(at))
    full = np.concatenate([z, np.zeros((n, len(at)))], axis=1)  # and the lowest of the other rows
    names = np.concatenate([at, [1, 2, 3, 4, 5, 6]])
    order = np.lexsort((np.broadcast_to(names, full.shape), -full), axis=1)[:, :len(at)]
    np.testing.assert_array_equal(host(ids), names[order])
    assert (np.abs(_wide(logprob) - (z[:, 5] - ref)) <= 2 * bound).all()
    idd = dev(np.tile(at.astype(np.int32), (n, 1)))
    logp = torch.log_softmax(torch.randn(n, len(at), device="cuda"), dim=1)
    loss, lse, logq = estp.distill_loss(dev(X), W, idd, logp, renormalise=False)
    assert (np.abs(_wide(lse) - ref) <= bound).all() and (np.abs(_wide(logq) - (z - ref[:, None])) <= 2 * bound[:, None]).all()
    dX, dW = estp.distill_loss_backward(dev(X), W, idd, logp, lse, logq, renormalise=False)
    p = np.exp(_wide(logp))
    G = p.sum(axis=1, keepdims=True) * np.exp(z - ref[:, None]) - p
    r = 2.0 ** -8 * 1.05
    want = G.T @ OP.widen(X)
    assert (np.abs(_wide(dW[dev(at)]) - want) <= r * (np.abs(want) + np.abs(G).T @ np.abs(OP.widen(X))) + 1e-6).all()
    want = G @ OP.widen(rows)
    assert (np.abs(_wide(dX) - want) <= r * (np.abs(want) + np.abs(G) @ np.abs(OP.widen(rows))) + 1e-5).all()


def test_binding_refuses_mis_sized_tensors():
    X, W = torch.zeros(4, 64, device="cuda"), torch.zeros(9, 64, device="cuda")
    ids, logp, f = torch.zeros(4, 3, dtype=torch.int32, device="cuda"), torch.zeros(4, 3, device="cuda"), torch.zeros(4, device="cuda")
    with pytest.raises(ValueError, match="ids must have 4 rows"):
        estp.distill_loss(X, W, ids[:3], logp)
    with pytest.raises(TypeError, match="ids must be"):
        estp.distill_loss(X, W, ids.long(), logp)
    with pytest.raises(ValueError, match="logp must hold 12"):
        estp.distill_loss(X, W, ids, f)
    for name in ("loss", "lse", "logq"):
        with pytest.raises(ValueError, match=name):
            estp.distill_loss(X, W, ids, logp, **{name: f[:3]})
    for name, bad in (("lse", f[:2]), ("logq", f), ("grad", f[:2])):
        args = {"lse": f, "logq": logp, "grad": None, name: bad}
        with pytest.raises(ValueError, match=name):
            estp.distill_loss_backward(X, W, ids, logp, **args)
    with pytest.raises(ValueError, match="dW must hold 576"):
        estp.distill_loss_backward(X, W, ids, logp, f, logp, dW=X)
    with pytest.raises(estp.EstpError, match="both null"):
        estp.distill_loss_backward(X, W, ids, logp, f, logp, want_dX=False, want_dW=False)
    with pytest.raises(estp.EstpError, match="K must be"):
        estp.distill_loss(X, W, torch.zeros(4, 129, dtype=torch.int32, device="cuda"), torch.zeros(4, 129, device="cuda"))
    with pytest.raises(estp.EstpError, match="temperature"):
        estp.distill_loss(X, W, ids, logp, temperature=0.0)


@pytest.mark.parametrize("dtype,n,other,d,V", [("bf16", 40, 300, 1024, 9000), ("f32", 90, 33, 64, 50000),
                                               ("f32", 20, 130, 64, 50000)])
def test_two_graphs_on_the_same_workspaces(dtype, n, other, d, V):
    # a step of loss and gradients each, of different forms and sizes; eager steps on those workspaces come between
    lib, code, calls, graphs = estp.load(), 0 if dtype == "bf16" else 1, [], []
    most = max(n, other)
    wss = [torch.empty(f(most, d, V, code), dtype=torch.uint8, device="cuda")
           for f in (lib.estp_distill_loss_workspace_size, lib.estp_distill_loss_backward_workspace_size)]
    W = dev(_inputs(71, 1, d, V, dtype)[1])

    def step(X, ids, logp, g, out=(None,) * 5, ws=(None, None)):
        loss, lse, logq = estp.distill_loss(X, W, ids, logp, 1.5, loss=out[0], lse=out[1], logq=out[2], workspace=ws[0])
        dX, dW = estp.distill_loss_backward(X, W, ids, logp, lse, logq, g, 1.5, dX=out[3], dW=out[4], workspace=ws[1])
        return loss, lse, logq, dX, dW

    for m in (n, other):
        X, _, ids, logp, g = _case(70 + m, m, d, V, 9, dtype)
        args = tuple(map(dev, (X, ids, logp, g)))
        calls.append((args, step(*args, ws=wss)))
    torch.cuda.synchronize()
    for args, out in calls:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(*args, out, wss)
        graphs.append(graph)
    for rep in range(3):
        wants = []
        for args, out in calls:
            if rep:
                args[0].copy_(args[0].roll(1, 0))
                args[2].copy_(args[2].flip(1))
            wants.append(step(*args))
            for a in out:
                a.fill_(-1)
        for graph in graphs:
            graph.replay()
        step(*calls[1][0], ws=wss)
        for (_, out), want in zip(calls, wants):
            assert all(torch.equal(a, b) for a, b in zip(out, want)), rep


@pytest.mark.parametrize("dtype,n,d,V", [("bf16", 7, 96, 4001), ("bf16", 64, 1056, 1003), ("f32", 30, 72, 50001),
                                         ("f32", 96, 136, 49153), ("f32", 130, 104, 33001), ("f32", 9, 40, 515)])
def test_outputs_end_where_their_arrays_end(dtype, n, d, V):
    case = _case(n + V, n, d, V, 7, dtype)
    X, W, ids, logp, g = map(dev, case)
    of = {"bf16": (torch.bfloat16, 2), "f32": (torch.float32, 4)}[dtype]
    guards = [Guarded(b) for b in (4 * n, 4 * n, 28 * n, of[1] * n * d, of[1] * V * d)]
    loss, lse, logq = (a.ws.view(torch.float32) for a in guards[:3])
    dX, dW = (a.ws.view(of[0]).view(-1, d) for a in guards[3:])
    estp.distill_loss(X, W, ids, logp, loss=loss, lse=lse, logq=logq.view(n, 7))
    estp.distill_loss_backward(X, W, ids, logp, lse, logq.view(n, 7), g, dX=dX, dW=dW)
    for a in guards:
        a.check()
    ref = HD.distill(*case[:4], 1.0, True, case[4], dtype)
    for name, a in (("loss", loss), ("lse", lse), ("logq", logq.view(n, 7)), ("dX", dX), ("dW", dW)):
        assert (np.abs(_wide(a) - ref[name]) <= ref[name + "_bound"]).all(), name


def test_the_most_tokens_that_a_call_takes():
    # 2^22 tokens of 25 entries, of which a few rows are compared
    n, d, V, K = 1 << 22, 32, 70, 25
    Xs, W, _, _ = _inputs(81, 4096, d, V, "bf16")
    g = torch.Generator(device="cuda").manual_seed(82)
    X = dev(Xs).repeat(n // 4096, 1)
    ids = torch.randint(0, V, (n, K), generator=g, device="cuda", dtype=torch.int32)
    logp = torch.randn(n, K, generator=g, device="cuda")
    grad = torch.rand(n, generator=g, device="cuda")
    loss, lse, logq = estp.distill_loss(X, dev(W), ids, logp)
    dX, _ = estp.distill_loss_backward(X, dev(W), ids, logp, lse, logq, grad, want_dW=False)
    rows = np.concatenate([np.arange(0, 70), np.arange(n // 2 - 30, n // 2 + 30), np.arange(n - 70, n)])
    some = [a[dev(rows)] for a in (ids, logp, grad)]
    ref = HD.distill(Xs[rows % 4096], W, *(host(a) for a in some[:2]), 1.0, True, host(some[2]), "bf16")
    for name, a in (("loss", loss), ("lse", lse), ("logq", logq), ("dX", dX)):
        assert (np.abs(_wide(a[dev(rows)]) - ref[name]) <= ref[name + "_bound"]).all(), name


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_any_constant_may_be_added_to_a_renormalised_row(dtype):
    # the type's lowest and highest numbers among them: as a row of zeros, bit for bit
    n, V = 40, 300
    X, W, ids, logp, g = map(dev, _case(91, n, 64, V, 7, dtype, ignored=0.0))
    logp.zero_()
    want = estp.distill_loss(X, W, ids, logp)
    want += estp.distill_loss_backward(X, W, ids, logp, *want[1:], g)
    big = torch.finfo(torch.float32).max
    for i, c in enumerate((-big, big, -2.0 ** 127, -1.1 * 2.0 ** 127, 1e30, -1e30, -3.0)):
        logp[i::7] = c
    got = estp.distill_loss(X, W, ids, logp)
    got += estp.distill_loss_backward(X, W, ids, logp, *got[1:], g)
    assert torch.isfinite(got[0]).all() and all(torch.equal(a, b) for a, b in zip(got, want))
    # beside other numbers the lowest has no weight
    logp.zero_()
    logp[:, ::2] = -float("inf")
    want = estp.distill_loss(X, W, ids, logp)
    logp[:, ::2] = -big
    live = (((ids >= 0) & (ids < V))[:, 1::2]).any(dim=1)
    assert live.any()
    for a, b in zip(estp.distill_loss(X, W, ids, logp), want):
        assert torch.equal(a[live], b[live])


@pytest.mark.parametrize("n", [70, 130])
def test_f32_from_parts_with_an_infinite_number_in_a_row_of_X(n):
    # products and sums of infinite numbers are as they are without parts: of up to 96 tokens and of more
    d, V, c = 64, 50000, 11
    X, W, ids, logp, g = _case(23, n, d, V, 6, "f32")
    clean = _check((X, W, ids, logp, g), "f32")
    live = (((ids >= 0) & (ids < V)) & (logp > -np.inf)).any(axis=1).nonzero()[0]
    r = int(live[5])
    Xd, Wd, idd, lpd, gd = map(dev, (X, W, ids, logp, g))
    bad = Xd.clone()
    bad[r, c] = float("inf")
    rest = torch.arange(n, device="cuda") != r
    # its own row is lost, and with it dW; the other rows keep their bits
    loss, lse, logq = estp.distill_loss(bad, Wd, idd, lpd)
    dX, dW = estp.distill_loss_backward(bad, Wd, idd, lpd, lse, logq, gd)
    held = dev((ids[r] >= 0) & (ids[r] < V))
    assert not torch.isfinite(lse[r]) and not torch.isfinite(loss[r]) and not torch.isfinite(logq[r][held]).any()
    assert not torch.isfinite(dX[r]).any() and not torch.isfinite(dW).any()
    for name, a in (("loss", loss), ("lse", lse), ("logq", logq), ("dX", dX)):
        assert torch.equal(a[rest], clean[name][rest]), name
    # beside the log-sum-exps of finite rows its weights are infinite where W's number is above 0 and 0 where it is below
    dX, dW = estp.distill_loss_backward(bad, Wd, idd, lpd, clean["lse"], clean["logq"], gd)
    assert not torch.isfinite(dX[r]).any() and torch.equal(dX[rest], clean["dX"][rest])
    other = torch.ones(V, dtype=torch.bool, device="cuda")
    other[idd[r][held].long()] = False
    up, down = other & (Wd[:, c] > 0), other & (Wd[:, c] < 0)
    sign = torch.sign(gd[r] * bad[r])
    assert torch.equal(dW[up], (sign * float("inf")).expand(int(up.sum()), d)) and torch.isnan(dW[down][:, c]).all()
    gd[r] = 0.0
    without = estp.distill_loss_backward(Xd, Wd, idd, lpd, clean["lse"], clean["logq"], gd)[1]
    keep = torch.arange(d, device="cuda") != c
    assert torch.equal(dW[down][:, keep], without[down][:, keep])


@pytest.mark.parametrize("n", [70, 130])
def test_f32_from_parts_of_very_small_numbers(n):
    # tokens of 60 to 95 nats below the others: entries of G from 2^-90 to below the smallest number.  Parts, weights and
    # products below 2^-126 may be taken as 0, which is all that dW is off by beside the bound of fp32 sums
    d, V = 64, 50000
    X, W, ids, logp, g = _case(25, n, d, V, 6, "f32")
    X[:, 0] = 1.0
    far = np.arange(3, V, 5)
    W[far, 0] = -(60.0 + 35.0 * np.random.default_rng(26).uniform(size=len(far))).astype(np.float32)
    Xd, Wd, idd, lpd, gd = map(dev, (X, W, ids, logp, g))
    loss, lse, logq = estp.distill_loss(Xd, Wd, idd, lpd)
    dX, dW = estp.distill_loss_backward(Xd, Wd, idd, lpd, lse, logq, gd)
    ref = HD.distill(X, W, ids, logp, 1.0, True, g, "f32")
    small = n * 2.0 ** -126 * (3 * np.abs(X).max() + 8)
    for name, a, room in (("loss", loss, 0), ("lse", lse, 0), ("logq", logq, 0), ("dX", dX, 0), ("dW", dW, small)):
        assert (np.abs(_wide(a) - ref[name]) <= ref[name + "_bound"] + room).all(), name
    tiny = np.abs(ref["dW"][far]).max(axis=1)
    assert (tiny < 2.0 ** -118).any() and (tiny > 2.0 ** -100).any()

"""Log-probabilities, entropies and alternatives on the GPU against the fp64 oracle (oracle/head.py), at the bounds it
derives; alternatives under the margin rule, and exactly where the logits are exact."""
import numpy as np
import pytest
import torch

import paper_2608_15592_amd as estp
from oracle import head as HD
from oracle import operators as OP
from tests._util import dev, host
from tests.test_gpu_operators_workspace import Guarded
from tests.test_gpu_token_loss import _bits, _inputs, _wide

pytestmark = pytest.mark.gpu


def _check(X, W, t, k, temperature=1.0, **kw):
    got = estp.token_logprobs(dev(X), dev(W), None if t is None else dev(t), k, temperature=temperature, **kw)
    ref = HD.token_logprobs(X, W, t, k, temperature)
    for name, a in zip(("logprob", "lse", "H"), got):
        if a is not None:
            over = np.abs(_wide(a) - ref[name]) - ref[name + "_bound"]
            assert (over <= 0).all(), f"{name}: {over.max()} over the bound at row {over.argmax()}"
    ids, top = host(got[3]), _wide(got[4])
    assert ids.shape == top.shape == (len(X), k)
    if k:
        assert (ids >= 0).all() and (ids < len(W)).all()
        assert all(len(set(r)) == k for r in ids.tolist())
        # the j-th largest as computed is no further from the j-th largest than a logit's error, nor from its own
        at, best = np.take_along_axis(ref["s"], ids, 1), np.take_along_axis(ref["s"], ref["top_id"], 1)
        assert (np.abs(at - best) <= ref["margin"][:, None]).all()
        over = np.abs(top - (at - ref["lse"][:, None])) - ref["logprob_bound"][:, None]
        assert (over <= 0).all()
        assert (np.diff(host(got[4]), axis=1) <= 0).all()
    if t is not None:
        assert (host(got[0])[(t < 0) | (t >= len(W))] == 0).all()
    return got


SHAPES = [(1, 32, 1, 1), (1, 64, 7, 7), (3, 32, 257, 20), (64, 96, 1000, 1), (65, 64, 256, 128), (127, 160, 4099, 5),
          (257, 128, 8193, 33), (385, 64, 16640, 8), (1030, 64, 3001, 64)]


@pytest.mark.parametrize("n,d,V,k", SHAPES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_values_and_alternatives(n, d, V, k, dtype):
    X, W, t, _ = _inputs(n + V, n, d, V, dtype, ignored=0.2 if n > 3 else 0.0)
    _check(X, W, t, k)


@pytest.mark.parametrize("temperature", [0.1, 0.7, 2.0, 100.0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_temperatures(temperature, dtype):
    X, W, t, _ = _inputs(3, 140, 128, 3000, dtype)
    _check(X, W, t, 12, temperature)


@pytest.mark.parametrize("n,d,V", [(5, 8, 30), (70, 40, 300), (130, 72, 1003)])
def test_f32_widths(n, d, V):
    X, W, t, _ = _inputs(n, n, d, V, "f32")
    _check(X, W, t, 9)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_without_targets_or_alternatives(dtype):
    X, W, t, _ = _inputs(6, 90, 64, 700, dtype)
    full = _check(X, W, t, 4)
    bare = _check(X, W, None, 0)
    assert bare[0] is None and torch.equal(bare[1], full[1]) and torch.equal(bare[2], full[2])
    some = _check(X, W, None, 4)
    assert torch.equal(some[3], full[3]) and torch.equal(some[4], full[4])


def _exact_inputs(seed, n, d, V, dtype):
    """Logits that are whole multiples of 2^-9 and exact in 32 bits in any order of summation: ties are frequent."""
    g = np.random.default_rng(seed)
    X, W = g.integers(-8, 9, (n, d)) / 8.0, g.integers(-12, 13, (V, d)) / 64.0
    return _bits(X, dtype), _bits(W, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,d,V,k", [(1, 32, 300, 128), (33, 32, 20000, 128), (300, 64, 9000, 20), (2100, 32, 8700, 50)])
def test_ties_go_to_the_lowest_index(n, d, V, k, dtype):
    X, W = _exact_inputs(n, n, d, V, dtype)
    ids, top = estp.token_logprobs(dev(X), dev(W), None, k)[3:]
    z = OP.widen(X) @ OP.widen(W).T
    np.testing.assert_array_equal(host(ids), np.argsort(-z, axis=1, kind="stable")[:, :k])
    tied = np.diff(np.sort(z, axis=1)[:, ::-1][:, :k], axis=1) == 0
    assert tied.any() and (np.diff(host(top), axis=1)[tied] == 0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [2, 2300])
def test_equal_logits(dtype, n):
    # rows of zeros, as a padded batch has them: every token equally probable
    V, k = 30000, 128
    X, W = _bits(np.zeros((n, 32)), dtype), _bits(np.random.default_rng(1).standard_normal((V, 32)), dtype)
    logprob, lse, H, ids, top = estp.token_logprobs(dev(X), dev(W), dev(np.full(n, 7, np.int32)), k)
    assert torch.equal(ids, torch.arange(k, dtype=torch.int32, device="cuda").expand(n, k))
    for a in (-logprob, lse, H, -top):
        assert (np.abs(_wide(a) - np.log(V)) <= 64 * OP.U * np.log(V)).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,V", [(3, 16000), (700, 16000), (385, 40001), (2305, 33000)])
@pytest.mark.parametrize("order", [1, -1])
def test_a_vocabulary_in_order_of_its_logits(dtype, n, V, order):
    # every next row of W is more (or less) probable than all before it: no bound from a sample keeps any out for long
    k = 100
    X, W, v = np.zeros((n, 32)), np.zeros((V, 32)), np.arange(V)
    X[:, 0], X[:, 1], X[:, 2] = 1.0, 1.0 / 128, 1.0 / 16384
    W[:, 0], W[:, 1], W[:, 2] = v >> 14, v >> 7 & 127, v & 127  # logit: v / 16384
    ids = estp.token_logprobs(dev(_bits(X, dtype)), dev(_bits(W[::order], dtype)), None, k)[3]
    want = np.arange(k) if order < 0 else V - 1 - np.arange(k)
    assert (host(ids) == want).all()


# few tokens, whose part of the depth stays in registers; vocabularies that end within a tile of 16 rows, fewer tiles than
# compute units, and several rounds of them
FEW = [(1, 1024, 5000), (16, 1024, 9001), (17, 1024, 77), (64, 1024, 4100), (5, 1536, 8197), (33, 1536, 4097),
       (64, 1536, 12300), (2, 2048, 16400), (31, 2048, 5003), (50, 2048, 4099), (9, 2560, 4500), (32, 2560, 4500),
       (40, 2560, 4500), (16, 3584, 4111), (20, 3584, 5000), (1, 4096, 4600), (16, 4096, 8200), (32, 4096, 4097),
       (33, 4096, 4097), (12, 512, 3000), (12, 4352, 3000)]


@pytest.mark.parametrize("n,d,V", FEW)
def test_few_tokens(n, d, V):
    X, W, t, _ = _inputs(n + d, n, d, V, "bf16", lean=3.0)
    ws = Guarded(estp.load().estp_token_logprobs_workspace_size(n, d, V, 6, 0))
    got = _check(X, W, t, 6, 0.9, workspace=ws.ws)
    ws.check()
    again = estp.token_logprobs(dev(X), dev(W), dev(t), 6, 0.9)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


# fp32 calls whose products are formed from parts in bf16: widths of a stage and others, tokens of each tile's width
SPLIT = [(1, 128, 98400, 2), (16, 264, 98500, 9), (30, 520, 50000, 9), (37, 1000, 49200, 20), (64, 264, 61000, 5),
         (90, 256, 50000, 20), (100, 72, 140001, 3), (200, 512, 17003, 128), (500, 256, 8300, 9)]


@pytest.mark.parametrize("n,d,V,k", SPLIT)
def test_f32_from_parts(n, d, V, k):
    X, W, t, _ = _inputs(n + d, n, d, V, "f32", ignored=0.1)
    ws = Guarded(estp.load().estp_token_logprobs_workspace_size(n, d, V, k, 1))
    got = _check(X, W, t, k, 1.1, workspace=ws.ws)
    ws.check()
    again = estp.token_logprobs(dev(X), dev(W), dev(t), k, 1.1)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


def test_f32_logits_are_as_exact_as_fp32_sums():
    # numbers of 24 significant bits and of very different sizes, logits that cancel: off by less than d roundings of
    # the largest partial sum (a chain of fp32 FMAs is off by up to d)
    n, d, V = 64, 512, 50000
    g = np.random.default_rng(5)
    X = (g.standard_normal((n, d)) * 2.0 ** g.integers(-6, 7, (n, d))).astype(np.float32)
    W = (g.standard_normal((V, d)) * 2.0 ** g.integers(-9, 3, (V, d))).astype(np.float32)
    top = estp.token_logprobs(dev(X), dev(W), None, 128, temperature=64.0)
    z = X.astype(np.float64) @ W.astype(np.float64).T
    size = np.abs(X).astype(np.float64) @ np.abs(W).astype(np.float64).T
    ids = host(top[3])
    got = (_wide(top[4]) + _wide(top[1])[:, None]) * 64.0
    at, of = np.take_along_axis(z, ids, 1), np.take_along_axis(size, ids, 1)
    # (the log-probability itself is rounded, at most twice at its own size and that of lse)
    room = 4 * OP.U * (np.abs(at) + 64.0 * np.abs(_wide(top[1])[:, None]))
    assert (np.abs(got - at) <= 8 * OP.U * of + room).all()


@pytest.mark.parametrize("dtype,n,V", [("bf16", 1, 5000), ("bf16", 20, 5000), ("bf16", 60, 5000), ("f32", 60, 49300)])
def test_a_non_finite_row_of_weights_stays_in_its_row(dtype, n, V):
    d = 2048
    X, W, _, _ = _inputs(n, n, d, V, dtype)
    want = estp.token_logprobs(dev(X), dev(W), None, 5)
    low = np.argmin(OP.widen(X) @ OP.widen(W).T, axis=1)[0]  # not an alternative of any row's, or of few
    Wd = dev(W)
    for at in (0, 1, d // 8, d - 1):  # in each wave's eighth
        Wd[low] = dev(W)[low]
        Wd[low, at] = -float("inf")
        Xd = dev(X)
        Xd[:, at] = 1.0
        ids = estp.token_logprobs(Xd, Wd, None, 5)[3]
        z = OP.widen(host(Xd.float())) @ OP.widen(W).T
        z[:, low] = -np.inf
        best, margin = np.sort(z, axis=1)[:, ::-1][:, :5], 2 * OP.logit_bound(host(Xd.float()), W)
        assert (np.abs(np.take_along_axis(z, host(ids), 1) - best) <= margin[:, None]).all()
    assert want[3].shape == (n, 5)


# many tokens of bf16 and a large vocabulary: bounds from a sample of its tiles, the last of them short or whole
LARGE = [(385, 32, 33000, 20), (400, 96, 32768, 1), (1500, 64, 33001, 128), (2048, 32, 40000, 64), (2300, 64, 36097, 5),
         (500, 32, 70000, 33), (513, 64, 33000, 0)]


@pytest.mark.parametrize("n,d,V,k", LARGE)
def test_large_vocabularies(n, d, V, k):
    X, W, t, _ = _inputs(n + V, n, d, V, "bf16", ignored=0.2)
    ws = Guarded(estp.load().estp_token_logprobs_workspace_size(n, d, V, k, 0))
    got = _check(X, W, t, k, 1.3, workspace=ws.ws)
    ws.check()
    again = estp.token_logprobs(dev(X), dev(W), dev(t), k, 1.3)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.parametrize("n,larger", [(385, 2048), (1, 2500), (384, 385), (700, 20000), (2049, 4000)])
def test_on_a_larger_calls_workspace(n, larger):
    d, V, k = 32, 33000, 30
    X, W, t, _ = _inputs(n, n, d, V, "bf16")
    want = estp.token_logprobs(dev(X), dev(W), dev(t), k)
    ws = Guarded(estp.load().estp_token_logprobs_workspace_size(larger, d, V, 40, 0))
    got = estp.token_logprobs(dev(X), dev(W), dev(t), k, workspace=ws.ws)
    ws.check()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("n,V,k", [(600, 33000, 128), (2100, 33000, 20), (400, 60000, 1)])
def test_ties_of_large_vocabularies(n, V, k):
    X, W = _exact_inputs(n, n, 32, V, "bf16")
    X[5] = 0
    ids = estp.token_logprobs(dev(X), dev(W), None, k)[3]
    z = OP.widen(X) @ OP.widen(W).T
    np.testing.assert_array_equal(host(ids), np.argsort(-z, axis=1, kind="stable")[:, :k])


def test_non_finite_logits_of_large_vocabularies():
    # infinities and NaN within and outside of the sample, one row NaN throughout
    n, V, k = 500, 33000, 16
    X, W = _exact_inputs(n, n, 32, V, "bf16")
    Xd, Wd = dev(X), dev(W)
    Xd[:, 0], Wd[:, 0] = 1.0, 0.0
    low, nan = [0, 300, 20000, 32999], [5, 700, 32998]
    Wd[low, 0], Wd[nan, 0] = float("-inf"), float("nan")
    Xd[7] = float("nan")
    _, lse, _, ids, _ = estp.token_logprobs(Xd, Wd, None, k)
    assert torch.isnan(lse).all() and torch.equal(ids[7], torch.arange(k, dtype=torch.int32, device="cuda"))
    z = OP.widen(host(Xd.float())) @ OP.widen(np.nan_to_num(host(Wd.float()), nan=0.0, neginf=0.0)).T
    z[:, low + nan] = -np.inf
    want = np.argsort(-z, axis=1, kind="stable")[:, :k]
    keep = np.arange(n) != 7
    np.testing.assert_array_equal(host(ids)[keep], want[keep])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [4, 2300])
def test_non_finite_logits(dtype, n):
    # a NaN row of W and one of -inf and +inf logits: NaN ranks last, its values are NaN
    V, k = 9001, 16
    X, W = _exact_inputs(n, n, 32, V, dtype)
    Xd, Wd = dev(X), dev(W)
    Xd[1:, 0] = 1.0
    Xd[0, 0] = 0.0
    Wd[:, 0] = 0.0
    Wd[8500, 0] = float("-inf")
    Xd[0] = float("nan")
    logprob, lse, H, ids, top = estp.token_logprobs(Xd, Wd, dev(np.full(n, 5, np.int32)), k)
    assert torch.isnan(lse[0]) and torch.isnan(logprob[0]) and torch.isnan(H[0]) and torch.isnan(top[0]).all()
    assert torch.equal(ids[0], torch.arange(k, dtype=torch.int32, device="cuda"))
    z = OP.widen(host(Xd.float())[1:]) @ OP.widen(np.where(np.isinf(host(Wd.float())), 0, host(Wd.float()))).T
    z[:, 8500] = -np.inf
    np.testing.assert_array_equal(host(ids)[1:], np.argsort(-z, axis=1, kind="stable")[:, :k])
    for a in (logprob, lse, H, top):
        assert torch.isfinite(a[1:]).all()
    Wd[8500, 0], Wd[3, 0] = 0.0, float("inf")
    ids, top = estp.token_logprobs(Xd, Wd, None, k)[3:]
    assert (ids[1:, 0] == 3).all() and not torch.isfinite(top[1:, 0]).any()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [3, 200, 2500])
def test_a_given_alternative_has_one_value(dtype, n):
    X, W, t, _ = _inputs(17, n, 96, 5000, dtype, lean=12.0)
    logprob, _, _, ids, top = estp.token_logprobs(dev(X), dev(W), dev(t), 30)
    hit = ids == dev(t)[:, None]
    assert hit.any() and torch.equal(top[hit], logprob[hit.any(dim=1)])


def test_tokens_in_blocks_and_the_same_bits_twice():
    # more tokens than one block; a row's values do not depend on its neighbours within a block of one size
    n, d, V, k = 17000, 32, 2500, 10
    X, W, t, _ = _inputs(18, n, d, V, "bf16", ignored=0.1)
    first = _check(X, W, t, k)
    again = estp.token_logprobs(dev(X), dev(W), dev(t), k)
    assert all(torch.equal(a, b) for a, b in zip(first, again))


def test_on_another_stream_with_given_outputs():
    n, d, V, k = 300, 64, 9000, 7
    X, W, t, _ = _inputs(19, n, d, V, "bf16")
    want = _check(X, W, t, k)
    out = {"logprob": torch.empty(n, device="cuda"), "lse": torch.empty(n, device="cuda"),
           "H": torch.empty(n, device="cuda"), "top_id": torch.empty(n, k, dtype=torch.int32, device="cuda"),
           "top_logprob": torch.empty(n, k, device="cuda")}
    ws = torch.full((estp.load().estp_token_logprobs_workspace_size(n, d, V, k, 0),), 255, dtype=torch.uint8,
                    device="cuda")
    Xd, Wd, td = dev(X), dev(W), dev(t)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = estp.token_logprobs(Xd, Wd, td, k, workspace=ws, stream=side, **out)
    torch.cuda.current_stream().wait_stream(side)
    for a, b, c in zip(got, want, out.values()):
        assert a is c and torch.equal(a, b)


def test_replayed_in_a_graph():
    n, d, V, k = 300, 64, 9000, 7
    X, W, t, _ = _inputs(20, n, d, V, "bf16")
    Xd, Wd, td = dev(X), dev(W), dev(t)
    ws = torch.empty(estp.load().estp_token_logprobs_workspace_size(n, d, V, k, 0), dtype=torch.uint8, device="cuda")
    out = estp.token_logprobs(Xd, Wd, td, k)
    names = ("logprob", "lse", "H", "top_id", "top_logprob")

    def step():
        estp.token_logprobs(Xd, Wd, td, k, workspace=ws, **dict(zip(names, out)))

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
        if rep:
            Xd.copy_(dev(_inputs(20 + rep, n, d, V, "bf16")[0]))
        want = estp.token_logprobs(Xd, Wd, td, k)
        for a in out:
            a.fill_(-1)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), rep


def test_binding_refuses_mis_sized_tensors():
    X, W = torch.zeros(4, 64, device="cuda"), torch.zeros(9, 64, device="cuda")
    t, f = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(4, device="cuda")
    with pytest.raises(ValueError, match="targets must hold 4"):
        estp.token_logprobs(X, W, t[:3], 2)
    with pytest.raises(ValueError, match="disagree on d"):
        estp.token_logprobs(X, W[:, :32].contiguous(), t, 2)
    for name in ("logprob", "lse", "H", "top_id", "top_logprob"):
        with pytest.raises((ValueError, TypeError), match=name):
            estp.token_logprobs(X, W, t, 2, **{name: f[:3]})
    with pytest.raises(ValueError, match="logprob needs targets"):
        estp.token_logprobs(X, W, None, 2, logprob=f)
    for k in (10, 129, -1, 2 ** 31 - 1):
        with pytest.raises(estp.EstpError, match="k"):
            estp.token_logprobs(X, W, t, k)
    with pytest.raises(ValueError, match="k must"):  # not one of 32 bits
        estp.token_logprobs(X, W, t, 2 ** 32 + 1)
    for temperature in (0.0, -1.0, float("nan"), float("inf")):
        with pytest.raises(estp.EstpError, match="temperature"):
            estp.token_logprobs(X, W, t, 2, temperature=temperature)
    with pytest.raises(estp.EstpError, match="workspace"):
        estp.token_logprobs(X, W, t, 2, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("dtype,n,other,d,V", [("bf16", 12, 700, 1024, 33000), ("bf16", 500, 3, 64, 33000),
                                               ("f32", 40, 17, 64, 50000), ("f32", 200, 9, 32, 9000)])
def test_two_graphs_on_one_workspace(dtype, n, other, d, V):
    # the calls of two graphs have different forms and sizes; eager calls on that workspace come between the replays
    k, code = 11, 0 if dtype == "bf16" else 1
    calls, graphs = [], []
    size = estp.load().estp_token_logprobs_workspace_size(max(n, other), d, V, k, code)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    W = dev(_inputs(61, 1, d, V, dtype)[1])
    for m in (n, other):
        X, _, t, _ = _inputs(60 + m, m, d, V, dtype)
        X, t = dev(X), dev(t)
        calls.append((X, t, estp.token_logprobs(X, W, t, k, workspace=ws)))
    names = ("logprob", "lse", "H", "top_id", "top_logprob")
    torch.cuda.synchronize()
    for X, t, out in calls:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            estp.token_logprobs(X, W, t, k, workspace=ws, **dict(zip(names, out)))
        graphs.append(graph)
    for rep in range(3):
        wants = []
        for X, t, out in calls:
            if rep:
                X.copy_(X.roll(1, 0) if rep == 1 else -X)
            wants.append(estp.token_logprobs(X, W, t, k))
            for a in out:
                a.fill_(-1)
        for graph in graphs:
            graph.replay()
        estp.token_logprobs(calls[0][0], W, None, k, workspace=ws)
        for (_, _, out), want in zip(calls, wants):
            assert all(torch.equal(a, b) for a, b in zip(out, want)), rep


@pytest.mark.parametrize("dtype,n,d,V,k", [("bf16", 3, 1024, 4001, 5), ("bf16", 390, 32, 33001, 17), ("bf16", 100, 64, 999, 128),
                                           ("f32", 33, 72, 50001, 3), ("f32", 5, 40, 515, 20)])
def test_outputs_end_where_their_arrays_end(dtype, n, d, V, k):
    X, W, t, _ = _inputs(n + V, n, d, V, dtype, ignored=0.2)
    X, W, t = dev(X), dev(W), dev(t)
    guards = [Guarded(4 * n * m) for m in (1, 1, 1, k, k)]
    out = [a.ws.view(torch.int32 if i == 3 else torch.float32) for i, a in enumerate(guards)]
    out[3:] = [a.view(n, k) for a in out[3:]]
    estp.token_logprobs(X, W, t, k, **dict(zip(("logprob", "lse", "H", "top_id", "top_logprob"), out)))
    for a in guards:
        a.check()
    assert all(torch.equal(a, b) for a, b in zip(out, estp.token_logprobs(X, W, t, k)))


@pytest.mark.parametrize("k", [0, 16])
@pytest.mark.parametrize("low", [[0], [300], [20000], [32999], [0, 300, 1024, 1280, 9000, 17000, 20000, 25700, 32998, 32999]])
@pytest.mark.parametrize("n", [450, 2048])
def test_tokens_of_no_probability_leave_an_entropy(n, low, k):
    # rows of W masked out by -inf, in tiles of the sample, in others (of 2048 tokens each workgroup has several of them)
    # and in the last, which is short: the values are those of the vocabulary without them
    V = 33000
    X, W = _exact_inputs(n + k, n, 32, V, "bf16")
    Xd, Wd = dev(X), dev(W)
    Xd[:, 0] = 1.0
    Wd[low, 0] = float("-inf")
    t = np.random.default_rng(k).integers(0, V, n).astype(np.int32)
    t[np.isin(t, low)] = 7
    got = estp.token_logprobs(Xd, Wd, dev(t), k, 0.7)
    rest, some = np.delete(np.arange(V), low), np.arange(0, n, 29)  # (tokens of all tiles' columns)
    logprob, lse, H, ids, top = (a[dev(some)] for a in got)
    ref = HD.token_logprobs(_bits(host(Xd.float()), "bf16")[some], W[rest], np.searchsorted(rest, t[some]), k, 0.7)
    for name, a in (("logprob", logprob), ("lse", lse), ("H", H)):
        assert (np.abs(_wide(a) - ref[name]) <= ref[name + "_bound"]).all(), name
    np.testing.assert_array_equal(host(ids), rest[ref["top_id"]])
    assert (np.abs(_wide(top) - ref["top_logprob"]) <= ref["logprob_bound"][:, None]).all()
    assert torch.isfinite(got[2]).all()


def test_entropy_of_a_mode_far_above_the_first_tile():
    # a background of zeros and, 55 to 62 units of ln 2 above it, two tokens that a lane folds together in one of its
    # later tiles: all else weighs less than 2^-40.  What is left are roundings of the second weight's exponent (at most 6
    # in base 2: 4 u), of two weights and their sums (2 u each), of a logarithm below 1 and of H and its change of base
    n, V, first, u = 2048, 33000, 2300, OP.U
    X, W, i = np.zeros((n, 96)), np.zeros((V, 96)), np.arange(n)
    place = first + 472 * np.arange(64)  # of 118 rows of four each: every 16-row block and wave
    which, height, gap = i % 64, 38.0 + (i % 19) * 0.25, (1 + i * 7 % 61) / 16.0
    X[i, which], X[:, 64], X[:, 65] = height, gap, (i % 128) / 1024.0
    W[place, np.arange(64)] = W[place + 1, np.arange(64)] = 1.0
    W[place + 1, 64], W[place, 65], W[place + 1, 65] = -1.0, 1.0, 1.0
    for k in (0, 3):
        lse, H, ids = estp.token_logprobs(dev(_bits(X, "bf16")), dev(_bits(W, "bf16")), None, k)[1:4]
        two = np.log1p(np.exp(-gap))
        want = two + gap / (1.0 + np.exp(gap))
        assert (np.abs(_wide(H) - want) <= 24 * u * (1.0 + want)).all()
        assert (np.abs(_wide(lse) - (height + X[:, 65] + two)) <= 4 * u * 64).all()
        if k:
            np.testing.assert_array_equal(host(ids)[:, :2], place[which][:, None] + np.arange(2))


@pytest.mark.parametrize("n", [400, 2000])
def test_entropy_of_peaked_distributions(n):
    # modes of 10 to 17 nats over logits of deviation 0.9, in any tile, at temperature 0.7.  A sum of weights is off by its
    # chain, 512 u, by 40 u of merges and by the weights' own errors, 300 u: exponents of up to 60 in base 2 and three moves
    # of a reference of up to 60.  So the mode's is off by 600 u, and the others' move H by 852 u p (|log p| + H) at most
    d, V = 64, 128256
    g = np.random.default_rng(n)
    W = np.zeros((V, d))
    W[:, :32] = g.integers(-8, 9, (V, 32)) / 32.0
    X = np.zeros((n, d))
    X[:, :32] = g.integers(-8, 9, (n, 32)) / 8.0
    X[:, :32] *= 0.7 * 0.9 / np.sqrt((X[:, :32] ** 2).sum(axis=1, keepdims=True) * (W[:, :32] ** 2).mean())
    X[:, :32] = np.round(X[:, :32] * 64) / 64
    t = g.integers(0, V, n)
    W[t[:31], 32 + np.arange(31)] = 1.0
    X[np.arange(n), 32 + np.arange(n) % 31] = 0.7 * g.uniform(10.0, 17.0, n)
    X, W = _bits(X, "bf16"), _bits(W, "bf16")
    H = estp.token_logprobs(dev(X), dev(W), None, 5, 0.7)[2]
    some = np.arange(0, n, n // 62)
    ref = HD.token_logprobs(X[some], W, None, 5, 0.7)["H"]
    assert (np.abs(_wide(H)[some] - ref) <= (600 + 1704 * ref) * OP.U).all() and ref.min() < 0.6


@pytest.mark.parametrize("dtype,n,V", [("bf16", 1, 5000), ("bf16", 20, 5000), ("bf16", 60, 5000), ("f32", 60, 49300)])
def test_values_beside_a_row_of_weights_with_an_infinite_number(dtype, n, V):
    # at places of the depth that different waves take: the values are those of the vocabulary without that row
    d = 2048
    X, W, _, _ = _inputs(n, n, d, V, dtype)
    low = V // 3
    rest = np.delete(np.arange(V), low)
    for at in (0, d // 8 + 1, d // 2, d - 1):
        Xd, Wd = dev(X), dev(W)
        Xd[:, at], Wd[low, at] = 1.0, float("-inf")
        _, lse, H, ids, top = estp.token_logprobs(Xd, Wd, None, 5)
        ref = HD.token_logprobs(_bits(host(Xd.float()), dtype), W[rest], None, 5)
        assert (np.abs(_wide(lse) - ref["lse"]) <= ref["lse_bound"]).all()
        assert (np.abs(_wide(H) - ref["H"]) <= ref["H_bound"]).all()
        assert (host(ids) != low).all()
        where = np.searchsorted(rest, host(ids))
        at_ids, best = (np.take_along_axis(ref["s"], i, 1) for i in (where, ref["top_id"]))
        assert (np.abs(at_ids - best) <= ref["margin"][:, None]).all()
        assert (np.abs(_wide(top) - (at_ids - ref["lse"][:, None])) <= ref["logprob_bound"][:, None]).all()

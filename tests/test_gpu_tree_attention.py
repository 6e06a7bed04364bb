"""Attention of drafted tokens over a cache, and the account of the weight its slots receive, on the GPU against
the fp64 oracle at the bounds it derives (oracle/operators.py)."""
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


def _mask_tensor(masks):
    return torch.tensor([m - (1 << 64) if m >> 63 else m for m in masks], dtype=torch.int64).cuda()


class Case:
    def __init__(self, seed, lens, T, Hq, Hkv, dh, dtype, tree=True, cap=None, sharp=1.0):
        g = np.random.default_rng(seed)
        self.lens, self.T, self.dtype = np.array(lens, np.int32), np.array(T), dtype
        self.cu = np.concatenate([[0], np.cumsum(T)]).astype(np.int32)
        n_q, B = int(self.cu[-1]), len(lens)
        self.max_q, self.max_kv = max(1, int(max(T))), max(1, int((self.lens + self.T).max()))
        self.cap = cap or self.max_kv
        self.Q = _bits(sharp * g.standard_normal((n_q, Hq, dh)), dtype)
        self.K, self.V = (_bits(g.standard_normal((B, Hkv, self.cap, dh)), dtype) for _ in range(2))
        self.masks = None
        if tree:
            self.masks = []
            for t in T:
                m = []
                for i in range(t):
                    parent = int(g.integers(-1, i)) if i else -1
                    m.append((m[parent] if parent >= 0 else 0) | 1 << i)
                self.masks += m
        self.acc = g.exponential(size=(B, Hkv, self.cap)).astype(np.float32)

    def mask(self):
        return None if self.masks is None else _mask_tensor(self.masks)

    def oracle(self, **kw):
        return OP.tree_attention(self.Q, self.K, self.V, self.lens, self.cu, self.masks, dtype=self.dtype, **kw)

    def args(self):
        return dev(self.lens), dev(self.cu), self.max_q, self.max_kv

    def attend(self, **kw):
        kw.setdefault("tree_mask", self.mask())
        return estp.tree_attention(dev(self.Q), dev(self.K), dev(self.V), *self.args(), **kw)

    def check(self, O, lse, acc=None, ref=None, skip=()):
        ref = ref or self.oracle()
        rows = [i for i in range(len(self.Q)) if i not in skip]
        assert (np.abs(_wide(O) - ref["O"]) <= ref["O_bound"])[rows].all()
        empty = np.isneginf(ref["lse"])
        got = _wide(lse)
        assert np.isneginf(got[empty]).all()
        assert (np.abs(got - np.where(empty, 0, ref["lse"]))[~empty] <= ref["lse_bound"][~empty]).all()
        if acc is not None:
            self.check_account(acc, ref)

    def check_account(self, acc, ref):
        want = self.acc + ref["got"]
        assert (np.abs(_wide(acc) - want) <= ref["got_bound"] + 2 * OP.U * np.abs(want)).all()
        untouched = ref["got"] == 0
        np.testing.assert_array_equal(host(acc)[untouched], self.acc[untouched])


CASES = [
    # lens, T, Hq, Hkv, dh
    ([0], [1], 1, 1, 32),
    ([1], [1], 2, 1, 64),
    ([33], [1], 4, 4, 128),
    ([700], [5], 12, 2, 128),
    ([63, 64, 65], [1, 1, 1], 8, 2, 64),
    ([0, 127, 300, 5], [3, 0, 64, 31], 8, 2, 64),
    ([1000, 17, 2049], [1, 16, 7], 32, 8, 128),
    ([129, 511], [64, 33], 7, 1, 32),
    ([40, 900], [23, 9], 6, 3, 128),
    ([5000], [1], 32, 8, 64),
    ([300], [2], 48, 2, 128),
]


@pytest.mark.parametrize("lens,T,Hq,Hkv,dh", CASES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tree", [True, False])
def test_attention_and_account(lens, T, Hq, Hkv, dh, dtype, tree):
    c = Case(sum(lens) + dh, lens, T, Hq, Hkv, dh, dtype, tree, cap=max(a + b for a, b in zip(lens, T)) + 3)
    acc = dev(c.acc)
    O, lse = c.attend(acc=acc)
    ref = c.oracle()
    c.check(O, lse, acc, ref)
    O2, lse2 = c.attend()  # without the account: the same, bit for bit
    assert torch.equal(O, O2) and torch.equal(lse, lse2)
    # the account by itself, all rows and some of them
    acc2 = dev(c.acc)
    estp.tree_importance(dev(c.Q), dev(c.K), lse, *c.args(), acc2, tree_mask=c.mask())
    c.check_account(acc2, ref)
    w = np.random.default_rng(1).choice([0.0, 1.0, 0.25], len(c.Q)).astype(np.float32)
    acc3 = dev(c.acc)
    estp.tree_importance(dev(c.Q), dev(c.K), lse, *c.args(), acc3, tree_mask=c.mask(), row_weight=dev(w))
    c.check_account(acc3, c.oracle(row_weight=w))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_sharp_scores(dtype):
    c = Case(3, [800, 90], [4, 9], 8, 2, 64, dtype, sharp=12.0)
    acc = dev(c.acc)
    O, lse = c.attend(acc=acc)
    c.check(O, lse, acc)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_see_nothing(dtype):
    c = Case(4, [0, 0], [5, 3], 4, 2, 64, dtype)
    c.masks[0] = c.masks[6] = 0          # nothing cached, nothing drafted
    c.masks[3] = 0b10100                 # the bits of tokens the sequence has
    c.masks[5] = 1 << 63 | 1             # and one it has not
    acc = dev(c.acc)
    O, lse = c.attend(acc=acc)
    c.check(O, lse, acc)
    assert not O[0].any() and not O[6].any() and torch.isneginf(lse[:, 0]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", [0, 50, 64])
def test_unseen_slots_may_hold_anything(dtype, lens):
    # non-finite keys and values in the drafted slots a row does not see, and past the sequence
    c = Case(5, [lens], [20], 8, 2, 64, dtype, cap=lens + 90)
    c.masks = [m & ~(1 << 3) if i != 3 else m for i, m in enumerate(c.masks)]
    clean = c.attend(), dev(c.acc)
    estp.tree_importance(dev(c.Q), dev(c.K), clean[0][1], *c.args(), clean[1], tree_mask=c.mask())
    K, V = dev(c.K), dev(c.V)
    bad = [float("nan"), float("inf"), float("-inf")]
    for j, x in enumerate(bad):
        K[:, :, lens + 20 + j::3] = x
        V[:, :, lens + 20 + j::3] = x
    K[:, 0, lens + 3], V[:, 0, lens + 3] = float("nan"), float("inf")
    V[:, 1, lens + 3, ::2] = float("nan")
    acc = dev(c.acc)
    O, lse = estp.tree_attention(dev(c.Q), K, V, *c.args(), tree_mask=c.mask(), acc=acc)
    rows = torch.arange(20, device="cuda") != 3
    assert torch.equal(O[rows], clean[0][0][rows]) and torch.equal(lse[:, rows], clean[0][1][:, rows])
    assert torch.isnan(O[3, :4]).all() and not torch.isfinite(O[3, 4:, ::2]).any()
    # the account leaves out the row that sees them
    acc, w = dev(c.acc), rows.float()
    acc2 = dev(c.acc)
    estp.tree_importance(dev(c.Q), K, lse, *c.args(), acc, tree_mask=c.mask(), row_weight=w)
    estp.tree_importance(dev(c.Q), dev(c.K), clean[0][1], *c.args(), acc2, tree_mask=c.mask(), row_weight=w)
    assert torch.equal(acc, acc2) and torch.isfinite(acc).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_and_slots_outside_the_sequences_are_left_alone(dtype):
    c = Case(6, [100, 30], [4, 2], 8, 2, 64, dtype, cap=120)
    Q = torch.cat([dev(c.Q), torch.full((2, 8, 64), float("nan"), device="cuda").to(dev(c.Q).dtype)])
    O, lse, acc = torch.full_like(Q, 7.0), torch.full((8, 8), 7.0, device="cuda"), dev(c.acc)
    mask = torch.cat([c.mask(), torch.full((2,), -1, dtype=torch.int64, device="cuda")])
    estp.tree_attention(Q, dev(c.K), dev(c.V), *c.args(), tree_mask=mask, O=O, lse=lse, acc=acc)
    c.check(O[:6], lse[:, :6], acc)
    assert (O[6:] == 7).all() and (lse[:, 6:] == 7).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_loose_bounds_change_nothing_but_roundings(dtype):
    # a serving program states the capacity, not each step's longest sequence
    c = Case(7, [200, 900], [1, 3], 8, 2, 128, dtype, cap=4000)
    acc = dev(c.acc)
    O, lse = estp.tree_attention(dev(c.Q), dev(c.K), dev(c.V), dev(c.lens), dev(c.cu), 4, 4000, tree_mask=c.mask(),
                                 acc=acc)
    c.check(O, lse, acc)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_counts_out_of_range_stay_in_bounds(dtype):
    # invalid lengths give no defined result, but read and write nothing outside their tensors
    c = Case(8, [50, 40, 60], [2, 3, 1], 4, 2, 32, dtype, cap=64)
    acc = torch.cat([dev(c.acc).view(-1), torch.full((1000,), 3.0, device="cuda")])
    lens = torch.tensor([-5, 2 ** 31 - 1, 60], dtype=torch.int32, device="cuda")
    cu = torch.tensor([0, 2, 1 << 20, 6], dtype=torch.int32, device="cuda")
    estp.tree_attention(dev(c.Q), dev(c.K), dev(c.V), lens, cu, 3, 64, tree_mask=c.mask(), acc=acc[:c.acc.size])
    torch.cuda.synchronize()
    assert (acc[c.acc.size:] == 3).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_offsets_far_below_zero_stay_in_bounds(dtype):
    c = Case(8, [50, 40, 60], [2, 3, 1], 4, 2, 32, dtype, cap=64)
    acc = torch.cat([dev(c.acc).view(-1), torch.full((1000,), 3.0, device="cuda")])
    cu = torch.tensor([0, 6, -(1 << 31), 6], dtype=torch.int32, device="cuda")
    estp.tree_attention(dev(c.Q), dev(c.K), dev(c.V), dev(c.lens), cu, 3, 64, tree_mask=c.mask(), acc=acc[:c.acc.size])
    torch.cuda.synchronize()
    assert (acc[c.acc.size:] == 3).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tree", [True, False])
def test_many_sequences_of_any_length(dtype, tree):
    # more sequences than lanes, some without rows, some with several items of rows, few chunks and many
    g = np.random.default_rng(20)
    lens = g.integers(0, 120, 150)
    T = g.integers(0, 4, 150)
    lens[[3, 70, 140]], T[[3, 70, 140]] = [2500, 900, 1700], [40, 0, 17]
    T[60:68] = 0
    c = Case(21, lens.tolist(), T.tolist(), 8, 2, 32, dtype, tree)
    acc = dev(c.acc)
    O, lse = c.attend(acc=acc)
    c.check(O, lse, acc)


@pytest.mark.parametrize("dtype,dh", [("bf16", 64), ("bf16", 128), ("f32", 64)])
def test_a_long_tree_of_many_heads(dtype, dh):
    # 64 tokens of 16 heads on one KV head: many items that share the keys, rows in several batches of the account
    c = Case(22, [3000, 9], [64, 50], 16, 1, dh, dtype)
    acc = dev(c.acc)
    O, lse = c.attend(acc=acc)
    c.check(O, lse, acc)


def test_two_captured_graphs_on_one_workspace():
    cs = [Case(23, [300, 40], [3, 9], 8, 2, 64, "bf16"), Case(24, [900], [1], 8, 2, 64, "bf16")]
    lib = estp.load()
    need = max(lib.estp_tree_attention_workspace_size(len(c.lens), c.max_q, len(c.Q), 8, 2, c.max_kv, 64, 0) for c in cs)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    graphs = []
    for c in cs:
        t = [dev(a) for a in (c.Q, c.K, c.V, c.lens, c.cu)]
        out = {"O": torch.empty_like(t[0]), "lse": torch.empty(8, len(c.Q), device="cuda"), "acc": dev(c.acc)}
        mask = c.mask()
        call = lambda: estp.tree_attention(*t, c.max_q, c.max_kv, tree_mask=mask, workspace=ws, **out)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            call()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            call()
        graphs.append((graph, c, out, t, mask))
    for rep in range(3):
        for graph, c, out, t, mask in graphs:
            out["acc"].copy_(dev(c.acc))
            out["O"].fill_(float("nan"))
            graph.replay()
        torch.cuda.synchronize()
        for graph, c, out, t, mask in graphs:
            c.check(out["O"], out["lse"], out["acc"])


def test_two_calls_at_once():
    # two streams, a workspace each: neither call disturbs the other
    cs = [Case(25, [4000, 40], [3, 9], 8, 2, 128, "bf16"), Case(26, [6000], [20], 8, 2, 128, "bf16")]
    want = [c.attend() for c in cs]
    torch.cuda.synchronize()
    args = [([dev(a) for a in (c.Q, c.K, c.V, c.lens, c.cu)], c.mask()) for c in cs]
    streams = [torch.cuda.Stream() for _ in cs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, c in enumerate(cs):
            with torch.cuda.stream(streams[i]):
                got[i].append(estp.tree_attention(*args[i][0], c.max_q, c.max_kv, tree_mask=args[i][1]))
    torch.cuda.synchronize()
    for i in range(2):
        for O, lse in got[i]:
            assert torch.equal(O, want[i][0]) and torch.equal(lse, want[i][1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_long_cache(dtype):
    n = 131_072
    c = Case(9, [n], [2], 4, 1, 128, dtype)
    acc = dev(c.acc)
    O, lse = c.attend(acc=acc)
    c.check(O, lse, acc)


def test_cache_past_32_bit_offsets():
    # K and V of 2.2e9 elements each; the sequences' own lengths are short
    B, Hkv, cap, dh = 2, 8, 1_075_000, 128
    c = Case(10, [300, 411], [3, 5], 16, Hkv, dh, "bf16", cap=500)
    K, V = (torch.zeros(B, Hkv, cap, dh, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    acc = torch.zeros(B, Hkv, cap, device="cuda")
    K[:, :, :500], V[:, :, :500], acc[:, :, :500] = dev(c.K), dev(c.V), dev(c.acc)
    O, lse = estp.tree_attention(dev(c.Q), K, V, *c.args(), tree_mask=c.mask(), acc=acc)
    c.check(O, lse, acc[:, :, :500].contiguous())
    assert not acc[:, :, 500:].any()
    # and a sequence at the very end of a long one
    lens = torch.tensor([0, cap - 5], dtype=torch.int32, device="cuda")
    K.zero_()
    V[1] = 1.0
    O, lse = estp.tree_attention(dev(c.Q), K, V, lens, dev(c.cu), 5, cap, tree_mask=c.mask(), acc=acc)
    torch.testing.assert_close(O[3:].float(), torch.ones_like(O[3:]).float(), rtol=0.01, atol=0)
    want = np.log(cap - 5 + np.array([bin(m).count("1") for m in c.masks[3:]]))
    np.testing.assert_allclose(host(lse[:, 3:]), np.broadcast_to(want, (16, 5)), rtol=1e-5)


def test_repeats_streams_and_stale_workspaces():
    c = Case(11, [900, 3000, 10], [1, 9, 4], 32, 8, 128, "bf16")
    acc = dev(c.acc)
    first = *c.attend(acc=acc), acc
    ws = torch.full((estp.load().estp_tree_attention_workspace_size(3, 9, 14, 32, 8, c.max_kv, 128, 0),), 255,
                    dtype=torch.uint8, device="cuda")  # NaN in all of it
    acc2 = dev(c.acc)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = *c.attend(acc=acc2, workspace=ws, stream=side), acc2
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(first, again):
        assert torch.equal(a, b)


def test_replayed_in_a_graph_as_the_cache_grows():
    c = Case(12, [200, 64, 1], [1, 1, 1], 8, 2, 64, "bf16", tree=False, cap=330)
    Q, K, V, lens, cu, acc = dev(c.Q), dev(c.K), dev(c.V), dev(c.lens), dev(c.cu), dev(c.acc)
    ws = torch.empty(estp.load().estp_tree_attention_workspace_size(3, 1, 3, 8, 2, 330, 64, 0), dtype=torch.uint8,
                     device="cuda")
    O, lse = torch.empty_like(Q), torch.empty(8, 3, device="cuda")

    def step():
        estp.tree_attention(Q, K, V, lens, cu, 1, 330, O=O, lse=lse, acc=acc, workspace=ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for rep in range(4):
        c.lens = c.lens + 30
        lens.copy_(dev(c.lens))
        acc.copy_(dev(c.acc))
        O.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        c.check(O, lse, acc)


def test_binding_refuses_mis_sized_tensors():
    z = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    i32 = torch.int32
    Q, C, lens, cu, acc = z(3, 4, 64), z(2, 2, 50, 64), z(2, dtype=i32), z(3, dtype=i32), z(2, 2, 50)
    bad = [({"lens": z(3, dtype=i32)}, "lens must hold 2"), ({"cu": z(2, dtype=i32)}, "cu_q must hold 3"),
           ({"V": z(2, 2, 49, 64)}, "V must"), ({"K": z(2, 2, 50, 32)}, "head size"),
           ({"tree_mask": z(3, dtype=i32)}, "tree_mask must be"), ({"acc": z(2, 2, 49)}, "acc must hold 200"),
           ({"O": z(3, 4, 32)}, "O must hold"), ({"lse": z(4, 2)}, "lse must hold 12")]
    for kw, match in bad:
        a = {"K": C, "V": C.clone(), "lens": lens, "cu": cu, **kw}
        with pytest.raises((ValueError, TypeError), match=match):
            estp.tree_attention(Q, a.pop("K"), a.pop("V"), a.pop("lens"), a.pop("cu"), 2, 50, **a)
    with pytest.raises(ValueError, match="row_weight must hold 3"):
        estp.tree_importance(Q, C, z(4, 3), lens, cu, 2, 50, acc, row_weight=z(2))
    with pytest.raises(estp.EstpError, match="max_kv"):
        estp.tree_attention(Q, C, C.clone(), lens, cu, 2, 51)
    with pytest.raises(ValueError, match="K must be contiguous"):
        estp.tree_attention(Q, C.transpose(1, 2), C, lens, cu, 2, 50)

"""Eviction from a cache on the GPU: exact against the oracle, and a run of the calls as they are used together."""
import numpy as np
import pytest
import torch

import oracle
import paper_2608_15592_amd as estp
from oracle import operators as OP
from synth import inputs as I
from tests._util import dev, host

pytestmark = pytest.mark.gpu


def _case(seed, lens, Hkv, dh, cap, dtype, values="heavy"):
    g = np.random.default_rng(seed)
    B = len(lens)
    K, V = (g.standard_normal((B, Hkv, cap, dh)).astype(np.float32) for _ in range(2))
    if dtype == "bf16":
        K, V = I.f32_to_bf16_bits(K), I.f32_to_bf16_bits(V)
    acc = np.exp(1.5 * g.standard_normal((B, Hkv, cap))).astype(np.float32)
    if values == "ties":
        acc = g.integers(0, 4, acc.shape).astype(np.float32)
    elif values == "equal":
        acc[:] = 1.0
    elif values == "odd":  # negative, zeros of both signs, infinities, NaN
        acc = g.standard_normal(acc.shape).astype(np.float32)
        for x in (0.0, -0.0, np.inf, -np.inf, np.nan, -np.nan, 1e-42, -1e-42):
            acc[g.uniform(size=acc.shape) < 0.06] = x
    pos = np.stack([[g.permutation(cap) for _ in range(Hkv)] for _ in range(B)]).astype(np.int32)
    return K, V, acc, pos, np.array(lens, np.int32), (np.array(lens) + g.integers(0, 9, B)).astype(np.int32)


def _check(K, V, acc, pos, lens, seen, keep, recent, sink, in_place):
    idx, new = OP.cache_evict(acc, pos, lens, seen, keep, recent, sink)
    Kd, Vd, ad, pd, ld = dev(K), dev(V), dev(acc), dev(pos), dev(lens)
    out = {} if in_place else {"acc_out": torch.full_like(ad, 5.0), "pos_out": torch.full_like(pd, 5)}
    got_lens, got_idx = estp.cache_evict(Kd, Vd, ad, pd, ld, dev(seen), keep, recent, sink,
                                         lens_out=ld if in_place else None, **out)
    np.testing.assert_array_equal(host(got_idx), idx)
    np.testing.assert_array_equal(host(got_lens), new)
    for got, was, fill in ((out.get("acc_out", ad), acc, 0.0), (out.get("pos_out", pd), pos, -1)):
        want = OP.evicted(was, idx, lens, fill)
        if not in_place:  # slots past the sequences
            for b, n in enumerate(lens):
                want[b, :, n:] = 5
            assert torch.equal(ad.view(torch.int32), dev(acc).view(torch.int32)) and torch.equal(pd, dev(pos))
        np.testing.assert_array_equal(host(got).view(np.int32), want.view(np.int32))
    for got, was in ((Kd, K), (Vd, V)):
        want = np.array(was)
        for b in range(K.shape[0]):
            for h in range(K.shape[1]):
                m = idx[b, h][idx[b, h] >= 0]
                want[b, h, :len(m)] = was[b, h, m]
        assert torch.equal(got, dev(want))  # rows past the kept ones too: they stay as they were


CASES = [
    # lens, Hkv, dh, cap, keep, recent, sink
    ([1], 1, 32, 1, 1, 0, 0),
    ([2], 1, 64, 2, 1, 1, 0),
    ([0, 5, 9], 2, 32, 12, 5, 2, 1),
    ([64, 65, 63], 3, 64, 70, 64, 10, 4),
    ([1000, 1024, 1025], 2, 128, 1030, 1024, 32, 4),
    ([700, 3000, 4097], 2, 64, 4100, 1024, 64, 4),
    ([5000, 40], 1, 128, 5000, 4999, 0, 0),
    ([9000], 2, 32, 9001, 17, 9, 8),
    ([300] * 20, 8, 32, 300, 299, 299, 0),
    ([70000], 1, 32, 70001, 33000, 100, 4),
]


@pytest.mark.parametrize("lens,Hkv,dh,cap,keep,recent,sink", CASES)
@pytest.mark.parametrize("values", ["heavy", "ties", "odd", "equal"])
@pytest.mark.parametrize("in_place", [True, False])
def test_eviction_is_exact(lens, Hkv, dh, cap, keep, recent, sink, values, in_place):
    dtype = "bf16" if values in ("heavy", "odd") else "f32"
    _check(*_case(len(lens) + cap, lens, Hkv, dh, cap, dtype, values), keep, recent, sink, in_place)


LONG = [
    # lens, Hkv, dh, cap, keep, recent, sink: about where slots no longer stay in registers, and past it
    ([16384, 16385, 9000], 2, 64, 16385, 16384, 64, 4),
    ([20000, 100, 0, 16385, 17000], 2, 32, 20000, 17000, 64, 4),
    ([17000, 16000], 1, 32, 17000, 17000, 64, 4),
    ([16000, 16384, 4096, 4097], 1, 32, 16384, 4096, 64, 4),
    ([20000, 5000, 32768], 2, 32, 32768, 5000, 64, 4),
    ([32769, 65536, 40000], 2, 32, 65536, 32768, 64, 4),
    ([65000], 1, 32, 65001, 64000, 3000, 4),
    ([65536, 65537, 131000], 1, 32, 131073, 100, 64, 4),
]


@pytest.mark.parametrize("lens,Hkv,dh,cap,keep,recent,sink", LONG)
@pytest.mark.parametrize("values", ["heavy", "ties", "odd"])
def test_eviction_from_long_caches(lens, Hkv, dh, cap, keep, recent, sink, values):
    _check(*_case(len(lens) + cap, lens, Hkv, dh, cap, "bf16", values), keep, recent, sink, values != "ties")


def test_long_caches_of_many_groups():
    # few segments a group
    g = np.random.default_rng(9)
    lens = np.concatenate([[16400, 0, 3000], g.integers(2500, 16401, 17)])
    _check(*_case(9, lens.tolist(), 8, 32, 16400, "bf16"), 3000, 64, 4, True)


@pytest.mark.parametrize("values", ["heavy", "ties", "equal"])
def test_more_guarded_slots_than_kept_in_a_long_cache(values):
    K, V, acc, pos, lens, seen = _case(12, [30000, 20000], 2, 32, 30000, "bf16", values)
    pos[:] = np.where(np.arange(30000) % 2, 0, pos)
    _check(K, V, acc, pos, lens, seen, 9000, 10, 5, False)


def test_long_cache_replayed_in_a_graph_on_a_stale_workspace():
    K, V, acc, pos, lens, seen = _case(13, [40000, 500], 2, 32, 40000, "bf16")
    t = [dev(a) for a in (K, V, acc, pos, lens, seen)]
    need = estp.load().estp_cache_evict_workspace_size(2, 2, 40000, 1000)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    idx = torch.empty(2, 2, 1000, dtype=torch.int32, device="cuda")
    call = lambda: estp.cache_evict(*t, 1000, 64, 4, lens_out=t[4], idx=idx, workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    want, new = OP.cache_evict(acc, pos, lens, seen, 1000, 64, 4)
    for rep in range(3):
        for a, b in zip(t, (K, V, acc, pos, lens, seen)):
            a.copy_(dev(b))
        ws.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        np.testing.assert_array_equal(host(idx), want)
        np.testing.assert_array_equal(host(t[4]), new)
        moved = OP.evicted(acc, want, lens, 0.0)
        np.testing.assert_array_equal(host(t[2]).view(np.int32), moved.view(np.int32))


def test_more_guarded_slots_than_kept():
    # positions that repeat guard more slots than the budget: the best of them stay
    K, V, acc, pos, lens, seen = _case(2, [500, 30], 2, 64, 500, "bf16", "ties")
    pos[:] = np.where(np.arange(500) % 2, 0, pos)
    _check(K, V, acc, pos, lens, seen, 100, 10, 5, True)


def test_cache_past_32_bit_offsets():
    B, Hkv, cap, dh = 2, 8, 1_075_000, 128
    K, V, acc, pos, lens, seen = _case(3, [600, 800], Hkv, dh, 800, "bf16")
    big = [torch.zeros(B, Hkv, cap, dh, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for t, a in zip(big, (K, V)):
        t[:, :, :800] = dev(a)
    ad, pd = torch.zeros(B, Hkv, cap, device="cuda"), torch.zeros(B, Hkv, cap, dtype=torch.int32, device="cuda")
    ad[:, :, :800], pd[:, :, :800] = dev(acc), dev(pos)
    got_lens, got = estp.cache_evict(*big, ad, pd, dev(lens), dev(seen), 400, 20, 4)
    idx, new = OP.cache_evict(acc, pos, lens, seen, 400, 20, 4)
    np.testing.assert_array_equal(host(got), idx)
    at = torch.from_numpy(idx).cuda()[..., None].expand(-1, -1, -1, dh)
    for t, a in zip(big, (K, V)):
        assert torch.equal(t[:, :, :400], dev(a).gather(2, at)) and not t[:, :, 800:].any()
    # all of a long sequence: the last 5 of its positions and the first 3 are what is left
    full = torch.full((B,), cap, dtype=torch.int32, device="cuda")
    pd.copy_(torch.arange(cap, dtype=torch.int32, device="cuda").expand_as(pd))
    big[1][:, :, cap - 5:] = torch.arange(5, device="cuda")[:, None].bfloat16()
    ad.zero_()
    got_lens, got = estp.cache_evict(*big, ad, pd, full, full, 8, 5, 3)
    assert got_lens.tolist() == [8, 8]
    want = torch.tensor([0, 1, 2] + list(range(cap - 5, cap)), device="cuda")
    assert torch.equal(got.long(), want.expand_as(got)) and torch.equal(pd[:, :, :8].long(), want.expand_as(got))
    assert torch.equal(big[1][:, :, 3:8].float(), torch.arange(5.0, device="cuda")[:, None].expand(B, Hkv, 5, dh))


def test_counts_out_of_range_stay_in_bounds():
    K, V, acc, pos, lens, seen = _case(4, [50, 50], 2, 32, 64, "bf16")
    lens[:] = [-7, 2 ** 31 - 1]
    guard = torch.full((512,), 9.0, device="cuda")
    ad = torch.cat([dev(acc).view(-1), guard])
    got, idx = estp.cache_evict(dev(K), dev(V), ad[:acc.size], dev(pos), dev(lens), dev(seen), 20, 4, 2)
    assert got.tolist() == [0, 20] and (idx[0] == -1).all() and (ad[acc.size:] == 9).all()
    assert int(idx.max()) < 64


def test_repeats_and_streams():
    K, V, acc, pos, lens, seen = _case(5, [3000, 100, 2500], 8, 128, 3000, "bf16", "ties")
    need = estp.load().estp_cache_evict_workspace_size(3, 8, 3000, 1000)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    outs = []
    side = torch.cuda.Stream()
    for kw in ({}, {"workspace": ws, "stream": side}):
        t = [dev(a) for a in (K, V, acc, pos)]
        side.wait_stream(torch.cuda.current_stream())
        outs.append([*t, *estp.cache_evict(*t, dev(lens), dev(seen), 1000, 64, 4, **kw)])
        torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(*outs):
        assert torch.equal(a, b)


def test_replayed_in_a_graph():
    K, V, acc, pos, lens, seen = _case(6, [300, 50], 2, 64, 300, "bf16")
    Kd, Vd, ad, pd, ld, sd = (dev(a) for a in (K, V, acc, pos, lens, seen))
    ws = torch.empty(estp.load().estp_cache_evict_workspace_size(2, 2, 300, 100), dtype=torch.uint8, device="cuda")
    idx = torch.empty(2, 2, 100, dtype=torch.int32, device="cuda")

    def step():
        estp.cache_evict(Kd, Vd, ad, pd, ld, sd, 100, 8, 2, lens_out=ld, idx=idx, workspace=ws)

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
        acc = np.roll(acc, 17, axis=2)
        for t, a in ((Kd, K), (Vd, V), (ad, acc), (pd, pos), (ld, lens)):
            t.copy_(dev(a))
        idx.fill_(-9)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want, new = OP.cache_evict(acc, pos, lens, seen, 100, 8, 2)
        np.testing.assert_array_equal(host(idx), want)
        np.testing.assert_array_equal(host(ld), new)
        np.testing.assert_array_equal(host(ad), OP.evicted(acc, want, lens, 0.0))


def test_binding_refuses_mis_sized_tensors():
    z = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype, device="cuda")  # noqa: E731
    i32 = torch.int32
    ok = dict(K=z(2, 2, 50, 64), V=z(2, 2, 50, 64), acc=z(2, 2, 50), pos=z(2, 2, 50, dtype=i32), lens=z(2, dtype=i32),
              seen=z(2, dtype=i32), keep=10)
    bad = [({"V": z(2, 2, 49, 64)}, "V must"), ({"acc": z(2, 2, 49)}, "acc must hold 200"),
           ({"pos": z(2, 2, 50)}, "pos must be"), ({"lens": z(3, dtype=i32)}, "lens must hold 2"),
           ({"seen": z(1, dtype=i32)}, "seen must hold 2"), ({"idx": z(2, 2, 9, dtype=i32)}, "idx must hold 40"),
           ({"acc_out": z(3)}, "acc_out must hold"), ({"lens_out": z(3, dtype=i32)}, "lens_out must hold 2")]
    for kw, match in bad:
        with pytest.raises((ValueError, TypeError), match=match):
            estp.cache_evict(**{**ok, **kw})
    for kw in ({"keep": 0}, {"keep": 51}, {"recent": 11}, {"sink": -1}, {"V": ok["K"]}):
        with pytest.raises(estp.EstpError):
            estp.cache_evict(**{**ok, **kw})


def test_a_serving_run():
    """Prefill importance starts the account, the cache is cut to a budget, drafted trees are attended and scored
    by the LM head, the accepted rows are credited, and the cache is cut again: every step against the oracle on
    the state the GPU has reached."""
    g = np.random.default_rng(7)
    B, Hq, Hkv, dh, d, V, cap, keep = 2, 8, 2, 64, 128, 900, 400, 150
    lens = np.array([330, 140], np.int32)
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    bf = lambda *s: I.f32_to_bf16_bits(g.standard_normal(s).astype(np.float32))  # noqa: E731
    q, k, v = bf(cu[-1], Hq, dh), bf(cu[-1], Hkv, dh), bf(cu[-1], Hkv, dh)
    S = estp.attn_importance(dev(q), dev(k), dev(cu), int(lens.max()))
    K, Vc = (torch.zeros(B, Hkv, cap, dh, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    acc, pos = torch.zeros(B, Hkv, cap, device="cuda"), torch.full((B, Hkv, cap), -1, dtype=torch.int32, device="cuda")
    for b in range(B):
        n, at = int(lens[b]), slice(int(cu[b]), int(cu[b + 1]))
        K[b, :, :n], Vc[b, :, :n] = dev(k[at]).transpose(0, 1), dev(v[at]).transpose(0, 1)
        acc[b, :, :n] = S[at] * n * (Hq // Hkv)
        pos[b, :, :n] = torch.arange(n, dtype=torch.int32, device="cuda")
    ld, seen = dev(lens), dev(lens)
    W = I.f32_to_bf16_bits((0.1 * g.standard_normal((V, d))).astype(np.float32))
    for step in range(3):
        before = [host(t) for t in (acc, pos, ld, seen)]
        _, idx = estp.cache_evict(K, Vc, acc, pos, ld, seen, keep, 32, 4, lens_out=ld)
        want, new = OP.cache_evict(*before, keep, 32, 4)
        np.testing.assert_array_equal(host(idx), want)
        np.testing.assert_array_equal(host(ld), new)
        np.testing.assert_array_equal(host(acc), OP.evicted(before[0], want, before[2], 0.0))
        # three drafted tokens after each sequence: 0, and 1 and 2 below it
        T, masks = 3, [0b1, 0b11, 0b101] * B
        Q = bf(B * T, Hq, dh)
        for b in range(B):
            n = int(new[b])
            K[b, :, n:n + T], Vc[b, :, n:n + T] = dev(bf(Hkv, T, dh)), dev(bf(Hkv, T, dh))
        cq = dev(np.arange(0, B * T + 1, T, dtype=np.int32))
        mask = torch.tensor(masks, device="cuda")
        O, lse = estp.tree_attention(dev(Q), K, Vc, ld, cq, T, cap, tree_mask=mask)
        cache = [host(t.view(torch.int16)).view(np.uint16) for t in (K, Vc)]
        ref = OP.tree_attention(Q, *cache, new, host(cq), masks, dtype="bf16")
        assert (np.abs(host(O.float()) - ref["O"]) <= ref["O_bound"]).all()
        # the LM head scores the drafted tokens; 0 and 2 are accepted
        X = O.reshape(B * T, Hq * dh)[:, :d].contiguous()
        tok = g.integers(0, V, B * T).astype(np.int32)
        mode = torch.empty(B * T, dtype=torch.int32, device="cuda")
        loss, head_lse = estp.token_loss(X, dev(W), dev(tok), vocab_argmax=mode)
        Xb = host(X.view(torch.int16)).view(np.uint16)
        ref_loss, ref_lse = OP.token_loss(Xb, W, tok)
        assert (np.abs(host(loss) - ref_loss) <= 2 * OP.lse_bound(Xb, W, ref_lse) + OP.logit_bound(Xb, W)).all()
        taken = np.array([1, 0, 1] * B, np.float32)
        was = host(acc).astype(np.float64)
        estp.tree_importance(dev(Q), K, lse, ld, cq, T, cap, acc, tree_mask=mask, row_weight=dev(taken))
        ref = OP.tree_attention(Q, *cache, new, host(cq), masks, dtype="bf16", row_weight=taken)
        assert (np.abs(host(acc) - was - ref["got"]) <= ref["got_bound"] + 2 * OP.U * (was + ref["got"])).all()
        # the accepted tokens take the slots after the cached ones: token 2 moves into token 1's
        for b in range(B):
            n = int(new[b])
            for t in (K, Vc, acc):
                t[b, :, n + 1] = t[b, :, n + 2].clone()
            acc[b, :, n + 2] = 0.0
            pos[b, :, n:n + 2] = seen[b] + torch.arange(2, dtype=torch.int32, device="cuda")
        ld += 2
        seen += 2
        assert oracle.widen(Xb).shape == (B * T, d)

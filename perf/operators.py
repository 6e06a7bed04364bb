"""The operators that serving and training programs call beside the scoring path, as measurable cases.

* ``loss``   - the LM-head loss of given next tokens (``token_loss``): drafted tokens to verify, log-probabilities of
  an RL batch
* ``train``  - the same with its gradients (``token_loss`` and ``token_loss_backward``)
* ``attend`` - attention of newly drafted tokens (one, a chain, a tree) over a cache, adding the weight every cached
  token receives to its account (``tree_attention``)
* ``credit`` - that account for the drafted rows that were accepted, from the rows' normalisers (``tree_importance``)
* ``evict``  - the cache cut to its most attended slots (``cache_evict``)

Where ``own`` is false, ``run`` computes them in elementary torch operations in 32 bits; where it is true, through the
library.  The model shapes are those of the scoring path's workloads.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

# hidden size, vocabulary, query heads, KV heads, head size
MODELS = {
    "llama-8b": (4096, 128256, 32, 8, 128),
    "llama-1b": (2048, 128256, 32, 8, 64),
    "qwen-1.5b": (1536, 151936, 12, 2, 128),
    "tiny": (64, 1000, 2, 2, 32),
}


def listed():
    return [
        # the 61 drafted tokens of a small batch, scored for acceptance
        {"name": "loss_drafts", "kind": "loss", "model": "llama-8b", "dtype": "bf16", "n_tok": 61, "ignored": 0.0},
        # log-probabilities of a 16 x 512-token sampling batch
        {"name": "loss_qwen", "kind": "loss", "model": "qwen-1.5b", "dtype": "bf16", "n_tok": 8192, "ignored": 0.0},
        # the smallest fp32 configuration: launches are all there is
        {"name": "train_tiny_f32", "kind": "train", "model": "tiny", "dtype": "f32", "n_tok": 128, "ignored": 0.0},
        # one ragged micro-batch of supervised tuning, a third of its tokens prompt (no loss there)
        {"name": "train_micro", "kind": "train", "model": "llama-1b", "dtype": "bf16", "n_tok": 1021, "ignored": 0.33},
        # a full training batch: the largest call
        {"name": "train_llama", "kind": "train", "model": "llama-8b", "dtype": "bf16", "n_tok": 4096, "ignored": 0.0},
        # one token of one long context
        {"name": "attend_long", "kind": "attend", "model": "llama-8b", "dtype": "bf16", "B": 1, "T": 1, "lo": 32767,
         "hi": 32767, "tree": False},
        # one token of each of 32 running requests
        {"name": "attend_batch", "kind": "attend", "model": "llama-8b", "dtype": "bf16", "B": 32, "T": 1, "lo": 500,
         "hi": 4000, "tree": False},
        # trees of 31 drafted tokens in 8 requests
        {"name": "attend_tree", "kind": "attend", "model": "llama-1b", "dtype": "bf16", "B": 8, "T": 31, "lo": 900,
         "hi": 8100, "tree": True},
        # five drafted tokens of a lone short request: the smallest call of the serving side
        {"name": "credit_chain", "kind": "credit", "model": "qwen-1.5b", "dtype": "bf16", "B": 1, "T": 5, "lo": 700,
         "hi": 700, "tree": False},
        # the accepted paths of a batch of trees
        {"name": "credit_tree", "kind": "credit", "model": "llama-8b", "dtype": "bf16", "B": 16, "T": 23, "lo": 700,
         "hi": 6000, "tree": True},
        # a step that has run a few slots over its budget
        {"name": "evict_step", "kind": "evict", "model": "qwen-1.5b", "dtype": "bf16", "B": 3, "lo": 1029, "hi": 1029,
         "keep": 1024, "recent": 32, "sink": 4},
        # prompts of mixed length cut to a quarter of the longest after their prefill
        {"name": "evict_prefill", "kind": "evict", "model": "llama-8b", "dtype": "bf16", "B": 32, "lo": 700,
         "hi": 4096, "keep": 1024, "recent": 64, "sink": 4},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["loss", "train", "train", "attend", "attend", "credit", "evict", "evict"])
    model = rng.choice(["llama-8b", "llama-1b", "qwen-1.5b"])
    f32 = rng.random() < 0.25
    case = {"kind": kind, "model": model, "dtype": "f32" if f32 else "bf16"}
    if kind in ("loss", "train"):
        if f32:
            case["model"] = rng.choice(["tiny", "llama-1b", "qwen-1.5b"])
        most = 400 if f32 else 8000 if kind == "loss" else 4000
        case.update(n_tok=_log_int(rng, 1, most), ignored=rng.choice([0.0, 0.2, 0.5]))
        return case
    Hkv, dh = MODELS[model][3:]
    room = 120_000_000 // (Hkv * dh)  # cached tokens of a whole batch
    a, b = sorted((_log_int(rng, 33, 60000), _log_int(rng, 33, 60000)))
    lo, hi = rng.choice([(a, b), (b, b)])
    B = min(_log_int(rng, 1, 48), max(1, room // hi))
    case.update(B=B, lo=lo, hi=hi)
    if kind == "evict":
        keep = max(8, int(hi * rng.uniform(0.1, 0.99)))
        case.update(keep=keep, recent=rng.randint(0, keep // 4), sink=rng.choice([0, 4]))
        return case
    T = _log_int(rng, 1, 64)
    case.update(T=T, tree=T > 2 and rng.random() < 0.6)
    # the scores of the plain form, and of the 64-bit one, stay within memory
    while case["B"] > 1 and case["B"] * T * MODELS[model][2] * hi > 1_200_000_000:
        case["B"] //= 2
    return case


# ----------------------------------------------------------------------------- inputs


def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _lengths(case):
    """Lengths spread evenly in the logarithm over [lo, hi], in a fixed shuffled order; the longest is hi."""
    B, lo, hi = case["B"], case["lo"], case["hi"]
    n = np.rint(lo * (hi / lo) ** ((np.arange(B) + 1.0) / B)).astype(np.int64)
    return np.random.default_rng(B).permutation(n)


def _rows(case):
    """Drafted tokens of each sequence: T, or in a batch between T / 2 and T."""
    B, T = case["B"], case["T"]
    return T - np.arange(B) % (T // 2 + 1)


def _tree(case, rows, seed):
    """Ancestor masks [n_q] (bit j: drafted token j is an ancestor or the row itself) and, per row, whether it lies on
    the accepted path (the ancestors of one row of each sequence)."""
    g = np.random.default_rng(seed)
    masks, taken = [], []
    for T in rows.tolist():
        m = []
        for t in range(T):
            parent = t - 1 if not case["tree"] else int(g.integers(max(-1, t - 6), t)) if t else -1
            m.append((m[parent] if parent >= 0 else 0) | 1 << t)
        path = m[int(g.integers(T // 2, T))]
        masks += [x - (1 << 64) if x >> 63 else x for x in m]
        taken += [path >> t & 1 for t in range(T)]
    return torch.tensor(masks, dtype=torch.int64).cuda(), torch.tensor(taken, dtype=torch.float32).cuda()


def _normal(g, shape, dtype, scale=1.0):
    return (scale * torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)).to(dtype)


def _cache(g, case, cap):
    Hkv, dh = MODELS[case["model"]][3:]
    return [torch.stack([_normal(g, (Hkv, cap, dh), _dtype(case)) for _ in range(case["B"])]) for _ in range(2)]


def _account(g, case, cap, lens):
    """Accumulated weights with a heavy tail; slots that never received any among them; 0 past the sequence."""
    acc = torch.exp(1.5 * torch.randn(case["B"], MODELS[case["model"]][3], cap, generator=g, device="cuda"))
    acc *= torch.rand(acc.shape, generator=g, device="cuda") > 0.03
    return acc * (torch.arange(cap, device="cuda") < lens[:, None, None])


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    d, V, Hq, Hkv, dh = MODELS[case["model"]]
    st = {"case": case}
    if case["kind"] in ("loss", "train"):
        n, dt = case["n_tok"], _dtype(case)
        st["W"] = _normal(g, (V, d), dt, 0.02)
        # hidden states of RMS 1 that lean towards their token by up to 12 nats, as a trained model's do
        t = torch.randint(V, (n,), generator=g, device="cuda")
        x = torch.randn(n, d, generator=g, device="cuda")
        x *= torch.rsqrt(x.square().mean(dim=1, keepdim=True))
        x += 12.0 * torch.rand(n, 1, generator=g, device="cuda") * st["W"][t].float() / (0.0004 * d)
        st["X"] = x.to(dt)
        if case["ignored"]:
            t[torch.rand(n, generator=g, device="cuda") < case["ignored"]] = -100
        st["targets"] = t.to(torch.int32)
        # the weight of each token's loss: a mean over the batch with advantages
        st["grad"] = (0.5 + torch.rand(n, generator=g, device="cuda")) / n
        return st
    lens = torch.from_numpy(_lengths(case).astype(np.int32)).cuda()
    st["lens"] = lens
    if case["kind"] == "evict":
        cap = case["hi"]
        st["K"], st["V"] = _cache(g, case, cap)
        st["acc"] = _account(g, case, cap, lens)
        # slots hold ascending positions, except where an earlier eviction has filled holes with later tokens
        pos = torch.arange(cap, dtype=torch.int32, device="cuda").repeat(case["B"], Hkv, 1)
        st["seen"] = lens + case["hi"] // 3
        gap = torch.arange(cap, device="cuda") >= case["keep"] // 2
        st["pos"] = torch.where(gap, pos + (st["seen"] - lens)[:, None, None], pos)
        st["acc_out"], st["pos_out"] = torch.zeros_like(st["acc"]), torch.zeros_like(st["pos"])
        return st
    rows = _rows(case)
    cap = case["hi"] + case["T"]
    st["K"], st["V"] = _cache(g, case, cap)
    cu = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    st["cu"] = torch.from_numpy(cu).cuda()
    sharp = 0.5 + 1.5 * torch.rand(Hq, 1, generator=g, device="cuda")
    st["Q"] = (sharp * torch.randn(int(cu[-1]), Hq, dh, generator=g, device="cuda")).to(_dtype(case))
    st["mask"], taken = _tree(case, rows, seed)
    st["max_kv"] = cap
    st["acc"] = _account(g, case, cap, lens)
    if case["kind"] == "credit":
        st["taken"] = taken
        st["lse"] = _attention64(st)[1].float()
    return st


# ----------------------------------------------------------------------------- plain forms


def _loss_plain(st):
    z = st["X"].float() @ st["W"].float().t()
    m = z.amax(dim=1, keepdim=True)
    lse = m[:, 0] + torch.log(torch.exp(z - m).sum(dim=1))
    live = st["targets"] >= 0
    t = torch.where(live, st["targets"], 0).long()
    loss = torch.where(live, lse - z.gather(1, t[:, None])[:, 0], 0.0)
    return z, lse, loss, live, t


def _train_plain(st):
    z, lse, loss, live, t = _loss_plain(st)
    p = torch.exp(z - lse[:, None])
    p.scatter_add_(1, t[:, None], torch.full_like(lse, -1.0)[:, None])
    p *= (st["grad"] * live)[:, None]
    dX = (p @ st["W"].float()).to(st["X"].dtype)
    dW = (p.t() @ st["X"].float()).to(st["W"].dtype)
    return {"loss": loss, "lse": lse, "dX": dX, "dW": dW}


def _padded(st):
    """Where each drafted row stands: its sequence, its place there, and the keys it sees [B, T, keys]."""
    T, lens = st["case"]["T"], st["lens"].long()
    cu = st["cu"].long()
    i = torch.arange(st["Q"].shape[0], device="cuda")
    b = torch.searchsorted(cu, i, right=True) - 1
    t = i - cu[b]
    bits = torch.zeros(lens.numel(), T, dtype=torch.int64, device="cuda")
    bits[b, t] = st["mask"]
    rel = torch.arange(st["max_kv"], device="cuda") - lens[:, None]  # place among the drafted tokens
    drafted = (rel >= 0) & (rel < (cu[1:] - cu[:-1])[:, None])
    sees = (rel < 0)[:, None] | drafted[:, None] & ((bits[:, :, None] >> rel.clamp(0, 63)[:, None]) & 1).bool()
    return b, t, sees


def _scores_plain(st):
    """Scores [B, Hkv, T, heads of a group, keys] of the padded rows, -inf where a row does not see a key."""
    B, Hkv, _, dh = st["K"].shape
    T, G = st["case"]["T"], st["Q"].shape[1] // Hkv
    b, t, sees = _padded(st)
    q = torch.zeros(B, T, Hkv, G, dh, device="cuda")
    q[b, t] = st["Q"].float().view(-1, Hkv, G, dh) / math.sqrt(dh)
    q = q.permute(0, 2, 1, 3, 4).reshape(B, Hkv, T * G, dh)
    s = q @ st["K"].float().transpose(2, 3)
    return b, t, s.view(B, Hkv, T, G, -1).masked_fill_(~sees[:, None, :, None], -math.inf)


def _attend_plain(st):
    b, t, s = _scores_plain(st)
    B, Hkv, T, G, n = s.shape
    m = s.amax(dim=4, keepdim=True)
    p = torch.exp(s - torch.where(torch.isfinite(m), m, 0.0))
    l = p.sum(dim=4, keepdim=True)
    lse = (m + torch.log(l))[..., 0]
    p = (p / torch.where(l > 0, l, 1.0)).view(B, Hkv, T * G, n)
    w = torch.zeros(B, T, G, device="cuda")  # 1 for the padded places that hold a row
    w[b, t] = 1.0
    st["acc"] += (w.view(B, 1, 1, T * G) @ p)[:, :, 0]
    o = (p @ st["V"].float()).view(B, Hkv, T, G, -1)[b, :, t].flatten(1, 2)
    return {"O": o.to(st["Q"].dtype), "lse": lse[b, :, t].flatten(1, 2).t().contiguous(), "acc": st["acc"]}


def _credit_plain(st):
    b, t, s = _scores_plain(st)
    B, Hkv, T, G, _ = s.shape
    lse = torch.zeros(B, T, Hkv, G, device="cuda")
    lse[b, t] = st["lse"].t().reshape(-1, Hkv, G)
    w = torch.zeros(B, T, device="cuda")
    w[b, t] = st["taken"]
    p = torch.exp(s - lse.permute(0, 2, 1, 3)[..., None])
    st["acc"] += (p * w[:, None, :, None, None]).sum(dim=(2, 3))
    return {"acc": st["acc"]}


def _evict_plain(st):
    case, lens, acc, pos = st["case"], st["lens"].long()[:, None, None], st["acc"], st["pos"]
    keep, cap = case["keep"], acc.shape[2]
    slot = torch.arange(cap, device="cuda")
    held = slot < lens
    guarded = (pos < case["sink"]) | (pos >= st["seen"][:, None, None] - case["recent"])
    # one whole number that orders the slots: held, guarded, weight, then the lowest slot
    bits = acc.view(torch.int32).long()  # ascending as the weights are, which are not negative
    key = ((held * 2 + (held & guarded)).long() << 52) | (bits << 20) | (cap - 1 - slot)
    rank = torch.empty_like(key)
    rank.scatter_(2, key.argsort(dim=2, descending=True), slot.expand_as(key).contiguous())
    kept = held & (rank < keep)
    # kept slots past `keep` fill the holes before it, both in ascending order
    late = torch.where(kept & (slot >= keep), slot, cap).sort(dim=2).values
    hole = ~kept[:, :, :keep]
    nth = torch.where(hole, hole.long().cumsum(dim=2) - 1, 0)
    src = torch.where(hole, late.gather(2, nth), slot[:keep])
    new = lens.clamp(max=keep)
    first = slot[:keep] < new
    idx = torch.where(first, src, -1).int()
    src = torch.where(first, src, slot[:keep])
    for name in ("K", "V"):
        st[name][:, :, :keep] = st[name].gather(2, src[..., None].expand(-1, -1, -1, st[name].shape[3]))
    out = torch.where(slot < new, torch.nn.functional.pad(acc.gather(2, src), (0, cap - keep)), 0.0)
    st["acc_out"].copy_(torch.where(held, out, st["acc_out"]))
    out = torch.where(slot < new, torch.nn.functional.pad(pos.gather(2, src), (0, cap - keep)), -1)
    st["pos_out"].copy_(torch.where(held, out, st["pos_out"]))
    return {"lens": new[:, 0, 0].int(), "idx": idx, "K": st["K"], "V": st["V"], "acc": st["acc_out"],
            "pos": st["pos_out"]}


# ----------------------------------------------------------------------------- one pass


def run(st):
    case = st["case"]
    kind = case["kind"]
    if not own:
        if kind == "loss":
            _, lse, loss, _, _ = _loss_plain(st)
            return {"loss": loss, "lse": lse}
        return {"train": _train_plain, "attend": _attend_plain, "credit": _credit_plain, "evict": _evict_plain}[kind](st)
    import paper_2608_15592_amd as estp
    if kind in ("loss", "train"):
        loss, lse = estp.token_loss(st["X"], st["W"], st["targets"])
        if kind == "loss":
            return {"loss": loss, "lse": lse}
        dX, dW = estp.token_loss_backward(st["X"], st["W"], st["targets"], lse, st["grad"])
        return {"loss": loss, "lse": lse, "dX": dX, "dW": dW}
    if kind == "attend":
        O, lse = estp.tree_attention(st["Q"], st["K"], st["V"], st["lens"], st["cu"], case["T"], st["max_kv"],
                                     tree_mask=st["mask"], acc=st["acc"])
        return {"O": O, "lse": lse, "acc": st["acc"]}
    if kind == "credit":
        estp.tree_importance(st["Q"], st["K"], st["lse"], st["lens"], st["cu"], case["T"], st["max_kv"], st["acc"],
                             tree_mask=st["mask"], row_weight=st["taken"])
        return {"acc": st["acc"]}
    lens, idx = estp.cache_evict(st["K"], st["V"], st["acc"], st["pos"], st["lens"], st["seen"], case["keep"],
                                 recent=case["recent"], sink=case["sink"], acc_out=st["acc_out"],
                                 pos_out=st["pos_out"])
    return {"lens": lens, "idx": idx, "K": st["K"], "V": st["V"], "acc": st["acc_out"], "pos": st["pos_out"]}


# ----------------------------------------------------------------------------- what a pass cannot do without


def work(case):
    need = _needs(case)
    return {k: float(v) for k, v in need.items()}


def _needs(case):
    d, V, Hq, Hkv, dh = MODELS[case["model"]]
    es = 4 if case["dtype"] == "f32" else 2
    if case["kind"] in ("loss", "train"):
        n = case["n_tok"]
        live = n * (1.0 - case["ignored"])
        if case["kind"] == "loss":
            return {"bytes": es * (n + V) * d + 12 * n, "flops": 2 * n * V * d}
        return {"bytes": 2 * es * (n + V) * d + 16 * n, "flops": 2 * n * V * d + 4 * live * V * d}
    lens = _lengths(case)
    if case["kind"] == "evict":
        # every weight and position read and written; as many K and V rows moved as the budget and the length
        # leave, if the kept slots are spread evenly over the sequence
        over = lens[lens > case["keep"]]
        moved = (case["keep"] * (1.0 - case["keep"] / over)).sum()
        return {"bytes": Hkv * (16 * lens.sum() + 4 * case["keep"] * len(lens) + 4 * es * dh * moved), "flops": 0.0}
    rows = _rows(case)
    keys = lens + rows
    n = int(rows.sum())
    pairs = (rows * keys).sum()
    if case["kind"] == "attend":
        return {"bytes": Hkv * keys.sum() * (2 * es * dh + 8) + n * Hq * (2 * es * dh + 4),
                "flops": 4 * dh * Hq * pairs}
    return {"bytes": Hkv * keys.sum() * (es * dh + 8) + n * Hq * (es * dh + 4), "flops": 2 * dh * Hq * pairs}


# ----------------------------------------------------------------------------- 64-bit values


def _attention64(st, weight=None):
    """(O, lse, weight received by each slot), sequence by sequence."""
    Q, K, V, cu = st["Q"].double(), st["K"], st["V"], st["cu"].tolist()
    B, Hkv, cap, dh = K.shape
    G = Q.shape[1] // Hkv
    O, lse = torch.zeros_like(Q), torch.zeros(Q.shape[1], Q.shape[0], dtype=torch.float64, device="cuda")
    got = torch.zeros(B, Hkv, cap, dtype=torch.float64, device="cuda")
    for b, n in enumerate(st["lens"].tolist()):
        T = cu[b + 1] - cu[b]
        mask = st["mask"][cu[b]:cu[b + 1]]
        sees = torch.ones(T, n + T, dtype=torch.bool, device="cuda")
        sees[:, n:] = (mask[:, None] >> torch.arange(T, device="cuda") & 1) > 0
        for h in range(Hkv):
            k, v = K[b, h, :n + T].double(), V[b, h, :n + T].double()
            q = Q[cu[b]:cu[b + 1], h * G:(h + 1) * G]
            s = (q.reshape(T * G, dh) @ k.t().contiguous()).view(T, G, -1) / math.sqrt(dh)
            s = torch.where(sees[:, None], s, -math.inf)
            l = torch.logsumexp(s, dim=2)
            p = torch.exp(s - l[..., None])
            lse[h * G:(h + 1) * G, cu[b]:cu[b + 1]] = l.t()
            O[cu[b]:cu[b + 1], h * G:(h + 1) * G] = (p.view(T * G, -1) @ v).view(T, G, dh)
            if weight is not None:  # the rows' given normalisers
                given = st["lse"][h * G:(h + 1) * G, cu[b]:cu[b + 1]].t().double()
                p = torch.exp(s - given[..., None]) * weight[cu[b]:cu[b + 1], None, None]
            got[b, h, :n + T] = p.sum(dim=(0, 1))
    return O, lse, got


def _train64(st):
    X, W = st["X"].double(), st["W"].double()
    logp = torch.log_softmax(X @ W.t(), dim=1)
    rows = torch.nonzero(st["targets"] >= 0)[:, 0]
    t = st["targets"][rows].long()
    loss = torch.zeros(X.shape[0], dtype=torch.float64, device="cuda")
    loss[rows] = -logp[rows, t]
    lse = (X * W[0]).sum(dim=1) - logp[:, 0]
    if st["case"]["kind"] == "loss":
        return {"loss": loss, "lse": lse}
    G = logp[rows].exp_()
    G[torch.arange(rows.numel(), device="cuda"), t] -= 1.0
    G *= st["grad"][rows, None].double()
    dX = torch.zeros_like(X)
    dX[rows] = G @ W
    return {"loss": loss, "lse": lse, "dX": dX, "dW": G.t().contiguous() @ X[rows]}


def _evict64(st):
    case = st["case"]
    keep = case["keep"]
    acc, pos = st["acc"].double().cpu().numpy(), st["pos"].cpu().numpy()
    B, Hkv, cap = acc.shape
    idx = np.full((B, Hkv, keep), -1, dtype=np.int64)
    acc_out, pos_out = np.zeros((B, Hkv, cap)), np.zeros((B, Hkv, cap), dtype=np.int64)
    lens, seen = st["lens"].tolist(), st["seen"].tolist()
    for b in range(B):
        n = lens[b]
        for h in range(Hkv):
            guarded = (pos[b, h, :n] < case["sink"]) | (pos[b, h, :n] >= seen[b] - case["recent"])
            best = np.lexsort((np.arange(n), -acc[b, h, :n], ~guarded))[:keep]
            place = np.arange(min(n, keep))
            holes = np.setdiff1d(place, best)
            place[holes] = np.sort(best[best >= keep])
            idx[b, h, :len(place)] = place
            acc_out[b, h, :len(place)], pos_out[b, h, :len(place)] = acc[b, h, place], pos[b, h, place]
            pos_out[b, h, len(place):n] = -1
            for C in (st["K"], st["V"]):
                C[b, h, :len(place)] = C[b, h, torch.from_numpy(place).cuda()]
    return {"lens": torch.tensor([min(n, keep) for n in lens]).cuda(), "idx": torch.from_numpy(idx).cuda(),
            "K": st["K"].double(), "V": st["V"].double(), "acc": torch.from_numpy(acc_out).cuda(),
            "pos": torch.from_numpy(pos_out).cuda()}


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] in ("loss", "train"):
        return _train64(st)
    if case["kind"] == "evict":
        return _evict64(st)
    O, lse, got = _attention64(st, st["taken"].double() if case["kind"] == "credit" else None)
    acc = st["acc"].double() + got
    return {"acc": acc} if case["kind"] == "credit" else {"O": O, "lse": lse, "acc": acc}

"""Log-probabilities with alternatives and distillation over the LM head, as measurable cases.

* ``logprobs`` - log-probabilities of given tokens, the entropy of their distributions and each one's most probable
  alternatives (``token_logprobs``): what a server returns beside its tokens, and what a teacher leaves for a student
* ``distill``  - a student's divergence from a teacher's top tokens (``distill_loss``): evaluation
* ``train``    - the same with its gradients (``distill_loss`` and ``distill_loss_backward``)

Where ``own`` is false, ``run`` computes them in elementary torch operations in 32 bits; where it is true, through the
library.  The model shapes are those of the scoring path's workloads.
"""
from __future__ import annotations

import math

import torch

own = False

# hidden size, vocabulary
MODELS = {
    "llama-8b": (4096, 128256),
    "llama-1b": (2048, 128256),
    "qwen-1.5b": (1536, 151936),
    "tiny": (64, 1000),
}


def listed():
    return [
        # the next token of a lone request, with five alternatives: the smallest call of the serving side
        {"name": "next_one", "kind": "logprobs", "model": "llama-8b", "dtype": "bf16", "n_tok": 1, "k": 5,
         "temperature": 1.0, "ignored": 0.0},
        # the next tokens of 48 running requests under a sampling temperature
        {"name": "next_batch", "kind": "logprobs", "model": "qwen-1.5b", "dtype": "bf16", "n_tok": 48, "k": 20,
         "temperature": 0.7, "ignored": 0.0},
        # drafted tokens of a few requests of a model in fp32
        {"name": "next_f32", "kind": "logprobs", "model": "llama-1b", "dtype": "f32", "n_tok": 37, "k": 20,
         "temperature": 1.0, "ignored": 0.0},
        # the scores of a few prompts' tokens, the last of each without a next one
        {"name": "score_prompts", "kind": "logprobs", "model": "llama-1b", "dtype": "bf16", "n_tok": 1511, "k": 5,
         "temperature": 1.0, "ignored": 0.01},
        # a teacher's pass over a batch: the top tokens that its student will be trained on
        {"name": "teacher_llama", "kind": "logprobs", "model": "llama-8b", "dtype": "bf16", "n_tok": 8192, "k": 64,
         "temperature": 2.0, "ignored": 0.0},
        # a student held against a teacher's records
        {"name": "eval_qwen", "kind": "distill", "model": "qwen-1.5b", "dtype": "bf16", "n_tok": 3001, "k": 32,
         "temperature": 1.0, "renormalise": True, "ignored": 0.0},
        # the tokens of one decoding step, watched for drift
        {"name": "eval_few", "kind": "distill", "model": "llama-1b", "dtype": "bf16", "n_tok": 12, "k": 16,
         "temperature": 1.0, "renormalise": False, "ignored": 0.0},
        # the smallest fp32 configuration: launches are all there is
        {"name": "train_tiny_f32", "kind": "train", "model": "tiny", "dtype": "f32", "n_tok": 128, "k": 8,
         "temperature": 1.0, "renormalise": True, "ignored": 0.0},
        # a small step in fp32
        {"name": "train_qwen_f32", "kind": "train", "model": "qwen-1.5b", "dtype": "f32", "n_tok": 90, "k": 20,
         "temperature": 2.0, "renormalise": True, "ignored": 0.1},
        # a draft model corrected on the tokens that were just verified
        {"name": "train_draft", "kind": "train", "model": "llama-1b", "dtype": "bf16", "n_tok": 40, "k": 10,
         "temperature": 1.0, "renormalise": True, "ignored": 0.0},
        # one ragged micro-batch, a quarter of its tokens prompt (no loss there)
        {"name": "train_micro", "kind": "train", "model": "llama-1b", "dtype": "bf16", "n_tok": 1021, "k": 32,
         "temperature": 2.0, "renormalise": True, "ignored": 0.25},
        # a full training batch: the largest call
        {"name": "train_llama", "kind": "train", "model": "llama-8b", "dtype": "bf16", "n_tok": 4096, "k": 64,
         "temperature": 1.0, "renormalise": False, "ignored": 0.0},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["logprobs", "logprobs", "distill", "train", "train"])
    f32 = rng.random() < 0.25
    model = rng.choice(["tiny", "llama-1b", "qwen-1.5b"] if f32 else ["llama-8b", "llama-1b", "qwen-1.5b"])
    most = 400 if f32 else 4000 if kind == "train" else 8000
    case = {"kind": kind, "model": model, "dtype": "f32" if f32 else "bf16", "n_tok": _log_int(rng, 1, most),
            "k": _log_int(rng, 1, 128), "temperature": rng.choice([0.7, 1.0, 2.0]),
            "ignored": rng.choice([0.0, 0.2, 0.5])}
    if kind != "logprobs":
        case["renormalise"] = rng.random() < 0.7
    return case


# ----------------------------------------------------------------------------- inputs


def _grid(x, steps, dtype):
    """Rounded to whole multiples of 1 / steps.  Hidden states and weights have 8 significant bits each, as those of a
    checkpoint held in 8 bits; their products then add up exactly in 32 bits, in any order, so that the alternatives of
    a token have one order, whose ties are real ones."""
    return (torch.round(x * steps) / steps).to(dtype)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    d, V = MODELS[case["model"]]
    n, k = case["n_tok"], case["k"]
    dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16

    def uniform(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    W = _grid(0.02 * torch.randn(V, d, generator=g, device="cuda"), 1024.0, dtype)
    # hidden states of RMS 1 that lean towards their token by up to 12 nats, as a trained model's do
    t = torch.randint(V, (n,), generator=g, device="cuda")
    x = torch.randn(n, d, generator=g, device="cuda")
    x *= torch.rsqrt(x.square().mean(dim=1, keepdim=True))
    x += 12.0 * uniform(n, 1) * W[t].float() / (0.0004 * d)
    st = {"case": case, "X": _grid(x, 32.0, dtype), "W": W}
    out = uniform(n) < case["ignored"]
    if case["kind"] == "logprobs":
        st["targets"] = torch.where(out, -100, t).to(torch.int32)
        return st
    # the teacher's tokens, the one that the student leans to in any place among them, with log-probabilities that
    # fall by a power of the rank and a tail left out; some rows hold fewer than k, the rest is -1
    step = torch.randint(1, V // k + 1, (n, 1), generator=g, device="cuda")
    place = torch.randint(k, (n, 1), generator=g, device="cuda")
    rank = torch.arange(k, device="cuda")
    ids = (t[:, None] + (rank - place) * step) % V
    fall = -(0.5 + 2.0 * uniform(n, 1)) * torch.log(1.0 + rank) + 0.3 * torch.randn(n, k, generator=g, device="cuda")
    held = torch.where(uniform(n, 1) < 0.2, 1 + (k * uniform(n, 1)).long(), k)
    held = torch.where(out[:, None], 0, held)
    logp = torch.log_softmax(fall.sort(dim=1, descending=True).values, dim=1) + torch.log(1.0 - 0.3 * uniform(n, 1))
    st["ids"] = torch.where(rank < held, ids, -1).to(torch.int32)
    st["logp"] = torch.where(rank < held, logp, 0.0)
    if case["kind"] == "train":
        # the weight of each token's loss: a mean over the batch, scaled as the temperature scales the gradient
        st["grad"] = case["temperature"] ** 2 * (0.5 + uniform(n)) / n
    return st


# ----------------------------------------------------------------------------- plain forms


def _head_plain(st):
    """Logits over the temperature, and their log-sum-exps."""
    z = st["X"].float() @ st["W"].float().t()
    s = z / st["case"]["temperature"]
    m = s.amax(dim=1, keepdim=True)
    return z, s, m[:, 0] + torch.log(torch.exp(s - m).sum(dim=1))


def _logprobs_plain(st):
    z, s, lse = _head_plain(st)
    V = z.shape[1]
    live = st["targets"] >= 0
    t = torch.where(live, st["targets"], 0).long()
    logprob = torch.where(live, s.gather(1, t[:, None])[:, 0] - lse, 0.0)
    p = torch.exp(s - lse[:, None])
    H = lse - (p * s).sum(dim=1)
    # one whole number that orders the vocabulary: the logit, then the lowest index
    bits = (z + 0.0).view(torch.int32).long()
    key = (torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits) << 32) | (V - 1 - torch.arange(V, device="cuda"))
    top = V - 1 - (key.topk(st["case"]["k"], dim=1).values & 0xFFFFFFFF)
    return {"logprob": logprob, "lse": lse, "H": H, "top_id": top.int(), "top_logprob": s.gather(1, top) - lse[:, None]}


def _distill_plain(st):
    """What both passes need: log-sum-exps and scaled logits, the teacher's places and weights, and the losses."""
    _, s, lse = _head_plain(st)
    held = (st["ids"] >= 0) & (st["ids"] < s.shape[1])
    ids = torch.where(held, st["ids"], 0).long()
    logp = torch.where(held, st["logp"], -math.inf)
    if st["case"]["renormalise"]:
        m = logp.amax(dim=1, keepdim=True).clamp(min=-1e30)
        logp = logp - m - torch.log(torch.exp(logp - m).sum(dim=1, keepdim=True))
    p = torch.where(held, torch.exp(logp), 0.0)
    logq = torch.where(held, s.gather(1, ids) - lse[:, None], 0.0)
    loss = torch.where(p > 0, p * (logp - logq), 0.0).sum(dim=1)
    return s, lse, ids, p, loss, logq


def _train_plain(st):
    s, lse, ids, p, loss, logq = _distill_plain(st)
    G = torch.exp(s - lse[:, None]) * p.sum(dim=1, keepdim=True)
    G.scatter_add_(1, ids, -p)
    G *= st["grad"][:, None] / st["case"]["temperature"]
    dX = (G @ st["W"].float()).to(st["X"].dtype)
    dW = (G.t() @ st["X"].float()).to(st["W"].dtype)
    return {"loss": loss, "lse": lse, "logq": logq, "dX": dX, "dW": dW}


# ----------------------------------------------------------------------------- one pass


def run(st):
    case = st["case"]
    kind = case["kind"]
    if not own:
        if kind == "logprobs":
            return _logprobs_plain(st)
        if kind == "train":
            return _train_plain(st)
        _, lse, _, _, loss, logq = _distill_plain(st)
        return {"loss": loss, "lse": lse, "logq": logq}
    import paper_2608_15592_amd as estp
    if kind == "logprobs":
        logprob, lse, H, top_id, top_logprob = estp.token_logprobs(st["X"], st["W"], st["targets"], case["k"],
                                                                   temperature=case["temperature"])
        return {"logprob": logprob, "lse": lse, "H": H, "top_id": top_id, "top_logprob": top_logprob}
    how = {"temperature": case["temperature"], "renormalise": case["renormalise"]}
    loss, lse, logq = estp.distill_loss(st["X"], st["W"], st["ids"], st["logp"], **how)
    out = {"loss": loss, "lse": lse, "logq": logq}
    if kind == "train":
        out["dX"], out["dW"] = estp.distill_loss_backward(st["X"], st["W"], st["ids"], st["logp"], lse, logq,
                                                          st["grad"], **how)
    return out


# ----------------------------------------------------------------------------- what a pass cannot do without


def work(case):
    d, V = MODELS[case["model"]]
    n, k = case["n_tok"], case["k"]
    size = 4 if case["dtype"] == "f32" else 2
    once, product = size * (n + V) * d, 2 * n * V * d
    if case["kind"] == "logprobs":
        need = once + 16 * n + 8 * n * k, product
    elif case["kind"] == "distill":
        need = once + 8 * n + 12 * n * k, product
    else:
        need = 2 * once + 12 * n + 12 * n * k, product + 2 * product * (1.0 - case["ignored"])
    return {"bytes": float(need[0]), "flops": float(need[1])}


# ----------------------------------------------------------------------------- 64-bit values


def _logprobs64(st):
    k, parts = st["case"]["k"], []
    W = st["W"].double()
    for x, t in zip(st["X"].split(512), st["targets"].split(512)):
        z = x.double() @ W.t()
        logp = torch.log_softmax(z / st["case"]["temperature"], dim=1)
        lse = z[:, 0] / st["case"]["temperature"] - logp[:, 0]
        H = torch.special.entr(logp.exp()).sum(dim=1)
        top = z.sort(dim=1, descending=True, stable=True).indices[:, :k]
        given = torch.where(t >= 0, logp.gather(1, t.clamp(min=0).long()[:, None])[:, 0], 0.0)
        parts.append((given, lse, H, top, logp.gather(1, top)))
    return dict(zip(("logprob", "lse", "H", "top_id", "top_logprob"), map(torch.cat, zip(*parts))))


def _distill64(st):
    case = st["case"]
    X, W = st["X"].double(), st["W"].double()
    z = (X @ W.t()) / case["temperature"]
    lse = torch.logsumexp(z, dim=1)
    logq = torch.zeros(st["ids"].shape, dtype=torch.float64, device="cuda")
    loss = torch.zeros_like(lse)
    target = torch.zeros_like(z)  # the teacher's probabilities, spread over the vocabulary
    for j in range(case["k"]):
        rows = torch.nonzero(st["ids"][:, j] >= 0)[:, 0]
        v = st["ids"][rows, j].long()
        logq[rows, j] = z[rows, v] - lse[rows]
        logp = st["logp"][rows, j].double()
        if case["renormalise"]:
            logp = logp - torch.where(st["ids"][rows] >= 0, st["logp"][rows].double(), -math.inf).logsumexp(dim=1)
        target[rows, v] += logp.exp()
        loss[rows] += logp.exp() * (logp - logq[rows, j])
    out = {"loss": loss, "lse": lse, "logq": logq}
    if case["kind"] == "train":
        z -= lse[:, None]
        G = z.exp_().mul_(target.sum(dim=1, keepdim=True)).sub_(target)
        G *= st["grad"].double()[:, None] / case["temperature"]
        out["dX"], out["dW"] = G @ W, G.t().contiguous() @ X
    return out


def exact(case, seed):
    st = prepare(case, seed)
    return _logprobs64(st) if case["kind"] == "logprobs" else _distill64(st)

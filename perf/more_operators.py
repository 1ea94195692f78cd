"""The drafter's losses on the LM head, with their gradients, and the teacher's top logits: what is measured of them, and
their plain forms.

Four passes, as the training of a drafter makes them:

``loss``      softmax cross entropy of h w^T over the vocabulary, a weight per row, rows without a target (evaluation)
``train``     the same with the gradients of the hidden states and of the head
``distill``   the Kullback-Leibler divergence from a teacher's top logits (ids and values, at a temperature), with both gradients
``top``       the top logits of a teacher's rows: ids and values, falling, lowest index first among equals

Rows without a target (a padded batch, positions that are not masked) have loss 0 and gradient 0.

``own`` false: elementary torch operations in fp32.  ``own`` true: this package's calls.
"""
import math

import torch

own = False


# ---------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------

def listed():
    return [
        # A block of 8 drafts of the smallest workload's shape: the shortest call there is.
        {"name": "loss-tiny", "op": "loss", "M": 8, "live": 8, "hid": 512, "V": 4096},
        # Evaluation of a drafter on 64 blocks of 32 (hidden 2048, the named workloads' vocabulary).
        {"name": "loss-eval", "op": "loss", "M": 2048, "live": 2048, "hid": 2048, "V": 151936},
        # A training step on one small block, some of its positions masked.
        {"name": "train-tiny", "op": "train", "M": 32, "live": 20, "hid": 512, "V": 4096},
        # The second stage of training: the last R <= 96 tokens of one answer, weights alpha^(R - i).
        {"name": "train-suffix", "op": "train", "M": 96, "live": 77, "hid": 2048, "V": 151936},
        # A vocabulary of odd size, a batch that is no multiple of anything.
        {"name": "train-odd", "op": "train", "M": 1000, "live": 611, "hid": 1024, "V": 50257},
        # The first stage: 4096 positions of which about half are masked, weights 1 / t.
        {"name": "train-batch", "op": "train", "M": 4096, "live": 2100, "hid": 2048, "V": 151936},
        # One block against the teacher's 8 best tokens; the same at the largest hidden size; a batch against 64.
        {"name": "distill-tiny", "op": "distill", "M": 32, "live": 32, "hid": 512, "V": 4096, "K": 8, "T": 1.0},
        {"name": "distill-wide", "op": "distill", "M": 512, "live": 400, "hid": 4096, "V": 151936, "K": 32, "T": 2.0},
        {"name": "distill-batch", "op": "distill", "M": 2048, "live": 2048, "hid": 2048, "V": 151936, "K": 64, "T": 1.0},
        # The teacher's logits of one token, of one block, of 64 blocks.
        {"name": "top-token", "op": "top", "M": 1, "V": 151936, "K": 8},
        {"name": "top-block", "op": "top", "M": 32, "V": 151936, "K": 64},
        {"name": "top-batch", "op": "top", "M": 2048, "V": 151936, "K": 64},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["loss", "train", "train", "distill", "distill", "top"])
    V = rng.choice([151936, _log_int(rng, 1000, 151936)])
    if op == "top":
        return {"op": op, "M": _log_int(rng, 1, 2048), "V": V, "K": _log_int(rng, 1, 128)}
    hid, M = 64 * _log_int(rng, 4, 64), _log_int(rng, 1, 4096)
    most = 2048 * 2048 * 151936 // (hid * V)                 # no more work than the largest listed case
    M = min(M, 2 * most)
    case = {"op": op, "M": M, "live": min(most, max(1, round(M * rng.choice([1.0, rng.random()])))), "hid": hid, "V": V}
    if op == "distill":
        case |= {"K": _log_int(rng, 1, 128), "T": rng.choice([1.0, 1.0, 0.7, 2.0])}
    return case


def work(case):
    M, V = case["M"], case["V"]
    if case["op"] == "top":
        return {"bytes": 4 * M * V + 8 * M * case["K"], "flops": M * V}
    L, hid, K = case["live"], case["hid"], case.get("K", 1)
    once = {"bytes": 2 * hid * (L + V) + 4 * M * (2 + K) + 4 * L * (K if "K" in case else 0), "flops": 2 * L * V * hid}
    if case["op"] == "loss":
        return once
    return {"bytes": once["bytes"] + 2 * hid * (M + V), "flops": 3 * once["flops"]}


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------

def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)


def _uniform(gen, *shape):
    return torch.rand(*shape, generator=gen, device="cuda", dtype=torch.float32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    M, V, op = case["M"], case["V"], case["op"]
    state = {"case": dict(case)}
    if op == "top":
        # a language model's logits: a few tokens far above a bulk
        z = 2.0 * _normal(gen, M, V)
        z += 12.0 * _uniform(gen, M, V).pow_(24)
        state["logits"] = z
        if own:
            state["ids"] = torch.empty(M, case["K"], dtype=torch.int32, device="cuda")
            state["values"] = torch.empty(M, case["K"], dtype=torch.float32, device="cuda")
        return state
    hid, K = case["hid"], case.get("K", 1)
    w = (_normal(gen, V, hid) / math.sqrt(hid)).to(torch.bfloat16)
    # the rows' lists of tokens: distinct, the best first, `live` rows have one
    first = torch.randint(V, (M, 1), generator=gen, device="cuda")
    step = torch.randint(1, max(2, V // K), (M, K), generator=gen, device="cuda").cumsum(1)
    ids = ((first + step) % V).to(torch.int32)
    rows = torch.randperm(M, generator=gen, device="cuda")
    dead = rows[case["live"]:]
    # hidden states of a drafter that is sure of some targets and not of others
    sure = 14.0 * _uniform(gen, M, 1)
    best = w[ids[:, 0].long()].float()
    h = _normal(gen, M, hid) + sure * best / best.square().sum(dim=1, keepdim=True).clamp_min(1e-6)
    state["h"], state["w"] = h.to(torch.bfloat16), w
    state["weight"] = 1.0 / (0.1 + 0.9 * _uniform(gen, M))                     # 1 / t of the row's sequence
    state["grad"] = torch.full((M,), 1.0 / case["live"], device="cuda")        # the mean's gradient
    if op == "distill":
        # the teacher's logits fall with the rank; some rows have fewer tokens than K (a nucleus)
        rank = torch.arange(1, K + 1, device="cuda", dtype=torch.float32)
        state["teacher"] = 20.0 - 1.5 * torch.log(rank) - 0.3 * _uniform(gen, M, K).cumsum(1)
        length = torch.where(_uniform(gen, M, 1) < 0.5, K, torch.randint(1, K + 1, (M, 1), generator=gen, device="cuda"))
        ids = torch.where(torch.arange(K, device="cuda")[None, :] < length, ids, -1)
    ids[dead] = -1
    state["ids"] = ids.contiguous()
    if own:
        from paper_2512_15176_b200 import runner
        state["head"] = runner.HeadLoss(w, M, top=K, grad=op != "loss")
    return state


# ---------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------

def _top(s):
    z, K = s["logits"], s["case"]["K"]
    # one whole number per token, ordered by value and then by falling index
    bits = z.view(torch.int32).long()
    key = torch.where(bits < 0, -(bits & 0x7fffffff), bits)
    at = torch.arange(z.shape[1], device="cuda")
    best = torch.topk((key << 32) - at, K, dim=1).values
    ids = (-best) & 0xffffffff
    return ids.to(torch.int32), torch.gather(z, 1, ids)


def _head(s):
    c = s["case"]
    M, V, K, T = c["M"], c["V"], c.get("K", 1), c.get("T", 1.0)
    live = torch.nonzero(s["ids"][:, 0] >= 0).view(-1)
    h, w = s["h"][live].float(), s["w"].float()
    ids, weight = s["ids"][live].long(), s["weight"][live]
    z = h @ w.t() / T
    top = z.amax(dim=1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(dim=1, keepdim=True)
    lse = (top + torch.log(total)).view(-1)
    held = ids >= 0
    at = torch.gather(z, 1, ids.clamp_min(0))
    if c["op"] == "distill":
        u = torch.where(held, s["teacher"][live] / T, -math.inf)
        u = u - u.amax(dim=1, keepdim=True)
        log_t = u - torch.log(torch.exp(u).sum(dim=1, keepdim=True))
        t = torch.exp(log_t)
        each = torch.where(held, t * (log_t - at + lse[:, None]), 0.0).sum(dim=1) * (T * T)
    else:
        t = torch.ones(live.numel(), 1, device="cuda")
        each = lse - at.view(-1)
    loss = torch.zeros(M, device="cuda").index_copy(0, live, weight * each)
    if c["op"] == "loss":
        return {"loss": loss, "lse": torch.zeros(M, device="cuda").index_copy(0, live, lse)}
    scale = (weight * s["grad"][live] * T)[:, None]
    g = e.div_(total)
    g.scatter_add_(1, ids.clamp_min(0), -t * held)
    g.mul_(scale)
    dh = torch.zeros(M, h.shape[1], device="cuda").index_copy(0, live, g @ w)
    return {"loss": loss, "dh": dh.to(torch.bfloat16), "dw": (g.t() @ h).to(torch.bfloat16)}


def run(state):
    c = state["case"]
    if not own:
        return _top(state) if c["op"] == "top" else _head(state)
    if c["op"] == "top":
        from paper_2512_15176_b200 import binding
        binding.deer_top_logits(state["logits"], state["ids"], state["values"])
        return state["ids"], state["values"]
    head = state["head"]
    if c["op"] == "distill":
        loss = head.distill(state["h"], state["ids"], state["teacher"], c["T"], state["weight"])
    else:
        loss = head.cross_entropy(state["h"], state["ids"].view(-1), state["weight"])
    if c["op"] == "loss":
        return {"loss": loss, "lse": head.lse}
    dh, dw = head.backward(state["grad"])
    return {"loss": loss, "dh": dh, "dw": dw}


# ---------------------------------------------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    M = case["M"]
    if case["op"] == "top":
        values, ids = torch.sort(s["logits"].double(), dim=1, descending=True, stable=True)
        return ids[:, :case["K"]].to(torch.int32), values[:, :case["K"]].contiguous()
    T = float(case.get("T", 1.0))
    h, w = s["h"].double(), s["w"].double()
    loss, lse = (torch.zeros(M, dtype=torch.float64, device="cuda") for _ in range(2))
    dh, dw = torch.zeros_like(h), torch.zeros_like(w)
    rows = [r for r, k in enumerate(s["ids"][:, 0].tolist()) if k >= 0]
    for i in range(0, len(rows), 256):
        r = torch.tensor(rows[i:i + 256], device="cuda")
        target = torch.zeros(len(r), case["V"], dtype=torch.float64, device="cuda")
        if case["op"] == "distill":
            listed_ = s["ids"][r] >= 0
            t = torch.softmax(torch.where(listed_, s["teacher"][r].double() / T, torch.full((), -math.inf, dtype=torch.float64, device="cuda")), dim=1)
            for j in range(case["K"]):
                target[torch.arange(len(r), device="cuda"), s["ids"][r, j].clamp_min(0).long()] += t[:, j]
        else:
            target[torch.arange(len(r), device="cuda"), s["ids"][r, 0].long()] = 1.0
        logp = torch.log_softmax(h[r] @ w.t() / T, dim=1)
        lse[r] = torch.logsumexp(h[r] @ w.t() / T, dim=1)
        some = target > 0
        loss[r] = s["weight"][r].double() * T * T * torch.where(some, target * (torch.log(torch.where(some, target, 1.0)) - logp), 0.0).sum(dim=1)
        g = (torch.exp(logp) - target) * (s["weight"][r].double() * s["grad"][r].double() * T)[:, None]
        dh[r] = g @ w
        dw += g.t() @ h[r]
    if case["op"] == "loss":
        return {"loss": loss, "lse": lse}
    return {"loss": loss, "dh": dh, "dw": dw}

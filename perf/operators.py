"""The operators of the 8-bit verifier layer: what is measured of them, and their plain forms.

Five operators that are used together, in the order in which a layer of the verifier calls them:

``rmsnorm``    residual addition + RMSNorm of bf16 rows, written as e4m3 codes with one fp32 scale per 128 columns
``linear``     e4m3 rows times an e4m3 weight, both with scales (rows: per 128 columns; weight: per 128 x 128 block)
``attention``  a block of k <= 32 rows against a paged cache of e4m3 keys and values with one fp32 scale per page of
               16 tokens and head; the tokens behind the last full page, and the block's own rows, are bf16
``store``      the accepted rows enter that cache: full pages are quantised, the rest stays in bf16
``quantize``   bf16 rows, or SiLU(gate) * up of them, as e4m3 codes with one scale per 128 columns

A scale is s = max(amax / 448, 2^-126) of the values it covers, a code the value / s rounded to e4m3.

``own`` false: elementary torch operations in fp32.  ``own`` true: this package's calls.
"""
import math

import torch

own = False

E4M3_MAX = 448.0
SCALE_MIN = 2.0 ** -126
PAGE = 16
TAIL = 48                      # rows of the bf16 tail of a sequence: three pages, page p in rows (p % 3) * 16 ...
GROUP = 128


# ---------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------

def listed():
    return [
        # Qwen3-8B shapes: hidden 4096, 32 query / 8 KV heads of 128, intermediate 12288; a draft block is 32 rows.
        # The normalisation that opens a sub-layer, one sequence's block / 64 sequences' blocks.
        {"name": "rmsnorm-block", "op": "rmsnorm", "M": 32, "K": 4096, "residual": True},
        {"name": "rmsnorm-batch", "op": "rmsnorm", "M": 2048, "K": 4096, "residual": True},
        # The attention output of one block ahead of the output projection; the gated activation of 16 blocks.
        {"name": "quantize-block", "op": "quantize", "M": 32, "K": 4096, "gated": False},
        {"name": "quantize-gated", "op": "quantize", "M": 512, "K": 12288, "gated": True},
        # The output projection of one token; the down projection of one block; gate and up of 16 blocks.
        {"name": "linear-token", "op": "linear", "M": 1, "K": 4096, "N": 4096, "residual": True},
        {"name": "linear-block", "op": "linear", "M": 32, "K": 12288, "N": 4096, "residual": True},
        {"name": "linear-batch", "op": "linear", "M": 512, "K": 4096, "N": 24576, "residual": False},
        # One token against a short odd prefix; the headline block (ctx 4096); the 30B-A3B heads (32 / 4) at 16 ragged
        # sequences of 2k to 16k tokens.
        {"name": "attention-token", "op": "attention", "B": 1, "k": 1, "Hq": 32, "Hkv": 8, "D": 128, "lo": 1003, "hi": 1003, "mask": "causal"},
        {"name": "attention-block", "op": "attention", "B": 1, "k": 32, "Hq": 32, "Hkv": 8, "D": 128, "lo": 4096, "hi": 4096, "mask": "causal"},
        {"name": "attention-ragged", "op": "attention", "B": 16, "k": 32, "Hq": 32, "Hkv": 4, "D": 128, "lo": 2048, "hi": 16384, "mask": "causal"},
        # What a verify step keeps of its blocks (between nothing and all 32 rows); four prompts that enter at once.
        {"name": "store-step", "op": "store", "B": 16, "k": 32, "Hkv": 8, "D": 128, "lo": 2048, "hi": 4111},
        {"name": "store-prompt", "op": "store", "B": 4, "k": 4096, "Hkv": 8, "D": 128, "lo": 0, "hi": 0},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rmsnorm", "quantize", "linear", "attention", "attention", "store"])
    if op == "rmsnorm":
        return {"op": op, "M": _log_int(rng, 1, 2048), "K": 16 * _log_int(rng, 4, 256), "residual": rng.random() < 0.7}
    if op == "quantize":
        return {"op": op, "M": _log_int(rng, 1, 512), "K": 16 * _log_int(rng, 4, 768), "gated": rng.random() < 0.5}
    if op == "linear":
        return {"op": op, "M": _log_int(rng, 1, 512), "K": 16 * _log_int(rng, 8, 256), "N": 16 * _log_int(rng, 4, 1536),
                "residual": rng.random() < 0.5}
    if op == "attention":
        Hkv, D = rng.choice([2, 4, 8]), rng.choice([64, 128, 128])
        B = _log_int(rng, 1, 32)
        hi = _log_int(rng, 1, min(16384, 524288 // (B * Hkv)))
        return {"op": op, "B": B, "k": rng.choice([1, _log_int(rng, 1, 32), 32]), "Hq": Hkv * rng.choice([1, 2, 4, 8] if Hkv < 8 else [1, 2, 4]),
                "Hkv": Hkv, "D": D, "lo": hi // 2, "hi": hi, "mask": rng.choice(["causal", "causal", "bidir", "states"])}
    k, B = _log_int(rng, 1, 4096), _log_int(rng, 1, 64)
    k = min(k, 16384 // B)
    # a longer run of rows than one block is a prompt's next piece, and pieces begin at a page
    lo = 0 if k > 32 else _log_int(rng, 1, 2048)
    return {"op": op, "B": B, "k": k, "Hkv": rng.choice([2, 4, 8]), "D": rng.choice([64, 128]), "lo": lo, "hi": 2 * lo}


def _lengths(case):
    """Committed lengths, spread over [lo, hi]: part of the case, so that its work is known without its inputs."""
    lo, hi = case["lo"], case["hi"]
    return [lo + int((hi - lo) * ((0.37 + 0.6180339887498949 * b) % 1.0) + 0.5) for b in range(case["B"])]


def _kept(case):
    """Rows that a store keeps of each sequence's k (a padded batch: between nothing and all of them)."""
    k = case["k"]
    return [k if b == 0 else int((k + 1) * ((0.91 + 0.7548776662466927 * b) % 1.0)) for b in range(case["B"])]


def work(case):
    op = case["op"]
    groups = lambda n: -(-n // GROUP)  # noqa: E731
    if op == "rmsnorm":
        M, K = case["M"], case["K"]
        read = M * K * 2 * (2 if case["residual"] else 1) + K * 2
        return {"bytes": read + M * K * (1 + (2 if case["residual"] else 0)) + M * groups(K) * 4, "flops": 5 * M * K}
    if op == "quantize":
        M, K = case["M"], case["K"]
        return {"bytes": M * K * (5 if case["gated"] else 3) + M * groups(K) * 4, "flops": (8 if case["gated"] else 3) * M * K}
    if op == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        return {"bytes": M * K + M * groups(K) * 4 + N * K + groups(N) * groups(K) * 4 + M * N * 2 * (2 if case["residual"] else 1),
                "flops": 2 * M * N * K}
    if op == "attention":
        B, k, Hq, Hkv, D = (case[x] for x in ("B", "k", "Hq", "Hkv", "D"))
        n = _lengths(case)
        full = sum(x // PAGE for x in n)
        tail = sum(x % PAGE for x in n)
        bytes_ = full * Hkv * (2 * PAGE * D + 8) + (tail + B * k) * Hkv * D * 4 + 2 * B * k * Hq * D * 2
        pairs = k * (k + 1) // 2 if case["mask"] == "causal" else k * k
        return {"bytes": bytes_, "flops": 4 * D * Hq * (k * sum(n) + B * pairs)}
    B, Hkv, D = case["B"], case["Hkv"], case["D"]
    rows = old = pages = rest = 0
    for n, keep in zip(_lengths(case), _kept(case)):
        sealed = (n + keep) // PAGE - n // PAGE
        rows, pages = rows + keep, pages + sealed
        old += n % PAGE if sealed else 0
        rest += (n + keep) % PAGE if sealed else keep
    return {"bytes": 2 * Hkv * (D * 2 * (rows + old) + pages * (PAGE * D + 4) + rest * D * 2), "flops": 6 * Hkv * D * (rows + old)}


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------

def _codes(v, amax):
    s = (amax / E4M3_MAX).clamp_min(SCALE_MIN)
    return (v / s).to(torch.float8_e4m3fn), s


def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)


def _rows_in_codes(v):
    """e4m3 codes of fp32 rows and their scales, one per 128 columns."""
    M, K = v.shape
    G = -(-K // GROUP)
    w = torch.nn.functional.pad(v, (0, G * GROUP - K)).view(M, G, GROUP)
    q, s = _codes(w, w.abs().amax(dim=2, keepdim=True))
    return q.view(M, G * GROUP)[:, :K].contiguous(), s.view(M, G)


def _cache(case, gen, room):
    """A paged cache in 8 bits: pages in random order, each sequence with its prefix and `room` tokens of mapped pages."""
    B, Hkv, D = case["B"], case["Hkv"], case["D"]
    n = _lengths(case)
    mapped = [-(-(x + room) // PAGE) + 1 for x in n]
    width, total = max(mapped), sum(mapped) + 8
    order = torch.randperm(total, generator=gen, device="cuda").to(torch.int32)
    at = torch.zeros(B, dtype=torch.int64)
    at[1:] = torch.tensor(mapped, dtype=torch.int64).cumsum(0)[:-1]
    idx = torch.arange(width)[None, :] + at[:, None]
    held = torch.arange(width)[None, :] < torch.tensor(mapped)[:, None]
    table = torch.where(held.cuda(), order[idx.clamp_max(total - 1).cuda()], -1).to(torch.int32).contiguous()
    state = {"page_table": table, "seq_len": torch.tensor(n, dtype=torch.int32, device="cuda"),
             "n_pages": torch.tensor(mapped, dtype=torch.int32, device="cuda"),
             "free_stack": order.flip(0).contiguous(), "free_top": torch.tensor([total - sum(mapped)], dtype=torch.int32, device="cuda"),
             "seq_ids": torch.arange(B, dtype=torch.int32, device="cuda")}
    # keys with a spread of channel magnitudes, as rotary and per-head norms leave them; values without
    spread = torch.exp(0.4 * _normal(gen, 1, Hkv, 1, D))
    for name, mag in (("k", spread), ("v", 1.0)):
        pool, scale = [], []
        for p in range(0, total, 4096):
            v = _normal(gen, min(4096, total - p), Hkv, PAGE, D) * mag
            q, s = _codes(v, v.abs().amax(dim=(2, 3), keepdim=True))
            pool.append(q)
            scale.append(s.view(-1, Hkv))
        state[name + "_pool"], state[name + "_scale"] = torch.cat(pool), torch.cat(scale)
        state[name + "_tail"] = (_normal(gen, B, Hkv, TAIL, D) * mag).to(torch.bfloat16)
    state["spread"] = spread.view(1, 1, Hkv, D)
    return state


def _with_handle(state):
    """The library's handle over the cache's tensors, which a program makes once."""
    from paper_2512_15176_b200 import binding as L
    names = ("k_pool", "v_pool", "k_scale", "v_scale", "k_tail", "v_tail", "page_table", "seq_len", "n_pages", "free_stack", "free_top")
    state["kv"] = L.KVCacheQuant(*(state[x] for x in names))
    return state


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    op = case["op"]
    bf = torch.bfloat16
    if op in ("rmsnorm", "quantize"):
        M, K = case["M"], case["K"]
        G = -(-K // GROUP)
        state = {"codes": torch.empty(M, K, dtype=torch.float8_e4m3fn, device="cuda"), "scales": torch.empty(M, G, device="cuda")}
        if op == "rmsnorm":
            x = _normal(gen, M, K)
            x[:, ::97] *= 20.0                                   # a residual stream has a few channels far above the rest
            state["x"] = x.to(bf)
            state["gamma"] = (1.0 + 0.3 * _normal(gen, K)).to(bf)
            state["residual"] = _normal(gen, M, K).to(bf) if case["residual"] else None
            state["sum"] = torch.empty(M, K, dtype=bf, device="cuda") if case["residual"] else None
        else:
            state["x"] = (1.5 * _normal(gen, M, 2 * K if case["gated"] else K)).to(bf)
    elif op == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        state = {}
        state["x"], state["x_scale"] = _rows_in_codes(_normal(gen, M, K))
        Gn, Gk = -(-N // GROUP), -(-K // GROUP)
        w = torch.zeros(Gn * GROUP, Gk * GROUP, device="cuda")
        w[:N, :K] = _normal(gen, N, K) / math.sqrt(K)
        w = w.view(Gn, GROUP, Gk, GROUP)
        q, s = _codes(w, w.abs().amax(dim=(1, 3), keepdim=True))
        state["w"] = q.view(Gn * GROUP, Gk * GROUP)[:N, :K].contiguous()
        state["w_scale"] = s.view(Gn, Gk).contiguous()
        state["residual"] = _normal(gen, M, N).to(bf) if case["residual"] else None
        state["y"] = torch.empty(M, N, dtype=bf, device="cuda")
    elif op == "attention":
        B, k, Hq, Hkv, D = (case[x] for x in ("B", "k", "Hq", "Hkv", "D"))
        state = _cache(case, gen, k)
        state["q"] = _normal(gen, B, k, Hq, D).to(bf)
        state["k_blk"] = (_normal(gen, B, k, Hkv, D) * state["spread"]).to(bf)
        state["v_blk"] = _normal(gen, B, k, Hkv, D).to(bf)
        state["out"] = torch.empty(B, k, Hq, D, dtype=bf, device="cuda")
        # a drafter's block after some iterations: rows still masked (1), decoded (0), absent (-1)
        draws = torch.rand(B, k, generator=gen, device="cuda")
        state["row_state"] = (1 - (draws < 0.6).int() - (draws < 0.2).int()).to(torch.int32) if case["mask"] == "states" else None
        state["max_len"] = max(_lengths(case))
        if own:
            from paper_2512_15176_b200 import binding as L
            need = L.deer_block_attn_quant_workspace_bytes(B, k, Hq, Hkv, D, state["max_len"])
            state["ws"] = torch.empty(max(16, need), dtype=torch.uint8, device="cuda")
            _with_handle(state)
    else:
        B, k, Hkv, D = (case[x] for x in ("B", "k", "Hkv", "D"))
        state = _cache(case, gen, k)
        state["k_rows"] = (_normal(gen, B, k, Hkv, D) * state["spread"]).to(bf)
        state["v_rows"] = _normal(gen, B, k, Hkv, D).to(bf)
        state["keep"] = torch.tensor(_kept(case), dtype=torch.int32, device="cuda")
        if own:
            _with_handle(state)
    state["case"] = dict(case)
    return state


# ---------------------------------------------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------------------------------------------

def _rmsnorm(s):
    h = s["x"].float()
    if s["residual"] is not None:
        h = h + s["residual"].float()
    y = h * torch.rsqrt(h.square().mean(dim=1, keepdim=True) + 1e-6) * s["gamma"].float()
    q, sc = _rows_in_codes(y)
    return (q, sc, h.to(torch.bfloat16)) if s["residual"] is not None else (q, sc)


def _quantize(s):
    x = s["x"].float()
    if s["case"]["gated"]:
        K = s["case"]["K"]
        g = x[:, :K]
        x = g / (1.0 + torch.exp(-g)) * x[:, K:]
    return _rows_in_codes(x)


def _linear(s):
    M, K = s["x"].shape
    N = s["w"].shape[0]
    x = s["x"].float() * s["x_scale"].repeat_interleave(GROUP, dim=1)[:, :K]
    w = s["w"].float() * s["w_scale"].repeat_interleave(GROUP, dim=0)[:N].repeat_interleave(GROUP, dim=1)[:, :K]
    y = x @ w.t()
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return y.to(torch.bfloat16)


def _block_mask(case, row_state, B, k):
    """[B][k][k]: which block rows each block row sees."""
    i = torch.arange(k, device="cuda")
    if case["mask"] == "causal":
        return (i[None, :] <= i[:, None]).expand(B, k, k)
    if row_state is None:
        return torch.ones(B, k, k, dtype=torch.bool, device="cuda")
    of, by = row_state[:, None, :], row_state[:, :, None]
    return ((by == 1) & (of >= 0)) | ((by == 0) & (of == 0))


def _attention(s):
    c = s["case"]
    B, k, Hq, Hkv, D = (c[x] for x in ("B", "k", "Hq", "Hkv", "D"))
    n = s["seq_len"].long()
    P = s["max_len"] // PAGE
    pages = s["page_table"][:, :P].long()
    keys, vals = [], []
    i = torch.arange(PAGE, device="cuda")
    at = ((n // PAGE) % 3)[:, None] * PAGE + i[None, :]                       # where the partly filled page lives in the tail
    for name, out in (("k", keys), ("v", vals)):
        pool = s[name + "_pool"].view(torch.uint8)[pages].view(torch.float8_e4m3fn).float() * s[name + "_scale"][pages][..., None, None]
        out.append(pool.permute(0, 2, 1, 3, 4).reshape(B, Hkv, P * PAGE, D))
        out.append(torch.gather(s[name + "_tail"], 2, at[:, None, :, None].expand(B, Hkv, PAGE, D)).float())
        out.append(s[name + "_blk"].float().permute(0, 2, 1, 3))
    K, V = torch.cat(keys, 2), torch.cat(vals, 2)
    seen = torch.cat([(torch.arange(P * PAGE, device="cuda")[None, :] < (n // PAGE * PAGE)[:, None]), i[None, :] < (n % PAGE)[:, None]], 1)
    seen = torch.cat([seen[:, None, :].expand(B, k, -1), _block_mask(c, s["row_state"], B, k)], 2)     # [B][k][keys]
    if s["row_state"] is not None:
        seen = seen & (s["row_state"] >= 0)[:, :, None]
    G = Hq // Hkv
    q = s["q"].float().view(B, k, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, k * G, D)
    z = (q @ K.transpose(2, 3)).view(B, Hkv, k, G, -1) / math.sqrt(D)
    z = z.masked_fill(~seen[:, None, :, None, :], -math.inf)
    top = z.amax(dim=-1, keepdim=True).clamp_min(-3.0e38)                     # an absent row sees nothing and gives zeros
    p = torch.exp(z - top)
    total = p.sum(dim=-1, keepdim=True)
    o = (p.view(B, Hkv, k * G, -1) @ V).view(B, Hkv, k, G, D) / total.clamp_min(1e-30)
    return o.permute(0, 2, 1, 3, 4).reshape(B, k, Hq, D).to(torch.bfloat16)


def _store(s):
    c = s["case"]
    B, k, Hkv, D = (c[x] for x in ("B", "k", "Hkv", "D"))
    n, end = s["seq_len"].long()[:, None], (s["seq_len"] + s["keep"]).long()[:, None]
    P = (k + PAGE - 1) // PAGE + 1                                            # pages that k rows can touch
    page = n // PAGE + torch.arange(P, device="cuda")[None, :]                # [B][P]
    t = n // PAGE * PAGE + torch.arange(P * PAGE, device="cuda")[None, :]     # [B][P * 16] token positions
    full = ((page + 1) * PAGE <= end)
    ids = torch.gather(s["page_table"].long(), 1, page.clamp_max(s["page_table"].shape[1] - 1))
    ids = torch.where(full, ids, ids.new_zeros(()))
    slot = (t // PAGE % 3) * PAGE + t % PAGE
    new = (t >= n) & (t < end) & (t >= end // PAGE * PAGE)                    # rows that end up in the tail
    # pages that do not become full, and rows that do not go to the tail, land in one spare row behind the buffers
    where = torch.where(full, ids, s["k_pool"].shape[0])
    row = torch.where(new, slot, TAIL)
    b = torch.arange(B, device="cuda")[:, None]
    for name in ("k", "v"):
        tail, rows = s[name + "_tail"], s[name + "_rows"]
        old = torch.gather(tail, 2, slot[:, None, :, None].expand(B, Hkv, P * PAGE, D))
        put = torch.gather(rows, 1, (t - n).clamp(0, k - 1)[:, :, None, None].expand(B, P * PAGE, Hkv, D)).permute(0, 2, 1, 3)
        v = torch.where((t < n)[:, None, :, None], old, put)                  # [B][Hkv][P * 16][D]
        pages = v.view(B, Hkv, P, PAGE, D).permute(0, 2, 1, 3, 4).float()
        q, sc = _codes(pages, pages.abs().amax(dim=(3, 4), keepdim=True))
        pool = torch.cat([s[name + "_pool"].view(torch.uint8), torch.zeros(1, Hkv, PAGE, D, dtype=torch.uint8, device="cuda")])
        pool[where] = q.view(torch.uint8)
        scale = torch.cat([s[name + "_scale"], torch.zeros(1, Hkv, device="cuda")])
        scale[where] = sc.view(B, P, Hkv)
        longer = torch.cat([tail, torch.zeros(B, Hkv, 1, D, dtype=tail.dtype, device="cuda")], 2)
        longer[b, :, row] = v.permute(0, 2, 1, 3)
        s[name + "_pool"].copy_(pool[:-1].view(torch.float8_e4m3fn))
        s[name + "_scale"].copy_(scale[:-1])
        tail.copy_(longer[:, :, :TAIL])
    return [s[x] for x in ("k_pool", "v_pool", "k_scale", "v_scale", "k_tail", "v_tail")]


def _own(s):
    from paper_2512_15176_b200 import binding as L
    c = s["case"]
    op = c["op"]
    if op == "rmsnorm":
        L.deer_rmsnorm_quant(s["x"], s["gamma"], s["codes"], s["scales"], 1e-6, residual=s["residual"], total=s["sum"])
        return (s["codes"], s["scales"], s["sum"]) if s["residual"] is not None else (s["codes"], s["scales"])
    if op == "quantize":
        L.deer_quantize(s["x"], s["codes"], s["scales"], gated=c["gated"])
        return s["codes"], s["scales"]
    if op == "linear":
        L.deer_linear_quant(s["x"], s["x_scale"], s["w"], s["w_scale"], s["y"], residual=s["residual"])
        return s["y"]
    if op == "attention":
        L.deer_block_attn_quant(s["kv"], s["seq_ids"], s["q"], s["k_blk"], s["v_blk"], s["out"], s["row_state"],
                                L.DEER_MASK_CAUSAL if c["mask"] == "causal" else L.DEER_MASK_BIDIR, 1.0 / math.sqrt(c["D"]),
                                s["max_len"], s["ws"])
        return s["out"]
    L.deer_kv_store(s["kv"], s["seq_ids"], s["k_rows"], s["v_rows"], s["keep"])
    return [s[x] for x in ("k_pool", "v_pool", "k_scale", "v_scale", "k_tail", "v_tail")]


def run(state):
    if own:
        return _own(state)
    return {"rmsnorm": _rmsnorm, "quantize": _quantize, "linear": _linear, "attention": _attention, "store": _store}[state["case"]["op"]](state)


# ---------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------

def _nearest_e4m3(v):
    """The e4m3 value nearest to each fp64 value (halves to the even code): steps of 2^(e - 3), of 2^-9 below 2^-6."""
    e = torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6)))
    step = torch.exp2(e - 3.0)
    return (torch.round(v / step) * step).clamp(-E4M3_MAX, E4M3_MAX)


def _groups_exact(y):
    M, K = y.shape
    codes, scales = torch.zeros_like(y), []
    for c in range(0, K, GROUP):
        part = y[:, c:c + GROUP]
        s = torch.clamp(part.abs().max(dim=1).values / E4M3_MAX, min=SCALE_MIN)
        codes[:, c:c + GROUP] = _nearest_e4m3(part / s[:, None])
        scales.append(s)
    return codes, torch.stack(scales, 1)


def _deq(codes, scale):
    return codes.double() * scale.double()


def exact(case, seed):
    global own
    was, own = own, False                                        # inputs only: no handle, no workspace
    try:
        s = prepare(case, seed)
    finally:
        own = was
    op = case["op"]
    if op == "rmsnorm":
        h = s["x"].double() + (s["residual"].double() if s["residual"] is not None else 0.0)
        y = h / torch.sqrt((h * h).sum(1, keepdim=True) / h.shape[1] + 1e-6) * s["gamma"].double()
        q, sc = _groups_exact(y)
        return (q, sc, h) if s["residual"] is not None else (q, sc)
    if op == "quantize":
        x = s["x"].double()
        if case["gated"]:
            g, u = x.chunk(2, dim=1)
            x = g * torch.sigmoid(g) * u
        return _groups_exact(x)
    if op == "linear":
        M, K, N = case["M"], case["K"], case["N"]
        y = torch.zeros(M, N, dtype=torch.float64, device="cuda")
        for c in range(0, K, GROUP):
            part = s["x"][:, c:c + GROUP].double() @ s["w"][:, c:c + GROUP].double().t()
            by_col = s["w_scale"][:, c // GROUP].double().repeat_interleave(GROUP)[:N]
            y += part * s["x_scale"][:, c // GROUP].double()[:, None] * by_col[None, :]
        return y + (s["residual"].double() if s["residual"] is not None else 0.0)
    if op == "attention":
        B, k, Hq, Hkv, D = (case[x] for x in ("B", "k", "Hq", "Hkv", "D"))
        out = torch.zeros(B, k, Hq, D, dtype=torch.float64, device="cuda")
        for b, n in enumerate(_lengths(case)):
            full, rest = n // PAGE, n % PAGE
            ids = s["page_table"][b, :full].long()
            at = (full % 3) * PAGE
            kv = []
            for name in ("k", "v"):
                pages = _deq(s[name + "_pool"].view(torch.uint8)[ids].view(torch.float8_e4m3fn), s[name + "_scale"][ids][:, :, None, None])
                prefix = pages.transpose(0, 1).reshape(Hkv, full * PAGE, D)
                kv.append(torch.cat([prefix, s[name + "_tail"][b, :, at:at + rest].double(), s[name + "_blk"][b].double().transpose(0, 1)], 1))
            for i in range(k):
                if case["mask"] == "causal":
                    cols = torch.arange(k, device="cuda") <= i
                elif s["row_state"] is None:
                    cols = torch.ones(k, dtype=torch.bool, device="cuda")
                else:
                    st = s["row_state"][b]
                    cols = torch.where(st[i] == 1, st >= 0, torch.where(st[i] == 0, st == 0, torch.zeros_like(st, dtype=torch.bool)))
                bias = torch.zeros(n + k, dtype=torch.float64, device="cuda")
                bias[n:] = torch.where(cols, 0.0, -math.inf)
                q = s["q"][b, i].double().view(Hkv, Hq // Hkv, D)
                w = torch.softmax(torch.einsum("hgd,htd->hgt", q, kv[0]) / math.sqrt(D) + bias, dim=-1)
                if s["row_state"] is not None:
                    w = torch.where(s["row_state"][b, i] < 0, torch.zeros_like(w), w)
                out[b, i] = torch.einsum("hgt,htd->hgd", w, kv[1]).reshape(Hq, D)
        return out
    got = {}
    for name in ("k", "v"):
        pool, scale, tail = s[name + "_pool"].double(), s[name + "_scale"].double(), s[name + "_tail"].double()
        before = tail.clone()
        for b, (n, keep) in enumerate(zip(_lengths(case), _kept(case))):
            first, last = n // PAGE, (n + keep) // PAGE
            line = torch.cat([before[b, :, (first % 3) * PAGE:(first % 3) * PAGE + n % PAGE],
                              s[name + "_rows"][b, :keep].double().transpose(0, 1)], 1)
            if last > first:
                whole = line[:, :(last - first) * PAGE].reshape(line.shape[0], last - first, PAGE, -1).transpose(0, 1)
                sc = torch.clamp(whole.abs().amax(dim=(2, 3)) / E4M3_MAX, min=SCALE_MIN)
                ids = s["page_table"][b, first:last].long()
                pool[ids] = _nearest_e4m3(whole / sc[:, :, None, None])
                scale[ids] = sc
            left = line[:, (last - first) * PAGE:]
            tail[b, :, (last % 3) * PAGE:(last % 3) * PAGE + left.shape[1]] = left
        got[name] = (pool, scale, tail)
    return [got["k"][0], got["v"][0], got["k"][1], got["v"][1], got["k"][2], got["v"][2]]

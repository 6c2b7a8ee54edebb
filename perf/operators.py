"""A paged key-value cache as a decoding loop uses it, as cases that can be timed: new tokens go into the cache
(`kv_append_paged`), one new token of every sequence reads it and adds to the weight of each cached token
(`attn_decode_paged`), and a sequence that has grown too long keeps its heaviest tokens (`kv_evict_paged`).

Caches are BF16, or INT8 with one FP32 scale per token and KV head; pages are handed out in random order, as by an
allocator that has run for a while.
"""
import torch

own = False


def listed():
    return [
        # The new token of every sequence of a decoding batch goes into an INT8 cache: the smallest call.
        {"name": "append_int8_b64", "op": "append", "int8": True, "B": 64, "lo": 256, "hi": 2048, "new": 1, "Hkv": 8, "D": 128, "page": 16},
        # Chunks of prompts of seven sequences, some long, some a few tokens, into a BF16 cache.
        {"name": "append_bf16_prompt", "op": "append", "int8": False, "B": 7, "lo": 37, "hi": 4100, "new": 0, "Hkv": 8, "D": 128, "page": 64},
        # The same into an INT8 cache.
        {"name": "append_int8_prompt", "op": "append", "int8": True, "B": 7, "lo": 37, "hi": 4100, "new": 0, "Hkv": 8, "D": 128, "page": 16},
        # One sequence at the start of its answer: latency counts.
        {"name": "attn_bf16_b1", "op": "attn", "int8": False, "B": 1, "lo": 1001, "hi": 1001, "Hq": 32, "Hkv": 8, "D": 128, "Dv": 128, "page": 16, "weights": False},
        # A batch of sequences of mixed lengths, BF16 pages, weights of the tokens kept for eviction.
        {"name": "attn_bf16_b32", "op": "attn", "int8": False, "B": 32, "lo": 2048, "hi": 8192, "Hq": 32, "Hkv": 8, "D": 128, "Dv": 128, "page": 16, "weights": True},
        # The same batch on an INT8 cache.
        {"name": "attn_int8_b32", "op": "attn", "int8": True, "B": 32, "lo": 2048, "hi": 8192, "Hq": 32, "Hkv": 8, "D": 128, "Dv": 128, "page": 16, "weights": True},
        # Eight query heads to a KV head, shorter sequences, INT8 pages, no weights wanted.
        {"name": "attn_int8_b24_g8", "op": "attn", "int8": True, "B": 24, "lo": 512, "hi": 4096, "Hq": 64, "Hkv": 8, "D": 128, "Dv": 128, "page": 16, "weights": False},
        # Two very long contexts: the split over the length carries everything.
        {"name": "attn_bf16_long_b2", "op": "attn", "int8": False, "B": 2, "lo": 100003, "hi": 131072, "Hq": 32, "Hkv": 8, "D": 128, "Dv": 128, "page": 64, "weights": True},
        # Many short conversations, a head of its own for every query head, heads of 80; some sequences are empty.
        {"name": "attn_bf16_mha_d80", "op": "attn", "int8": False, "B": 48, "lo": 0, "hi": 1500, "Hq": 16, "Hkv": 16, "D": 80, "Dv": 80, "page": 32, "weights": True},
        # A batch whose caches are cut to a quarter of the longest: the ordinary eviction, INT8.
        {"name": "evict_int8_b32", "op": "evict", "int8": True, "B": 32, "lo": 2048, "hi": 8192, "Hkv": 8, "D": 128, "page": 16, "budget": 2048, "recent": 256, "sinks": 4},
        # A few tokens over the budget, every few steps: the smallest one.
        {"name": "evict_bf16_b4", "op": "evict", "int8": False, "B": 4, "lo": 900, "hi": 1088, "Hkv": 8, "D": 128, "page": 16, "budget": 1024, "recent": 128, "sinks": 4},
        # A long document cut to an eighth, right after its prompt.
        {"name": "evict_bf16_long_b1", "op": "evict", "int8": False, "B": 1, "lo": 131072, "hi": 131072, "Hkv": 8, "D": 128, "page": 64, "budget": 16384, "recent": 1024, "sinks": 4},
    ]


def _log(rng, lo, hi):
    """A size between lo and hi, spread over its logarithm."""
    return min(hi, max(lo, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    op = rng.choice(["append", "attn", "attn", "evict"])
    case = {"op": op, "int8": rng.random() < 0.5, "Hkv": rng.choice([1, 2, 4, 8, 16]), "D": rng.choice([64, 80, 96, 128, 128, 128, 192, 256]),
            "page": rng.choice([8, 16, 16, 20, 32, 64, 128])}
    # no more tokens than 480 MB of keys and values hold
    most = int(480e6 / (case["Hkv"] * 2 * case["D"] * 2))
    B = _log(rng, 1, 128)
    hi = _log(rng, 64, max(65, min(131072, 2 * most // (B + 1), most // B * 2)))
    hi = max(1, min(hi, most // B))
    case.update(B=B, hi=hi, lo=int(hi * rng.choice([0.0, 0.1, 0.25, 0.5, 1.0])))
    if op == "append":
        case["new"] = rng.choice([0, 1, 1, 3])
        case["lo"] = max(case["lo"], case["new"])
        case["hi"] = max(case["hi"], case["lo"])
    elif op == "attn":
        case["Hq"] = case["Hkv"] * rng.choice([1, 2, 4, 5, 7, 8, 16, 20])
        case["Dv"] = rng.choice([case["D"], case["D"], 64])
        case["weights"] = rng.random() < 0.6
    else:
        case["budget"] = max(1, int(hi * rng.uniform(0.1, 1.1)))
        case["sinks"] = min(4, case["budget"] // 4)
        case["recent"] = int(case["budget"] * rng.choice([0.0, 0.1, 0.5]))
    return case


# ---- sizes that follow from a case alone ------------------------------------------------------------------------------------
def _lengths(case):
    """Lengths of the sequences, from lo to hi in even steps (which sequence has which goes by the seed)."""
    B, lo, hi = case["B"], case["lo"], case["hi"]
    return [hi if B == 1 else lo + (hi - lo) * i // (B - 1) for i in range(B)]


def _element(case):
    return 1 if case["int8"] else 2


def work(case):
    L, Hkv, D, e = _lengths(case), case["Hkv"], case["D"], _element(case)
    scales = 8 if case["int8"] else 0
    if case["op"] == "append":
        n = sum(L) if case["new"] == 0 else case["B"] * case["new"]
        return {"bytes": n * Hkv * (2 * D * 2 + 2 * D * e + scales), "flops": 0}
    if case["op"] == "attn":
        Dv, Hq = case["Dv"], case["Hq"]
        n = sum(L) * Hkv * ((D + Dv) * e + scales + (8 if case["weights"] else 0)) + case["B"] * Hq * (D + Dv) * 2
        return {"bytes": n, "flops": 2 * sum(L) * Hq * (D + Dv)}
    kept = sum(min(v, case["budget"]) for v in L)
    return {"bytes": sum(L) * Hkv * 4 + kept * Hkv * (2 * (2 * D * e + scales) + 8), "flops": 0}


# ---- what a serving program has in hand -----------------------------------------------------------------------------------
def _quantised(g, shape):
    """Codes of N(0,1) rows with one scale each, as they stand in an INT8 cache."""
    codes = torch.empty(shape, dtype=torch.int8, device="cuda")
    scale = torch.empty(shape[:-1], device="cuda")
    step = max(1, (1 << 27) // (shape[1] * shape[2] * shape[3]))
    for i in range(0, shape[0], step):
        x = torch.randn((min(step, shape[0] - i),) + shape[1:], generator=g, device="cuda")
        s = x.abs().amax(-1) / 127.0
        scale[i:i + step] = s
        codes[i:i + step] = torch.round(x / s[..., None]).clamp_(-127, 127).to(torch.int8)
    return codes, scale


def _pool(g, case, blocks, D):
    shape = (blocks, case["page"], case["Hkv"], D)
    if case["int8"]:
        return _quantised(g, shape)
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.bfloat16), None


def _table(perm, need, first=0):
    """Block table [B, most blocks] of sequences that need so many blocks each, from a permutation; -1 where there is none."""
    B, width = len(need), max(1, max(need))
    table = torch.full((B, width), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n] + first
        at += n
    return table.cuda()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    c = torch.Generator()
    c.manual_seed(seed)
    B, Hkv, D, page = case["B"], case["Hkv"], case["D"], case["page"]
    Dv = case.get("Dv", D)
    L = torch.tensor(_lengths(case))[torch.randperm(B, generator=c)].tolist()
    need = [(v + page - 1) // page for v in L]
    used = sum(need)
    st = {"op": case["op"], "max_seqlen": max(L)}
    more = 3                                      # pages that belong to nobody
    if case["op"] == "evict":
        kept = [min(v, case["budget"]) for v in L]
        new_need = [(v + page - 1) // page for v in kept]
        st["first_dst"] = used + more
        st["dst_table"] = _table(torch.randperm(sum(new_need), generator=c).int(), new_need, used + more)
        more += sum(new_need)
    st["k"], st["k_scale"] = _pool(g, case, used + more, D)
    st["v"], st["v_scale"] = _pool(g, case, used + more, Dv)
    st["table"] = _table(torch.randperm(used, generator=c).int(), need)
    st["seqlens"] = torch.tensor(L, dtype=torch.int32, device="cuda")
    ld = max(1, max(L))
    if case["op"] == "append":
        new = L if case["new"] == 0 else [case["new"]] * B
        cu = [0]
        for n in new:
            cu.append(cu[-1] + n)
        st["cu_new"] = torch.tensor(cu, dtype=torch.int32, device="cuda")
        st["k_new"] = torch.randn((cu[-1], Hkv, D), generator=g, device="cuda", dtype=torch.bfloat16)
        st["v_new"] = torch.randn((cu[-1], Hkv, D), generator=g, device="cuda", dtype=torch.bfloat16)
    elif case["op"] == "attn":
        st["q"] = torch.randn((B, case["Hq"], D), generator=g, device="cuda", dtype=torch.bfloat16)
        st["scale"] = D ** -0.5
        # what earlier tokens have added so far, of the size of what this one adds
        st["weights"] = torch.rand((B, Hkv, ld), generator=g, device="cuda").mul_(case["Hq"] / (Hkv * ld)) if case["weights"] else None
    else:
        # accumulated weights: few tokens carry most, many ties at zero where a token was never looked at
        w = torch.randn((B, Hkv, ld), generator=g, device="cuda").mul_(2.0).exp_()
        st["weights"] = torch.where(torch.rand((B, Hkv, ld), generator=g, device="cuda") < 0.1, 0.0, w)
        st["budget"], st["recent"], st["sinks"] = case["budget"], case["recent"], case["sinks"]
        st["new_weights"] = torch.zeros((B, Hkv, case["budget"]), device="cuda")
        st["kept"] = torch.zeros((B, Hkv, case["budget"]), dtype=torch.int32, device="cuda")
        st["new_seqlens"] = torch.zeros(B, dtype=torch.int32, device="cuda")
    return st


# ---- the plain forms ------------------------------------------------------------------------------------------------------------
def _append_plain(st):
    cu, L, table, page = st["cu_new"].long(), st["seqlens"].long(), st["table"].long(), st["k"].shape[1]
    n = st["k_new"].shape[0]
    i = torch.arange(n, device="cuda")
    b = torch.searchsorted(cu, i, right=True) - 1
    pos = L[b] - cu[b + 1] + i
    block, slot = table[b, pos // page], pos % page
    for new, pool, scale in ((st["k_new"], st["k"], st["k_scale"]), (st["v_new"], st["v"], st["v_scale"])):
        if scale is None:
            pool[block, slot] = new
        else:
            x = new.float()
            m = x.abs().amax(-1)
            s = m / torch.full_like(m, 127.0)
            pool[block, slot] = torch.round(x / torch.where(s > 0, s, 1.0)[..., None]).clamp(-127, 127).to(torch.int8)
            scale[block, slot] = s
    # codes are whole numbers that follow from IEEE arithmetic alone: they have to be equal
    return [st["k"], st["v"], st["k_scale"], st["v_scale"]]


def _rows(pool, scale, table):
    """The rows of all sequences in order, FP32: [B, positions, Hkv, D]."""
    pages = table.clamp(min=0).long()
    x = pool[pages].float()
    if scale is not None:
        x = x * scale[pages][..., None]
    return x.reshape(table.shape[0], -1, pool.shape[2], pool.shape[3])


def _attn_plain(st):
    q, L = st["q"].float(), st["seqlens"].long()
    B, Hq, D = q.shape
    k = _rows(st["k"], st["k_scale"], st["table"])
    n, Hkv = k.shape[1], k.shape[2]
    seen = torch.arange(n, device="cuda")[None, :] < L[:, None]
    s = torch.matmul(q.view(B, Hkv, Hq // Hkv, D), k.permute(0, 2, 3, 1)) * st["scale"]
    del k
    s = torch.where(seen[:, None, None, :], s, float("-inf"))
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(m == float("-inf"), 0.0, m))
    total = p.sum(-1, keepdim=True)
    p = p / torch.where(total > 0, total, 1.0)
    v = torch.where(seen[:, :, None, None], _rows(st["v"], st["v_scale"], st["table"]), 0.0)
    out = torch.matmul(p, v.permute(0, 2, 1, 3)).reshape(B, Hq, -1).to(torch.bfloat16)
    if st["weights"] is None:
        return [out]
    ld = st["weights"].shape[2]
    st["weights"] += p.sum(2)[:, :, :ld]
    return [out, st["weights"]]


def _evict_plain(st):
    w, L, budget = st["weights"], st["seqlens"].long(), st["budget"]
    B, Hkv, n = w.shape
    pos = torch.arange(n, device="cuda")
    seen = pos[None, :] < L[:, None]
    safe = seen & ((pos[None, :] < st["sinks"]) | (pos[None, :] >= L[:, None] - st["recent"]))
    # by weight, then (stable) the protected ones first and what is not there last
    by_weight = torch.sort(w, dim=-1, descending=True, stable=True).indices
    group = torch.where(safe, 0, torch.where(seen, 1, 2))[:, None, :].expand(B, Hkv, n)
    order = by_weight.gather(-1, torch.sort(group.gather(-1, by_weight), dim=-1, stable=True).indices)
    new = L.clamp(max=budget)
    rank = torch.arange(min(budget, n), device="cuda")
    there = (rank[None, :] < new[:, None])[:, None, :]
    kept = torch.sort(torch.where(there, order[..., :min(budget, n)], n), dim=-1).values
    there = there.expand_as(kept)
    b, h, r = there.nonzero(as_tuple=True)
    src = kept[b, h, r]
    page = st["k"].shape[1]
    block, slot = st["table"].long()[b, src // page], src % page
    to_block, to_slot = st["dst_table"].long()[b, r // page], r % page
    for pool in (st["k"], st["v"], st["k_scale"], st["v_scale"]):
        if pool is not None:
            pool[to_block, to_slot, h] = pool[block, slot, h]
    st["kept"][b, h, r] = src.int()
    st["new_weights"][b, h, r] = w[b, h, src]
    st["new_seqlens"].copy_(new)
    return _evicted(st)


def _evicted(st):
    """The pages that the kept tokens went to, and what belongs to them."""
    first = st["first_dst"]
    pools = [None if st[x] is None else st[x][first:] for x in ("k", "v", "k_scale", "v_scale")]
    return pools + [st["new_seqlens"], st["new_weights"], st["kept"]]


# ---- the pass ---------------------------------------------------------------------------------------------------------------------
def run(st):
    if not own:
        return {"append": _append_plain, "attn": _attn_plain, "evict": _evict_plain}[st["op"]](st)
    from paper_2605_13915_b200 import binding as msd
    k, v, ks, vs, table, L = st["k"], st["v"], st["k_scale"], st["v_scale"], st["table"], st["seqlens"]
    if st["op"] == "append":
        msd.kv_append_paged(st["k_new"], st["v_new"], k, v, ks, vs, table, L, st["cu_new"])
        return [k, v, ks, vs]
    if st["op"] == "attn":
        if "ws" not in st:      # a serving program keeps its workspace and output buffer
            B, Hq, _ = st["q"].shape
            w = st["weights"]
            st["ws"] = msd.workspace(msd.attn_decode_paged_workspace_bytes(B, Hq, k.shape[2], v.shape[3], 0 if w is None else w.shape[2]))
            st["out"] = torch.empty((B, Hq, v.shape[3]), dtype=torch.bfloat16, device="cuda")
        msd.attn_decode_paged(st["q"], k, v, ks, vs, table, L, st["scale"], weights=st["weights"], ws=st["ws"], out=st["out"])
        return [st["out"]] if st["weights"] is None else [st["out"], st["weights"]]
    msd.kv_evict_paged(k, v, ks, vs, table, L, st["weights"], st["budget"], st["dst_table"], recent=st["recent"], sinks=st["sinks"],
                       new_seqlens=st["new_seqlens"], new_weights=st["new_weights"], kept=st["kept"])
    return _evicted(st)


# ---- from the definitions, in 64 bits, a sequence at a time --------------------------------------------------------------------
def _sequence(pool, scale, blocks, L):
    x = pool[blocks].double()
    if scale is not None:
        x = x * scale[blocks].double().unsqueeze(-1)
    return x.flatten(0, 1)[:L]


def exact(case, seed):
    st = prepare(case, seed)
    page, L = case["page"], st["seqlens"].tolist()
    if case["op"] == "append":
        if not case["int8"]:
            k, v = st["k"].double(), st["v"].double()
        else:
            k, v = st["k_scale"].double(), st["v_scale"].double()
        cu = st["cu_new"].tolist()
        for b, n in enumerate(L):
            pos = torch.arange(n - (cu[b + 1] - cu[b]), n, device="cuda")
            block, slot = st["table"][b][pos // page].long(), pos % page
            for to, new in ((k, st["k_new"]), (v, st["v_new"])):
                x = new[cu[b]:cu[b + 1]].double()
                to[block, slot] = x.abs().amax(-1) / 127.0 if case["int8"] else x
        return [None, None, k, v] if case["int8"] else [k, v, None, None]
    if case["op"] == "attn":
        B, Hq, D = st["q"].shape
        G = Hq // case["Hkv"]
        out = torch.zeros((B, Hq, case["Dv"]), dtype=torch.float64, device="cuda")
        weights = None if st["weights"] is None else st["weights"].double()
        for b, n in enumerate(L):
            if n == 0:
                continue
            blocks = st["table"][b, :(n + page - 1) // page].long()
            k, v = _sequence(st["k"], st["k_scale"], blocks, n), _sequence(st["v"], st["v_scale"], blocks, n)
            for h in range(case["Hkv"]):
                heads = slice(h * G, (h + 1) * G)
                p = torch.softmax(st["q"][b, heads].double() @ k[:, h].T * st["scale"], dim=-1)
                out[b, heads] = p @ v[:, h]
                if weights is not None:
                    weights[b, h, :n] += p.sum(0)
        return [out] if weights is None else [out, weights]
    first = st["first_dst"]
    pools = [st["k"], st["v"], st["k_scale"], st["v_scale"]]
    pools = [None if x is None or x.dtype == torch.int8 else x.double() for x in pools]
    new_weights = st["new_weights"].double()
    for b, n in enumerate(L):
        for h in range(case["Hkv"]):
            w = st["weights"][b, h, :n].double()
            if n > case["budget"]:
                w[:case["sinks"]] = float("inf")
                w[n - case["recent"]:] = float("inf")
                keep = torch.sort(torch.argsort(-w, stable=True)[:case["budget"]]).values
            else:
                keep = torch.arange(n, device="cuda")
            at = torch.arange(keep.numel(), device="cuda")
            src, dst = st["table"][b][keep // page].long(), st["dst_table"][b][at // page].long()
            for x in pools:
                if x is not None:
                    x[dst, at % page, h] = x[src, keep % page, h]
            new_weights[b, h, at] = st["weights"][b, h].double()[keep]
    return [None if x is None else x[first:] for x in pools] + [None, new_weights, None]

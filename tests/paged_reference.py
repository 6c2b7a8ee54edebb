"""Paged caches for the tests, and what the operators on them should give: plain loops over sequences and heads in 64 bits."""
import torch


def make_cache(lengths, Hkv, D, Dv, page, int8=False, seed=0, layout="tokens", spare=3, poison=True, scale_of_k=1.0, device="cuda"):
    """A cache that holds `lengths` tokens of each sequence on pages in random order.  layout: "tokens" [blocks, page, heads, D],
    "heads" (the same as a view of [blocks, heads, page, D]) or "joint" (k and v side by side in one allocation).
    poison: rows that belong to no token, and pages that belong to nobody, hold NaN (BF16) or extreme codes and NaN scales (INT8)."""
    g = torch.Generator().manual_seed(seed)
    need = [(n + page - 1) // page for n in lengths]
    blocks = sum(need) + spare
    order = torch.randperm(blocks, generator=g)
    table = torch.full((len(lengths), max([1] + need)), -1, dtype=torch.int32)
    used = torch.zeros(blocks, page, dtype=torch.bool)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n].int()
        for j in range(n):
            used[order[at + j], :min(page, lengths[b] - j * page)] = True
        at += n

    def rows(width, factor):
        x = (torch.randn(blocks, page, Hkv, width, generator=g) * factor).to(torch.bfloat16)
        if not int8:
            if poison:
                x[~used] = float("nan")
            return x, None
        f = x.float()
        m = f.abs().amax(-1)
        s = m / torch.full_like(m, 127.0)
        q = torch.round(f / torch.where(s > 0, s, 1.0)[..., None]).clamp(-127, 127).to(torch.int8)
        if poison:
            q[~used] = -128
            s[~used] = float("nan")
        return q, s

    def laid_out(x):
        if layout == "heads":
            return x.to(device).permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
        return x.to(device)

    k, ks = rows(D, scale_of_k)
    v, vs = rows(Dv, 1.0)
    if layout == "joint":
        both = torch.cat([k, v], -1).to(device)
        k, v = both[..., :D], both[..., D:]
    else:
        k, v = laid_out(k), laid_out(v)
    if ks is not None:
        ks, vs = ks.to(device), vs.to(device)
        if layout == "heads":
            ks, vs = (x.permute(0, 2, 1).contiguous().permute(0, 2, 1) for x in (ks, vs))
    return {"k": k, "v": v, "k_scale": ks, "v_scale": vs, "table": table.to(device),
            "seqlens": torch.tensor(lengths, dtype=torch.int32, device=device)}


def sequence(c, b, what):
    """Rows of sequence b in order, 64 bits: [L, Hkv, width]."""
    pool, scale = c[what], c[what + "_scale"]
    page, n = pool.shape[1], int(c["seqlens"][b])
    blocks = c["table"][b, :(n + page - 1) // page].long()
    x = pool[blocks].double().flatten(0, 1)[:n]
    if scale is not None:
        x = x * scale[blocks].double().flatten(0, 1)[:n][..., None]
    return x


def attention(q, c, softmax_scale):
    """(out [B,Hq,Dv], lse [B,Hq], weights: a list of [Hkv, L], sums of p|v| [B,Hq,Dv], of |q||k| [B,Hq]: what the rounding errors go by)."""
    B, Hq, D = q.shape
    Hkv, Dv = c["k"].shape[2], c["v"].shape[3]
    G = Hq // Hkv
    out = torch.zeros(B, Hq, Dv, dtype=torch.float64, device=q.device)
    lse = torch.full((B, Hq), float("-inf"), dtype=torch.float64, device=q.device)
    mass, reach, weights = torch.zeros_like(out), torch.zeros_like(lse), []
    for b in range(B):
        n = int(c["seqlens"][b])
        w = torch.zeros(Hkv, n, dtype=torch.float64, device=q.device)
        if n:
            k, v = sequence(c, b, "k"), sequence(c, b, "v")
            for h in range(Hkv):
                heads = slice(h * G, (h + 1) * G)
                x = q[b, heads].double()
                s = x @ k[:, h].T * softmax_scale
                p = torch.softmax(s, -1)
                out[b, heads], mass[b, heads] = p @ v[:, h], p @ v[:, h].abs()
                lse[b, heads] = torch.logsumexp(s, -1)
                reach[b, heads] = (x.abs() @ k[:, h].abs().T).amax(-1) * abs(softmax_scale)
                w[h] = p.sum(0)
        weights.append(w)
    return out, lse, weights, mass, reach


def evicted(weights, n, budget, recent, sinks):
    """Positions that stay of n tokens with these weights (a list of floats), in order."""
    if n <= budget:
        return list(range(n))
    sure = set(range(min(sinks, n))) | set(range(n - recent, n))
    key = lambda j: (float("inf"), 1) if weights[j] != weights[j] else (weights[j] + 0.0, 0)      # NaN above everything
    rest = sorted((j for j in range(n) if j not in sure), key=lambda j: (-key(j)[0], -key(j)[1], j))
    return sorted(sure | set(rest[:budget - len(sure)]))

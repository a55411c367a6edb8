"""Performance cases of the operators beside the linear layers: what else a decoder layer does between its projections.

  append     keys (rotated by their positions) and values into the paged 8-bit cache, queries rotated on the way
  attention  softmax attention of the new tokens over that cache, one token a sequence or many
  lora       low-rank adapters of the requests in a batch, added to what a shared projection gave

Head counts and projections are those of the benchmark's model shapes (32 query heads on 8, 32 on 32, 64 on 8; 64 or 128
wide; N x K of the linear layers); sequence lengths and batches are generic.
"""
import math

import torch

own = False

DEV = "cuda:0"
PAGE = 64


def _append(name, heads, kv_heads, dim, seqs, new, context, interleaved=False, rot=0):
    return {"name": name, "op": "append", "heads": heads, "kv_heads": kv_heads, "dim": dim, "seqs": seqs, "new": new, "context": context,
            "interleaved": interleaved, "rot": rot or dim, "page": PAGE}


def _attention(name, heads, kv_heads, dim, seqs, new, context):
    return {"name": name, "op": "attention", "heads": heads, "kv_heads": kv_heads, "dim": dim, "seqs": seqs, "new": new, "context": context,
            "page": PAGE}


def _lora(name, M, N, K, rank, adapters, per_token):
    return {"name": name, "op": "lora", "M": M, "N": N, "K": K, "rank": rank, "adapters": adapters, "per_token": per_token}


def listed():
    return [
        # one new token of one sequence, small model: nothing but latency
        _append("append_1b_one", 32, 8, 64, 1, 1, 1000),
        # a decode step of a large batch
        _append("append_70b_batch128", 64, 8, 128, 128, 1, 4000),
        # prompts of several requests at once, ragged, each behind some cached tokens that end inside a block
        _append("append_8b_prompts", 32, 8, 128, 5, 1700, 300),
        # decoding of a single short sequence, small model
        _attention("attention_1b_one", 32, 8, 64, 1, 1, 777),
        # decoding of one very long sequence: the work has to be split along it
        _attention("attention_70b_long", 64, 8, 128, 1, 1, 130999),
        # batched decoding, ragged
        _attention("attention_8b_batch64", 32, 8, 128, 64, 1, 8000),
        # batched decoding where every query head has a key head of its own
        _attention("attention_7b_batch16", 32, 32, 128, 16, 1, 4000),
        # a few guessed tokens of each sequence checked at once
        _attention("attention_8b_verify5", 32, 8, 128, 16, -5, 8000),
        # prompts of several requests, each behind a cached prefix
        _attention("attention_8b_prompts", 32, 8, 128, 3, 2000, 3000),
        # the adapter of one token beside a fused qkv projection
        _lora("lora_70b_one", 1, 10240, 8192, 16, 8, True),
        # a decode batch in which every request may have an adapter of its own
        _lora("lora_8b_batch16", 16, 6144, 4096, 32, 48, True),
        # prompts of a few requests beside gate and up
        _lora("lora_8b_prompts", 2011, 28672, 4096, 64, 5, False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges, sizes spread over their logarithm."""
    op = rng.choice(["append", "attention", "attention", "lora"])
    if op == "lora":
        M = rng.choice([rng.randint(1, 16), _log_int(rng, 17, 2000)])
        few = M > 64
        return {"op": op, "M": M, "N": _log_int(rng, 257, 28672), "K": 64 * _log_int(rng, 8, 64 if few else 220), "rank": 8 * rng.randint(1, 8),
                "adapters": rng.randint(1, 5) if few else rng.randint(1, 48), "per_token": not few}
    heads, kv_heads = rng.choice([(32, 8), (32, 32), (64, 8), (20, 4), (12, 12), (24, 1), (7, 7), (40, 8)])
    dim = rng.choice([64, 128, 128])
    kind = rng.choice(["one", "few", "many"])
    if op == "append":
        seqs = _log_int(rng, 1, 200) if kind != "many" else rng.randint(1, 6)
        new = 1 if kind == "one" else -rng.randint(2, 9) if kind == "few" else _log_int(rng, 20, 1400)
        return {"op": op, "heads": heads, "kv_heads": kv_heads, "dim": dim, "seqs": seqs, "new": new,
                "context": _log_int(rng, 10, 4000 if kind != "many" else 800), "interleaved": rng.random() < 0.4,
                "rot": dim if rng.random() < 0.75 else dim // 2, "page": rng.choice([32, 64, 64, 128])}
    if kind == "many":
        seqs, new, context = rng.randint(1, 3), _log_int(rng, 30, 1500), _log_int(rng, 10, 3000)
        heads, kv_heads = rng.choice([(32, 8), (32, 32), (20, 4), (12, 12), (24, 1)])
    else:
        seqs = _log_int(rng, 1, 64)
        new = 1 if kind == "one" else -rng.randint(2, 8)
        context = _log_int(rng, 30, max(60, min(100000, 500000 * 8 // (seqs * kv_heads * (1 if kind == "one" else 3)))))
    return {"op": op, "heads": heads, "kv_heads": kv_heads, "dim": dim, "seqs": seqs, "new": new, "context": context,
            "page": rng.choice([32, 64, 64, 128])}


def _lengths(case):
    """New tokens and cached tokens of each sequence. `new` 1: one each; below zero: that many each; above one: prompts of up to that many."""
    r = torch.Generator().manual_seed(case["context"] * 1009 + case["seqs"] * 31 + case["new"] + 1000)
    B = case["seqs"]
    frac = torch.rand(B, generator=r)
    frac[0] = 1.0
    cached = (case["context"] * (0.35 + 0.65 * frac)).round().int().tolist()
    if case["new"] > 1:
        f = torch.rand(B, generator=r)
        f[0] = 1.0
        new = [max(1, int(round(case["new"] * x))) for x in (0.3 + 0.7 * f).tolist()]
    else:
        new = [abs(case["new"])] * B
    return new, [c + n for c, n in zip(cached, new)]


def _cache_case(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    heads, hk, D, page = case["heads"], case["kv_heads"], case["dim"], case["page"]
    new, length = _lengths(case)
    B, T = len(new), sum(new)
    blocks = [-(-n // page) for n in length]
    width, pages = max(blocks), sum(blocks) + 3
    host = torch.Generator().manual_seed(seed)
    order = torch.randperm(pages, generator=host).tolist()
    table = torch.full((B, width), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(blocks):
        table[b, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    starts = torch.tensor([0] + new, dtype=torch.int32).cumsum(0).to(torch.int32)

    def codes(std):
        out = torch.empty(pages, hk, page, D, dtype=torch.float8_e4m3fn, device=DEV)
        step = max(1, (1 << 27) // (hk * page * D))
        for i in range(0, pages, step):
            n = min(step, pages - i)
            out[i:i + n] = (torch.randn(n, hk, page, D, generator=g, device=DEV, dtype=torch.float16) * std).clamp_(-448, 448)
        return out

    def scales(lo, hi):
        return torch.exp2(torch.randint(lo, hi + 1, (pages, hk), generator=g, device=DEV).float())

    cache = {"k": codes(100.0), "v": codes(100.0), "k_scale": scales(-8, -6), "v_scale": scales(-8, -6)}
    # projections come out of one fused matrix product: q, k and v of a token lie in one row
    row = torch.randn(T, heads + 2 * hk, D, generator=g, device=DEV, dtype=torch.float16)
    # some heads attend to everything, some to a few keys; some channels of the keys are far larger than the others
    row[:, :heads] *= (0.5 + torch.arange(heads, device=DEV) % 4).half()[:, None]
    row[:, heads:heads + hk] *= 1 + 4 * (torch.rand(hk, D, generator=g, device=DEV) < 0.03).half()
    return {"case": case, "cache": cache, "row": row, "q": row[:, :heads], "k": row[:, heads:heads + hk], "v": row[:, heads + hk:],
            "starts": starts.to(DEV), "lengths": torch.tensor(length, dtype=torch.int32, device=DEV), "table": table.to(DEV),
            "max_new": max(new)}


def _scratch():
    """What a program keeps for the calls of a stream."""
    return torch.zeros(16 << 20, dtype=torch.uint8, device=DEV)


def prepare(case, seed):
    op = case["op"]
    if op == "lora":
        g = torch.Generator(device=DEV).manual_seed(seed)
        M, N, K, R, L = case["M"], case["N"], case["K"], case["rank"], case["adapters"]
        x = torch.randn(M, K, generator=g, device=DEV).half()
        a = (torch.randn(L, R, K, generator=g, device=DEV) / math.sqrt(K)).half()
        b = (torch.randn(L, N, R, generator=g, device=DEV) * 0.5).half()
        base = torch.randn(M, N, generator=g, device=DEV).half()
        if case["per_token"]:
            adapter = torch.randint(-1, L, (M,), generator=g, device=DEV, dtype=torch.int32)
            adapter[0] = seed % L
        else:   # requests one behind the other, the last of them without an adapter
            adapter = (torch.arange(M, device=DEV, dtype=torch.int32) * (L + 1) // M)
            adapter[adapter >= L] = -1
        scaling = 0.5 + torch.rand(L, generator=g, device=DEV)
        return {"case": case, "x": x, "a": a, "b": b, "base": base, "adapter": adapter, "scaling": scaling, "y": torch.empty_like(base),
                "scratch": _scratch()}
    s = _cache_case(case, seed)
    if op == "append":
        rot, n = case["rot"], s["table"].shape[1] * case["page"]
        turn = 500000.0 ** (-torch.arange(rot // 2, dtype=torch.float64, device=DEV) * 2 / rot)
        angle = torch.arange(n, dtype=torch.float64, device=DEV)[:, None] * turn
        s["rope"] = torch.stack([angle.cos(), angle.sin()], -1).float().contiguous()
    s["out"] = torch.empty(s["q"].shape, dtype=torch.float16, device=DEV)
    s["scratch"] = _scratch()
    return s


# ---- plain forms

def _rotate(x, rope, interleaved):
    """Pairs (a, b) -> (a c - b s, b c + a s) over the first dimensions of a head; rope [tokens][pairs][2], the rest stays."""
    n = 2 * rope.shape[1]
    c, s = rope[:, None, :, 0], rope[:, None, :, 1]
    if interleaved:
        a, b = x[..., 0:n:2], x[..., 1:n:2]
        y = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    else:
        a, b = x[..., :n // 2], x[..., n // 2:n]
        y = torch.cat([a * c - b * s, b * c + a * s], -1)
    return torch.cat([y, x[..., n:]], -1)


def _positions(starts, lengths, T):
    t = torch.arange(T, device=DEV, dtype=torch.int32)
    seq = torch.searchsorted(starts, t, right=True) - 1
    return (t - starts[seq + 1] + lengths[seq]).long()


def _plain_append(s):
    case, cache, rope = s["case"], s["cache"], s["rope"]
    page, T = case["page"], s["k"].shape[0]
    starts, lengths, table = s["starts"].long(), s["lengths"].long(), s["table"].long()
    here = rope[_positions(s["starts"], s["lengths"], T)]
    k, q = (_rotate(s[n].float(), here, case["interleaved"]) for n in ("k", "q"))
    # the blocks that get new tokens, padded with the last of each sequence, whose copies come out the same
    first = lengths - (starts[1:] - starts[:-1])
    width = (s["max_new"] + page - 2) // page + 1
    block = torch.minimum(first[:, None] // page + torch.arange(width, device=DEV), (lengths[:, None] - 1) // page)
    at = table.gather(1, block).reshape(-1)
    pos = block[:, :, None] * page + torch.arange(page, device=DEV)
    is_new = (pos >= first[:, None, None]) & (pos < lengths[:, None, None])
    token = torch.where(is_new, pos - first[:, None, None] + starts[:-1, None, None], 0)
    fresh = (block * page >= first[:, None]).reshape(-1, 1)
    is_old = (pos < first[:, None, None]).reshape(-1, 1, page, 1)   # slots behind a sequence's last token stay as they are
    is_new = is_new.reshape(-1, 1, page, 1)
    for name, x in (("k", k), ("v", s["v"].float())):
        codes, scale = cache[name], cache[name + "_scale"]
        x = x[token.reshape(-1, page)].permute(0, 2, 1, 3)
        top = (x * is_new).abs().amax((-1, -2))
        m, e = torch.frexp(top)
        e = torch.where(top > 0, e - 9 + (m > 0.875).int(), -40).clamp(-40, 20)
        want = torch.exp2(e.float())
        old = scale[at]
        now = torch.where(fresh, want, torch.maximum(want, old))
        held = codes[at].float()
        held = torch.where(is_old, held * (old / now)[:, :, None, None], held)
        codes[at] = torch.where(is_new, x / now[:, :, None, None], held).to(torch.float8_e4m3fn)
        scale[at] = now
    return {"k": cache["k"], "v": cache["v"], "k_scale": cache["k_scale"], "v_scale": cache["v_scale"], "q": q.half()}


def _plain_attention(s):
    case, cache = s["case"], s["cache"]
    page, hk, D, heads = case["page"], case["kv_heads"], case["dim"], case["heads"]
    starts, lengths, table = s["starts"].long(), s["lengths"].long(), s["table"].long().clamp_min(0)
    B, n, g = table.shape[0], s["max_new"], heads // hk
    S = table.shape[1] * page

    def whole(name):   # [B][kv head][S][D]
        x = cache[name][table].float() * cache[name + "_scale"][table][..., None, None]
        return x.permute(0, 2, 1, 3, 4).reshape(B, hk, S, D)

    count = starts[1:] - starts[:-1]
    i = torch.arange(n, device=DEV)
    token = (starts[:-1, None] + i).clamp_max(s["q"].shape[0] - 1)
    q = s["q"][token].float().reshape(B, n, hk, g, D).permute(0, 2, 1, 3, 4).reshape(B, hk, n * g, D)
    score = (q @ whole("k").transpose(-1, -2)).mul_(1 / math.sqrt(D))
    hidden = torch.arange(S, device=DEV) > (lengths - count)[:, None, None] + i[:, None]          # [B][n][S]
    score.view(B, hk, n, g, S).masked_fill_(hidden[:, None, :, None, :], -math.inf)
    score = score.sub_(score.amax(-1, keepdim=True)).exp_()
    total = score.sum(-1, keepdim=True)
    v = whole("v").masked_fill_((torch.arange(S, device=DEV) >= lengths[:, None])[:, None, :, None], 0.0)
    out = ((score @ v) / total).reshape(B, hk, n, g, D).permute(0, 2, 1, 3, 4).reshape(B, n, heads, D).half()
    t = torch.arange(s["q"].shape[0], device=DEV)
    seq = torch.searchsorted(starts, t, right=True) - 1
    return out[seq, t - starts[seq]]


def _plain_lora(s):
    x, a, b, adapter = s["x"].float(), s["a"], s["b"], s["adapter"].long()
    (M, K), (L, R, _), N = x.shape, a.shape, b.shape[1]
    has = (adapter >= 0).float()
    if M < L:   # few tokens: the adapters of each
        mine = adapter.clamp_min(0)
        z = (a[mine].float() @ x[:, :, None]).mul_((s["scaling"][mine] * has)[:, None, None])
        delta = (b[mine].float() @ z)[:, :, 0]
    else:       # all adapters in one product, those that are not a token's own at zero
        z = (x @ a.float().reshape(L * R, K).t()).reshape(M, L, R)
        z = z * ((adapter[:, None] == torch.arange(L, device=DEV)).float() * s["scaling"])[:, :, None]
        delta = z.reshape(M, L * R) @ b.float().permute(0, 2, 1).reshape(L * R, N)
    return (s["base"].float() + delta).half()


def run(state):
    op = state["case"]["op"]
    if own:
        import paper_2502_15779_b200 as rcp
        s = state
        if op == "lora":
            return rcp.rcp_lora_add(s["x"], s["a"], s["b"], s["adapter"], s["scaling"], base=s["base"], y=s["y"], workspace=s["scratch"])
        c = s["cache"]
        kv = rcp.KvCache(c["k"], c["v"], c["k_scale"], c["v_scale"])
        if op == "append":
            q = rcp.rcp_kv_append(s["k"], s["v"], kv, s["starts"], s["lengths"], s["table"], rope=s["rope"],
                                  interleaved=s["case"]["interleaved"], q=s["q"], q_out=s["out"], max_new=s["max_new"])
            return {"k": c["k"], "v": c["v"], "k_scale": c["k_scale"], "v_scale": c["v_scale"], "q": q}
        return rcp.rcp_kv_attention(s["q"], kv, s["starts"], s["lengths"], s["table"], max_new=s["max_new"], out=s["out"],
                                    workspace=s["scratch"])
    return _plain_lora(state) if op == "lora" else _plain_append(state) if op == "append" else _plain_attention(state)


def work(case):
    op = case["op"]
    if op == "lora":
        M, N, K, R = case["M"], case["N"], case["K"], case["rank"]
        used = min(case["adapters"], M)
        return {"bytes": 2 * M * K + 4 * M * N + 2 * used * R * (N + K), "flops": 2 * M * R * (N + K)}
    new, length = _lengths(case)
    T, heads, hk, D, page = sum(new), case["heads"], case["kv_heads"], case["dim"], case["page"]
    if op == "append":
        touched = sum((n - 1) // page - (n - m) // page + 1 for m, n in zip(new, length))
        return {"bytes": T * (hk * D * 6 + heads * D * 4 + case["rot"] * 4) + touched * hk * 16, "flops": T * (heads + hk) * case["rot"] * 3}
    pairs = sum(m * (n - m) + m * (m + 1) // 2 for m, n in zip(new, length))
    return {"bytes": sum(length) * hk * D * 2 + T * heads * D * 4 + sum(-(-n // page) for n in length) * (hk * 8 + 4),
            "flops": pairs * heads * D * 4}


# ---- the definitions in 64 bits, a sequence (or an adapter) at a time

def exact(case, seed):
    op = case["op"]
    s = prepare(case, seed)
    if op == "lora":
        y = s["base"].double()
        for l in range(case["adapters"]):
            rows = torch.nonzero(s["adapter"] == l)[:, 0]
            if rows.numel():
                y[rows] += s["scaling"][l].double() * ((s["x"][rows].double() @ s["a"][l].double().t()) @ s["b"][l].double().t())
        return y
    cache, page, table = s["cache"], case["page"], s["table"].tolist()
    starts, lengths = s["starts"].tolist(), s["lengths"].tolist()
    if op == "append":
        rope, rot = s["rope"].double(), case["rot"]
        q_all = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
        codes = {n: cache[n].float() for n in ("k", "v")}
        scale = {n: cache[n + "_scale"].double() for n in ("k", "v")}
        lo = torch.arange(0, rot, 2) if case["interleaved"] else torch.arange(rot // 2)
        hi = lo + (1 if case["interleaved"] else rot // 2)
        for b, n in enumerate(lengths):
            t0, t1 = starts[b], starts[b + 1]
            p0 = n - (t1 - t0)
            cos, sin = rope[p0:n, None, :, 0], rope[p0:n, None, :, 1]
            turned = {}
            for name in ("q", "k"):
                x = s[name][t0:t1].double()
                y = x.clone()
                y[..., lo] = x[..., lo] * cos - x[..., hi] * sin
                y[..., hi] = x[..., hi] * cos + x[..., lo] * sin
                turned[name] = y
            q_all[t0:t1] = turned["q"]
            turned["v"] = s["v"][t0:t1].double()
            for blk in range(p0 // page, (n - 1) // page + 1):
                at, f, l = table[b][blk], max(p0, blk * page), min(n, (blk + 1) * page)
                for name in ("k", "v"):
                    x = turned[name][f - p0:l - p0].transpose(0, 1)                       # [kv head][tokens][D]
                    want = torch.exp2(torch.ceil(torch.log2(x.abs().amax((1, 2)) / 448)).clamp(-40, 20))
                    now = want if f == blk * page else torch.maximum(want, scale[name][at])
                    if f > blk * page:
                        held = codes[name][at][:, :f - blk * page]
                        held.copy_((held.double() * (scale[name][at] / now)[:, None, None]).to(torch.float8_e4m3fn))
                    codes[name][at][:, f - blk * page:l - blk * page] = (x / now[:, None, None]).to(torch.float8_e4m3fn).float()
                    scale[name][at] = now
        return {"k": codes["k"], "v": codes["v"], "k_scale": scale["k"], "v_scale": scale["v"], "q": q_all}
    hk, D, g = case["kv_heads"], case["dim"], case["heads"] // case["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    for b, n in enumerate(lengths):
        t0, t1 = starts[b], starts[b + 1]
        ids = torch.tensor(table[b][:-(-n // page)], device=DEV)
        p = torch.arange(n - (t1 - t0), n, device=DEV)
        hidden = (torch.arange(n, device=DEV)[None] > p[:, None]).repeat_interleave(g, 0)
        for h in range(hk):
            k, v = ((cache[x][ids, h].double() * cache[x + "_scale"][ids, h].double()[:, None, None]).reshape(-1, D)[:n] for x in ("k", "v"))
            w = (s["q"][t0:t1, h * g:(h + 1) * g].double().reshape(-1, D) @ k.t()) / math.sqrt(D)
            w = torch.softmax(w.masked_fill_(hidden, -math.inf), -1)
            out[t0:t1, h * g:(h + 1) * g] = (w @ v).reshape(t1 - t0, g, D)
    return out

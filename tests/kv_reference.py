"""Plain forms of the operators on the paged 8-bit cache and of the adapters, a sequence and a head at a time: the append in the
arithmetic its interface pins (so codes and scales are compared bit for bit), attention and adapters in 64 bits."""
import math

import torch

EXP_MIN, EXP_MAX, CAP = -40, 9, 131072.0


def rope_table(positions, rot, base=10000.0, device="cuda:0"):
    """cosine and sine of position * base^(-2 i / rot), angles in 64 bits"""
    turn = base ** (-torch.arange(rot // 2, dtype=torch.float64, device=device) * 2 / rot)
    angle = torch.arange(positions, dtype=torch.float64, device=device)[:, None] * turn
    return torch.stack([angle.cos(), angle.sin()], -1).float().contiguous()


def rotate(x, rope_row, interleaved):
    """x float32 [heads][dim] of one position, each product and sum rounded once (a kernel of torch's each)"""
    n = 2 * rope_row.shape[0]
    c, s = rope_row[:, 0], rope_row[:, 1]
    y = x.clone()
    lo = torch.arange(0, n, 2, device=x.device) if interleaved else torch.arange(n // 2, device=x.device)
    hi = lo + 1 if interleaved else lo + n // 2
    a, b = x[:, lo], x[:, hi]
    ac, bs, bc, as_ = a * c, b * s, b * c, a * s
    y[:, lo], y[:, hi] = ac - bs, bc + as_
    return y


def exponent(amax):
    """smallest e with amax <= 448 * 2^e"""
    if amax == 0:
        return EXP_MIN
    m, e = math.frexp(amax)
    return min(max(e - 9 + (1 if m > 0.875 else 0), EXP_MIN), EXP_MAX)


def append(cache, k, v, starts, lengths, table, rope=None, interleaved=False, q=None, max_new=None):
    """What rcp_kv_append leaves behind: (KvCache of copies, rotated q with NaN in rows that are left as they were)."""
    kc, vc, ks, vs = (t.clone() for t in cache)
    pages, kv_heads, page, dim = kc.shape
    q_out = None if q is None else torch.full(q.shape, math.nan, dtype=torch.float16, device=q.device)
    width = table.shape[1]
    for b in range(len(lengths)):
        t0, t1 = starts[b], starts[b + 1]
        first, n = lengths[b] - (t1 - t0), min(t1 - t0, max_new or t1 - t0)
        blocks = {}
        for i in range(n):
            pos = first + i
            known = 0 <= pos < min(lengths[b], width * page)
            if q_out is not None:
                q_out[t0 + i] = (rotate(q[t0 + i].float(), rope[pos], interleaved).half() if rope is not None else q[t0 + i]) if known else 0
            if known:
                blocks.setdefault(pos // page, []).append((pos % page, t0 + i, pos))
        for blk, tokens in blocks.items():
            pg = int(table[b, blk])
            if not 0 <= pg < pages:
                continue
            for x, codes, scale in ((k, kc, ks), (v, vc, vs)):
                rows = []
                for _, t, pos in tokens:
                    r = x[t].float()
                    if x is k and rope is not None:
                        r = rotate(r, rope[pos], interleaved)
                    rows.append(torch.where(torch.isnan(r), torch.zeros_like(r), r.clamp(-CAP, CAP)))
                rows = torch.stack(rows)                                  # [tokens][kv_heads][dim]
                for h in range(kv_heads):
                    e = exponent(float(rows[:, h].abs().max()))
                    from_ = tokens[0][0]
                    if from_ > 0:
                        old = round(math.log2(float(scale[pg, h])))
                        if e > old:
                            held = codes[pg, h, :from_]
                            codes[pg, h, :from_] = (held.float() * 2.0 ** (old - e)).to(torch.float8_e4m3fn)
                        e = max(e, old)
                    scale[pg, h] = 2.0 ** e
                    codes[pg, h, from_:from_ + len(tokens)] = (rows[:, h] * 2.0 ** -e).to(torch.float8_e4m3fn)
    return (kc, vc, ks, vs), q_out


def attention(q, cache, starts, lengths, table, sm_scale, max_new=None):
    """(out, bound) in 64 bits, NaN in rows that are left as they were. bound: how far a result may be off when weights are rounded to fp16
    for the product with the values and everything else is fp32 (terms below)."""
    kc, vc, ks, vs = cache
    pages, kv_heads, page, dim = kc.shape
    heads = q.shape[1]
    g = heads // kv_heads
    out = torch.full(q.shape, math.nan, dtype=torch.float64, device=q.device)
    tol = torch.full_like(out, math.nan)
    width = table.shape[1]
    for b in range(len(lengths)):
        t0, t1 = starts[b], starts[b + 1]
        n = min(t1 - t0, max_new or t1 - t0)
        if n == 0:
            continue
        end = min(max(lengths[b], 0), width * page)
        pos = torch.arange(n, device=q.device) + lengths[b] - (t1 - t0)
        j = torch.arange(end, device=q.device)
        pg = table[b].to(q.device).long()[j // page]
        there = (pg >= 0) & (pg < pages)
        j, pg = j[there], pg[there]
        out[t0:t0 + n] = 0
        tol[t0:t0 + n] = 0
        if j.numel() == 0:
            continue
        seen = (j[None, :] <= pos[:, None]) & (pos[:, None] < end) & (pos[:, None] >= 0)
        for h in range(kv_heads):
            K = kc[pg, h, j % page].double() * ks[pg, h].double()[:, None]
            V = vc[pg, h, j % page].double() * vs[pg, h].double()[:, None]
            for hh in range(h * g, (h + 1) * g):
                Q = q[t0:t0 + n, hh].double()
                s = (Q @ K.t()) * sm_scale
                s = s.masked_fill(~seen, -math.inf)
                top = s.amax(1, keepdim=True)
                p = torch.where(seen, torch.exp(s - torch.where(torch.isinf(top), torch.zeros_like(top), top)), torch.zeros_like(s))
                total = p.sum(1, keepdim=True)
                some = (total > 0).double()
                total = total.clamp_min(1e-300)
                o, a = p @ V / total, p @ V.abs() / total
                # a score is a sum of dim products in fp32, in an order and with a rounding the tensor core chooses: 2^-22 of the sum of
                # magnitudes for each; exponent, its argument's roundings: 2^-20 of a weight
                mag = (Q.abs() @ K.abs().t()) * sm_scale
                delta = dim * 2.0 ** -22 * torch.where(seen, mag, torch.zeros_like(mag)).amax(1, keepdim=True) + 2.0 ** -20
                # a weight: half a step of fp16, 2^-11 (in the format's range: weights below 2^-21 of the largest lose 2^-32 of it each at most,
                # `floor`); numerator and denominator each off by delta; sums in fp32: keys * 2^-24; the result: half a step, or 2^-25 among fp16's subnormals
                floor = 2.0 ** -32 * seen.sum(1, keepdim=True).double() * V.abs().amax()
                t = (2.0 ** -11 + 2 * delta + j.numel() * 2.0 ** -23) * a + floor / total + 2.0 ** -11 * o.abs() * 1.01 + 2.0 ** -25
                out[t0:t0 + n, hh] = o * some
                tol[t0:t0 + n, hh] = t * some
    return out, tol


def lora(x, a, b, adapter, scaling, base):
    """(y, bound) in 64 bits. Rounding of both sums in fp32 (2^-24 a term, as if every one were rounded at full size), of z to fp16 where the
    second product goes through the tensor cores in two parts (2^-21 of a term is left out), and of the result to fp16."""
    M, K = x.shape
    L, R, _ = a.shape
    N = b.shape[1]
    y = torch.zeros(M, N, dtype=torch.float64, device=x.device) if base is None else base.double()
    size = y.abs()
    for i in range(L):
        rows = torch.nonzero(adapter == i)[:, 0]
        if rows.numel():
            X, A, B, s = x[rows].double(), a[i].double(), b[i].double(), float(scaling[i])
            y[rows] += s * (X @ A.t() @ B.t())
            size[rows] += abs(s) * (X.abs() @ A.abs().t() @ B.abs().t())
    return y, (K + R + 4) * 2.0 ** -24 * size + 2.0 ** -20 * size + 2.0 ** -11 * y.abs() * 1.01 + 2.0 ** -25

"""The paged 8-bit cache on the GPU: rcp_kv_append bit for bit against its pinned arithmetic, rcp_kv_attention against 64 bits."""
import math

import pytest
import torch

import kv_reference as ref
import paper_2502_15779_b200 as rcp

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def rand(*shape, seed=0, std=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(*shape, generator=g, device=DEV) * std).half()


def random_cache(pages, kv_heads, page, dim, seed=0, lo=-8, hi=-5):
    """Codes all over the format (its two NaNs left out), scales of a few exponents."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    raw = [torch.randint(0, 256, (pages, kv_heads, page, dim), generator=g, device=DEV, dtype=torch.uint8) for _ in range(2)]
    raw = [torch.where((r & 127) >= 0x70, r & 0xBF, r).view(torch.float8_e4m3fn) for r in raw]
    scales = [torch.exp2(torch.randint(lo, hi + 1, (pages, kv_heads), generator=g, device=DEV).float()) for _ in range(2)]
    return rcp.KvCache(*raw, *scales)


def make_table(lengths, page, pages, seed=0, width=None):
    """Pages in random order, entries behind a sequence's last page pointing outside."""
    g = torch.Generator().manual_seed(seed)
    need = [-(-n // page) for n in lengths]
    width = width or max(max(need), 1)
    order = torch.randperm(pages, generator=g)
    assert sum(need) <= pages
    table, at = torch.full((len(lengths), width), -1, dtype=torch.int32), 0
    table[:, 1::2] = pages + 5
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n].int()
        at += n
    return table


def tensors(starts, lengths, table):
    return (torch.tensor(starts, dtype=torch.int32, device=DEV), torch.tensor(lengths, dtype=torch.int32, device=DEV), table.to(DEV).contiguous())


def starts_of(new, at=0):
    out = [at]
    for n in new:
        out.append(out[-1] + n)
    return out


def same_bits(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


# new tokens and cached ones of each sequence, heads, kv heads, dim, page, rotated dimensions, interleaved
APPEND = [
    ([1], [0], 4, 2, 64, 32, 64, False),
    ([1, 1, 1], [0, 31, 32], 8, 8, 128, 32, 128, False),
    ([1, 0, 2, 0], [63, 5, 127, 0], 6, 2, 128, 64, 128, True),
    ([70, 1, 200], [10, 64, 0], 8, 2, 64, 64, 32, False),
    ([129, 300], [127, 1], 3, 3, 128, 128, 64, True),
    ([33, 31, 32, 64, 65], [0, 1, 0, 32, 31], 5, 1, 64, 32, 48, False),
    ([257], [128], 20, 4, 128, 128, 128, False),
    ([5] * 40, [60 + 3 * i for i in range(40)], 4, 1, 128, 64, 128, False),
    ([1] * 3 + [900] + [1] * 150, [7] * 154, 4, 1, 64, 64, 64, True),      # blocks are found by search
]


@pytest.mark.parametrize("new,cached,heads,kv_heads,dim,page,rot,interleaved", APPEND)
@pytest.mark.parametrize("hint", [False, True])
def test_append_gives_the_pinned_codes(new, cached, heads, kv_heads, dim, page, rot, interleaved, hint):
    lengths = [n + c for n, c in zip(new, cached)]
    pages = sum(-(-n // page) for n in lengths) + 2
    cache = random_cache(pages, kv_heads, page, dim, seed=1)
    table = make_table(lengths, page, pages, seed=2)
    starts, T = starts_of(new, 2), sum(new) + 5           # two rows in front and three behind belong to nobody
    row = rand(T, heads + 2 * kv_heads, dim, seed=3, std=2.0)
    row[:2], row[-3:] = math.nan, math.inf
    q, k, v = row[:, :heads], row[:, heads:heads + kv_heads], row[:, heads + kv_heads:]
    rope = ref.rope_table(table.shape[1] * page, rot)
    want, want_q = ref.append(cache, k, v, starts, lengths, table, rope, interleaved, q)
    q_out = torch.full((T, heads, dim), math.nan, dtype=torch.float16, device=DEV)
    got_q = rcp.rcp_kv_append(k, v, cache, *tensors(starts, lengths, table), rope=rope, interleaved=interleaved, q=q, q_out=q_out,
                              max_new=max(new) if hint else 0)
    for name, g, w in zip(cache._fields, cache, want):
        assert same_bits(g, w), name
    assert same_bits(got_q, want_q)


def test_append_without_rotation_or_queries():
    page, lengths = 64, [100, 3]
    cache = random_cache(5, 2, page, 64, seed=4)
    table = make_table(lengths, page, 5)
    k, v = rand(103, 2, 64, seed=5), rand(103, 2, 64, seed=6)
    want, _ = ref.append(cache, k, v, [0, 100, 103], lengths, table)
    assert rcp.rcp_kv_append(k, v, cache, *tensors([0, 100, 103], lengths, table)) is None
    assert all(same_bits(g, w) for g, w in zip(cache, want))


def test_append_token_by_token_rescales_what_the_block_holds():
    """Magnitudes that grow, shrink, reach the largest fp16 number, are subnormal or zero; every step against the plain form."""
    page, dim = 32, 64
    cache = rcp.make_kv_cache(3, 2, dim, page, DEV)
    table = torch.tensor([[2, 0]], dtype=torch.int32)
    sizes = [0.0, 2.0 ** -20, 1e-3, 0.5, 448.0, 447.9, 449.0, 1.0, 896.0, 60000.0, 1e-4, 65504.0] + [float(1.5 ** i) for i in range(25)]
    rope = ref.rope_table(64, dim)
    for i, size in enumerate(sizes):
        k, v = (rand(1, 2, dim, seed=10 * i + s).clamp(-1, 1).float().mul(size).half() for s in (0, 1))
        k[0, 0, 0] = v[0, 1, 3] = size
        args = ([0, 1], [i + 1], table)
        want, _ = ref.append(cache, k, v, *args, rope)
        rcp.rcp_kv_append(k, v, cache, *tensors(*args), rope=rope, max_new=1)
        for name, g, w in zip(cache._fields, cache, want):
            assert same_bits(g, w), (i, name)


def test_a_power_of_two_scale_makes_the_order_of_appends_immaterial():
    """In one call or in several, where no value falls below the format's range."""
    page, dim, n = 64, 128, 150
    k, v = (rand(n, 2, dim, seed=s).float() for s in (20, 21))
    k, v = (torch.sign(x).half() * (x.abs() + 0.25).half() for x in (k, v))
    table = torch.tensor([[1, 3, 0]], dtype=torch.int32)
    one, many = rcp.make_kv_cache(4, 2, dim, page, DEV), rcp.make_kv_cache(4, 2, dim, page, DEV)
    rcp.rcp_kv_append(k, v, one, *tensors([0, n], [n], table))
    at = 0
    for m in (1, 62, 2, 40, 45):
        rcp.rcp_kv_append(k[at:at + m], v[at:at + m], many, *tensors([0, m], [at + m], table))
        at += m
    assert at == n and all(same_bits(a, b) for a, b in zip(one, many))


def test_append_bad_pages_and_positions():
    """Pages outside the cache, lengths below the number of new tokens, positions behind the table, more tokens than max_new: nothing is
    stored for them, and everything else is stored as ever."""
    page, dim, kv_heads = 32, 64, 2
    cache = random_cache(6, kv_heads, page, dim, seed=7)
    table = torch.tensor([[0, -1, 1], [2, 3, 6], [4, -2147483648, 2147483647], [5, 5, 5]], dtype=torch.int32)
    new, lengths = [90, 50, 40, 20], [96, 110, 12, 8]
    starts = starts_of(new)
    k, v, q = rand(200, kv_heads, dim, seed=8), rand(200, kv_heads, dim, seed=9), rand(200, 4, dim, seed=10)
    rope = ref.rope_table(96, dim)
    for max_new in (0, 25):
        c = rcp.KvCache(*(t.clone() for t in cache))
        want, want_q = ref.append(c, k, v, starts, lengths, table, rope, False, q, max_new or None)
        q_out = torch.full(q.shape, math.nan, dtype=torch.float16, device=DEV)
        got_q = rcp.rcp_kv_append(k, v, c, *tensors(starts, lengths, table), rope=rope, q=q, q_out=q_out, max_new=max_new)
        assert all(same_bits(g, w) for g, w in zip(c, want)) and same_bits(got_q, want_q)


def test_append_nan_and_infinity_do_not_spoil_a_block():
    page, dim = 64, 128
    cache = random_cache(1, 1, page, dim, seed=11)
    k, v = rand(3, 1, dim, seed=12), rand(3, 1, dim, seed=13)
    k[1, 0, 5], v[1, 0, 6], v[2, 0, 7], k[2, 0, 9] = math.nan, math.nan, math.inf, -math.inf
    args = ([0, 3], [20, ], torch.zeros(1, 1, dtype=torch.int32))
    want, _ = ref.append(cache, k, v, *args, None)
    rcp.rcp_kv_append(k, v, cache, *tensors(*args))
    assert all(same_bits(g, w) for g, w in zip(cache, want))
    assert bool(torch.isfinite(cache.k.float()).all()) and bool(torch.isfinite(cache.v.float()).all())


def test_append_rotates_queries_in_place():
    page, dim, T = 64, 128, 37
    cache = rcp.make_kv_cache(1, 1, dim, page, DEV)
    q = rand(T, 6, dim, seed=14)
    k = rand(T, 1, dim, seed=15)
    rope = ref.rope_table(64, dim)
    args = ([0, T], [50], torch.zeros(1, 1, dtype=torch.int32))
    _, want = ref.append(cache, k, k, *args, rope, True, q)
    assert same_bits(rcp.rcp_kv_append(k, k, cache, *tensors(*args), rope=rope, interleaved=True, q=q, q_out=q), want)


# new and cached tokens, heads, kv heads, dim, page
ATTENTION = [
    ([1], [0], 4, 4, 64, 32),
    ([1], [776], 32, 8, 64, 64),
    ([1, 1, 1, 1], [0, 31, 32, 33], 8, 8, 128, 32),
    ([1, 0, 1, 1, 0], [64, 9, 63, 1000, 0], 8, 1, 128, 64),
    ([1] * 7, [100 * i + 13 for i in range(7)], 5, 5, 128, 128),
    ([1] * 33, [17 * i for i in range(33)], 24, 1, 128, 64),
    ([1], [20011], 16, 2, 128, 64),
    ([1, 1], [9000, 5], 40, 8, 64, 128),
    ([2, 5, 1, 8], [30, 511, 0, 77], 32, 8, 128, 64),
    ([4, 3], [2000, 64], 20, 4, 64, 32),
    ([3, 1], [100, 3000], 7, 7, 128, 32),
    ([9, 17, 33], [0, 1, 100], 6, 2, 128, 64),
    ([64], [0], 4, 4, 128, 64),
    ([65, 1, 129], [3, 50, 200], 8, 2, 128, 64),
    ([300], [129], 12, 4, 64, 64),
    ([127, 128, 1, 2, 256], [0, 0, 31, 32, 1000], 4, 1, 128, 128),
    ([513, 1], [777, 2], 5, 1, 128, 32),
    ([200, 31], [0, 600], 48, 2, 64, 64),
    ([200], [2500], 32, 8, 128, 64),
    ([90, 3, 1], [3000, 10, 2000], 16, 2, 64, 32),
    ([400], [900], 4, 2, 128, 128),
    ([1], [20000], 24, 1, 128, 64),
    ([1, 2], [19000, 12345], 8, 1, 64, 128),
    ([3, 1, 1], [10000, 15000, 11000], 3, 1, 128, 32),
    ([9, 0, 30, 1], [300, 0, 40, 900], 12, 3, 128, 64),
    ([1] * 32, [i * 7 for i in range(32)], 4, 4, 64, 32),
    ([2] * 18, [1500] * 18, 16, 8, 64, 128),
]


def check_attention(out, want, tol):
    left = torch.isnan(want)
    assert bool(torch.isnan(out[left]).all()), "rows of no sequence were written"
    off = (out.double() - want).abs()[~left]
    assert bool((off <= tol[~left]).all()), f"off by {float((off / tol[~left].clamp_min(1e-30)).max()):.3f} of the bound"


@pytest.mark.parametrize("new,cached,heads,kv_heads,dim,page", ATTENTION)
@pytest.mark.parametrize("hint", [False, True])
def test_attention_against_64_bits(new, cached, heads, kv_heads, dim, page, hint):
    lengths = [n + c for n, c in zip(new, cached)]
    pages = sum(-(-n // page) for n in lengths) + 2
    cache = random_cache(pages, kv_heads, page, dim, seed=21)
    table = make_table(lengths, page, pages, seed=22)
    # slots behind a length hold NaN codes: they may hold anything
    for b, n in enumerate(lengths):
        if n % page:
            for t in (cache.k, cache.v):
                t.view(torch.uint8)[int(table[b, n // page]), :, n % page:] = 0x7F
    starts, T = starts_of(new, 1), sum(new) + 4
    row = rand(T, heads + 3, dim, seed=23)                       # queries are part of wider rows
    row[:1], row[-3:] = math.nan, math.nan
    q = row[:, 1:1 + heads]
    want, tol = ref.attention(q, cache, starts, lengths, table, dim ** -0.5)
    out = torch.full((T, heads, dim), math.nan, dtype=torch.float16, device=DEV)
    got = rcp.rcp_kv_attention(q, cache, *tensors(starts, lengths, table), out=out, max_new=max(new) if hint else 0)
    check_attention(got, want, tol)


@pytest.mark.parametrize("new", [1, 6, 150])
@pytest.mark.parametrize("size", [0.0, 1e-3, 8.0, 300.0])
def test_attention_flat_and_peaked_weights(new, size):
    """Scores all alike, ordinary, or so large that one key takes all; block scales that differ by many powers of two."""
    page, dim, heads, kv_heads, n = 64, 128, 8, 2, 700
    cache = random_cache(12, kv_heads, page, dim, seed=31, lo=-20, hi=-4)
    cache.v_scale[::3] = 2.0 ** -40
    cache.v_scale[1::3] = 2.0 ** -2
    table = make_table([n], page, 12, seed=32)
    q = (rand(new, heads, dim, seed=33).float() * size).half()
    want, tol = ref.attention(q, cache, [0, new], [n], table, dim ** -0.5)
    got = rcp.rcp_kv_attention(q, cache, *tensors([0, new], [n], table))
    check_attention(got, want, tol)


@pytest.mark.parametrize("new", [1, 40, 300])
def test_attention_missing_pages_and_positions(new):
    """Keys in pages outside the cache are not there; rows that are left with none, or whose position does not exist, are zero."""
    page, dim, heads, kv_heads = 32, 64, 4, 2
    cache = random_cache(20, kv_heads, page, dim, seed=41)
    width = 12
    table = torch.full((4, width), -1, dtype=torch.int32)
    table[0, ::2] = torch.arange(6, dtype=torch.int32)       # every second page is missing
    table[1] = 1 << 30                                       # all of them
    table[2] = torch.arange(6, 18, dtype=torch.int32)        # a length below the number of new tokens
    table[3] = torch.arange(6, 18, dtype=torch.int32)        # a length beyond the table
    lengths = [380, 370, max(new - 3, 0), width * page + 2]
    new_each = [new] * 4
    starts = starts_of(new_each)
    q = rand(4 * new, heads, dim, seed=42)
    want, tol = ref.attention(q, cache, starts, lengths, table, dim ** -0.5)
    out = torch.full(q.shape, math.nan, dtype=torch.float16, device=DEV)
    got = rcp.rcp_kv_attention(q, cache, *tensors(starts, lengths, table), out=out)
    check_attention(got, want, tol)


def test_attention_of_more_tokens_than_max_new_leaves_the_rest():
    page, dim, heads = 64, 64, 4
    cache = random_cache(6, 2, page, dim, seed=51)
    table = make_table([200, 90], page, 6, seed=52)
    starts, lengths = [0, 50, 53], [200, 90]
    q = rand(53, heads, dim, seed=53)
    want, tol = ref.attention(q, cache, starts, lengths, table, 0.1, max_new=20)
    out = torch.full(q.shape, math.nan, dtype=torch.float16, device=DEV)
    check_attention(rcp.rcp_kv_attention(q, cache, *tensors(starts, lengths, table), sm_scale=0.1, max_new=20, out=out), want, tol)


def test_attention_of_many_short_sequences():
    """More sequences than a CTA has threads, some without new tokens or without any tokens, few rows and many among them."""
    page, dim, heads, kv_heads, B = 32, 64, 8, 4, 700
    g = torch.Generator().manual_seed(55)
    new = (torch.rand(B, generator=g) * 3).int().tolist()
    new[5], new[300], new[699] = 150, 40, 60
    lengths = [n + int(x) for n, x in zip(new, (torch.rand(B, generator=g) * 90).int())]
    lengths[0] = new[0] = 0
    pages = sum(-(-n // page) for n in lengths)
    cache = random_cache(pages, kv_heads, page, dim, seed=56)
    table = make_table(lengths, page, pages, seed=57)
    starts = starts_of(new)
    q = rand(sum(new) + 2, heads, dim, seed=58)
    want, tol = ref.attention(q, cache, starts, lengths, table, dim ** -0.5)
    out = torch.full(q.shape, math.nan, dtype=torch.float16, device=DEV)
    check_attention(rcp.rcp_kv_attention(q, cache, *tensors(starts, lengths, table), out=out), want, tol)
    # one token each: the kernel of few rows alone
    new, starts = [1] * B, starts_of([1] * B)
    q = rand(B, heads, dim, seed=59)
    lengths = [max(n, 1) for n in lengths]
    table = make_table(lengths, page, pages + B, seed=60)
    cache = random_cache(pages + B, kv_heads, page, dim, seed=61)
    want, tol = ref.attention(q, cache, starts, lengths, table, dim ** -0.5)
    check_attention(rcp.rcp_kv_attention(q, cache, *tensors(starts, lengths, table), max_new=1), want, tol)


@pytest.mark.parametrize("heads,kv_heads", [(40, 1), (200, 1), (64, 1), (65, 1), (128, 2), (3, 3)])
@pytest.mark.parametrize("new", [1, 3])
def test_attention_many_query_heads_of_a_key_head(heads, kv_heads, new):
    page, dim, lengths = 64, 128, [500, 64, 131]
    cache = random_cache(13, kv_heads, page, dim, seed=44)
    table = make_table(lengths, page, 13, seed=45)
    q = rand(3 * new, heads, dim, seed=46)
    for seqs in (1, 3):
        starts = starts_of([new] * seqs)
        want, tol = ref.attention(q[:seqs * new], cache, starts, lengths[:seqs], table[:seqs], dim ** -0.5)
        check_attention(rcp.rcp_kv_attention(q[:seqs * new], cache, *tensors(starts, lengths[:seqs], table[:seqs]), max_new=new), want, tol)


@pytest.mark.parametrize("new", [1, 9, 100])
def test_attention_a_bad_query_stays_alone_and_a_scale_of_zero_weighs_all_alike(new):
    page, dim, heads, kv_heads, n = 64, 64, 8, 2, 400
    cache = random_cache(8, kv_heads, page, dim, seed=47)
    table = make_table([n], page, 8, seed=48)
    args = tensors([0, new], [n], table)
    q = rand(new, heads, dim, seed=49)
    want, tol = ref.attention(q, cache, [0, new], [n], table, dim ** -0.5)
    q[0, 1, 3], q[new // 2, 6, 0], q[new - 1, 7, 9] = math.nan, math.inf, math.nan
    got = rcp.rcp_kv_attention(q, cache, *args)
    fine = torch.ones(new, heads, dtype=torch.bool, device=DEV)
    for t, h in ((0, 1), (new // 2, 6), (new - 1, 7)):
        fine[t, h] = False
    assert bool(((got.double() - want).abs() <= tol)[fine].all())
    assert bool(torch.isnan(got[0, 1]).all()) and bool(torch.isnan(got[new - 1, 7]).all())
    q = rand(new, heads, dim, seed=50)
    check_attention(rcp.rcp_kv_attention(q, cache, *args, sm_scale=0.0), *ref.attention(q, cache, [0, new], [n], table, 0.0))


def test_attention_in_the_place_of_its_queries():
    page, dim, heads, kv_heads = 64, 128, 8, 2
    for new, length in ((1, 5000), (150, 700)):
        cache = random_cache(90, kv_heads, page, dim, seed=51)
        table = make_table([length], page, 90, seed=52)
        args = tensors([0, new], [length], table)
        q = rand(new, heads, dim, seed=53)
        want = rcp.rcp_kv_attention(q.clone(), cache, *args)
        assert torch.equal(rcp.rcp_kv_attention(q, cache, *args, out=q), want)


def test_attention_results_repeat_and_leave_the_workspace_ready():
    page, dim, heads, kv_heads = 64, 128, 16, 2
    lengths = [5000, 1, 900, 12000]
    cache = random_cache(300, kv_heads, page, dim, seed=61)
    table = make_table(lengths, page, 300, seed=62)
    args = tensors(starts_of([1] * 4), lengths, table)
    q, ws = rand(4, heads, dim, seed=63), rcp.make_kv_workspace(DEV)
    first = rcp.rcp_kv_attention(q, cache, *args, workspace=ws).clone()
    other = rcp.rcp_kv_attention(rand(4, heads, dim, seed=64), cache, *args, workspace=ws)
    assert not torch.equal(first, other)
    for _ in range(20):
        assert torch.equal(rcp.rcp_kv_attention(q, cache, *args, workspace=ws), first)


@pytest.mark.parametrize("dim,heads,new,length", [(128, 32, 20, 3000), (128, 32, 200, 1500), (64, 16, 40, 5000)])
def test_attention_of_many_ctas_at_once(dim, heads, new, length):
    """Enough sequences that every SM is at work and its warps drift apart; several runs, each the same and each right."""
    page, kv_heads, B = 64, 8, 16
    lengths = [length - 17 * b for b in range(B)]
    pages = sum(-(-n // page) for n in lengths)
    cache = random_cache(pages, kv_heads, page, dim, seed=65)
    table = make_table(lengths, page, pages, seed=66)
    args = tensors(starts_of([new] * B), lengths, table)
    q, ws = rand(B * new, heads, dim, seed=67), rcp.make_kv_workspace(DEV)
    outs = [rcp.rcp_kv_attention(q, cache, *args, workspace=ws) for _ in range(25)]
    torch.cuda.synchronize()
    assert int(ws[:4].view(torch.int32)) == 0
    want, tol = ref.attention(q, cache, starts_of([new] * B), lengths, table, dim ** -0.5)
    check_attention(outs[0], want, tol)
    assert all(torch.equal(o, outs[0]) for o in outs[1:])


@pytest.mark.parametrize("new,cached,heads,kv_heads,dim", [([300], [129], 12, 4, 64), ([65, 1, 129], [3, 50, 200], 8, 2, 128), ([70], [0], 4, 1, 128)])
def test_attention_of_short_prompts_many_times(new, cached, heads, kv_heads, dim):
    """A few tiles of keys, whose ends the kernel's warps reach in any order: no wait may give up and every run gives the same."""
    page, lengths = 64, [n + c for n, c in zip(new, cached)]
    pages = sum(-(-n // page) for n in lengths) + 1
    cache = random_cache(pages, kv_heads, page, dim, seed=68)
    args = tensors(starts_of(new), lengths, make_table(lengths, page, pages, seed=69))
    q, ws = rand(sum(new), heads, dim, seed=70), rcp.make_kv_workspace(DEV)
    first = rcp.rcp_kv_attention(q, cache, *args, workspace=ws)
    bad = torch.zeros((), dtype=torch.int64, device=DEV)
    for _ in range(400):
        bad += (rcp.rcp_kv_attention(q, cache, *args, workspace=ws) != first).sum()
    assert int(ws[:4].view(torch.int32)) == 0 and int(bad) == 0


def test_captured_calls_follow_lengths_and_tables():
    """Append and attention of a decode step captured once; lengths and tables change between replays."""
    page, dim, heads, kv_heads, B = 32, 64, 8, 2, 3
    lengths0 = [30, 64, 5]
    cache = random_cache(40, kv_heads, page, dim, seed=71)
    table = torch.randperm(40, generator=torch.Generator().manual_seed(72))[:B * 8].int().reshape(B, 8)
    starts, lengths, tab = tensors(starts_of([1] * B), lengths0, table)
    rope = ref.rope_table(8 * page, dim)
    row = rand(B, heads + 2 * kv_heads, dim, seed=73)
    q, k, v = row[:, :heads], row[:, heads:heads + kv_heads], row[:, heads + kv_heads:]
    q_rot, out = (torch.empty(B, heads, dim, dtype=torch.float16, device=DEV) for _ in range(2))
    ws = rcp.make_kv_workspace(DEV)

    def step():
        rcp.rcp_kv_append(k, v, cache, starts, lengths, tab, rope=rope, q=q, q_out=q_rot, max_new=1)
        rcp.rcp_kv_attention(q_rot, cache, starts, lengths, tab, max_new=1, out=out, workspace=ws)

    saved = [t.clone() for t in cache]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    torch.cuda.current_stream().wait_stream(s)
    for t, w in zip(cache, saved):
        t.view(torch.uint8).copy_(w.view(torch.uint8))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    at = list(lengths0)
    for i in range(70):
        at = [min(n + 1 + (b == 1) * 0, 8 * page) for b, n in enumerate(at)]
        row.copy_(rand(B, heads + 2 * kv_heads, dim, seed=100 + i))
        lengths.copy_(torch.tensor(at, dtype=torch.int32))
        want_cache, want_q = ref.append(cache, k, v, starts_of([1] * B), at, table, rope, False, q)
        graph.replay()
        assert all(same_bits(g, w) for g, w in zip(cache, want_cache)) and same_bits(q_rot, want_q), i
        if i % 10 == 0:
            want, tol = ref.attention(q_rot, cache, starts_of([1] * B), at, table, dim ** -0.5)
            check_attention(out, want, tol)


def test_calls_on_several_streams():
    page, dim, heads, kv_heads = 64, 128, 8, 2
    streams = [torch.cuda.Stream() for _ in range(3)]
    sets = []
    for i in range(3):
        lengths = [3000 + 500 * i, 70]
        cache = random_cache(90, kv_heads, page, dim, seed=81 + i)
        table = make_table(lengths, page, 90, seed=82 + i)
        args = tensors([0, 1, 2], lengths, table)
        q = rand(2, heads, dim, seed=83 + i)
        want = rcp.rcp_kv_attention(q, cache, *args)
        sets.append((q, cache, args, want, rcp.make_kv_workspace(DEV), torch.empty_like(want)))
    torch.cuda.synchronize()
    for _ in range(10):
        for st, (q, cache, args, _, ws, out) in zip(streams, sets):
            with torch.cuda.stream(st):
                rcp.rcp_kv_attention(q, cache, *args, out=out, workspace=ws)
    torch.cuda.synchronize()
    for _, _, _, want, _, out in sets:
        assert torch.equal(out, want)


def test_cache_beyond_four_gibibytes():
    """Offsets into the codes pass 32 bits."""
    page, dim, kv_heads, heads = 128, 128, 8, 16
    pages = (1 << 32) // (page * dim * kv_heads) + 40
    if torch.cuda.mem_get_info()[0] < 3 * pages * page * dim * kv_heads:
        pytest.skip("not enough free memory")
    cache = rcp.make_kv_cache(pages, kv_heads, dim, page, DEV)
    assert cache.k.numel() > 1 << 32
    lengths = [500, 300]
    table = torch.tensor([[pages - 1, 0, pages - 3, pages // 2], [pages - 5, pages - 6, 1, -1]], dtype=torch.int32)
    k, v = rand(800, kv_heads, dim, seed=91), rand(800, kv_heads, dim, seed=92)
    args = tensors([0, 500, 800], lengths, table)
    rcp.rcp_kv_append(k, v, cache, *args)
    small = rcp.make_kv_cache(7, kv_heads, dim, page, DEV)
    near = torch.tensor([[0, 1, 2, 3], [4, 5, 6, -1]], dtype=torch.int32)
    rcp.rcp_kv_append(k, v, small, *tensors([0, 500, 800], lengths, near))
    for far, here in zip(table.flatten().tolist(), near.flatten().tolist()):
        if far >= 0:
            assert all(same_bits(a[far], b[here]) for a, b in zip(cache, small))
    for starts, new in (([0, 1, 2], 1), ([0, 200, 400], 200)):
        q = rand(2 * new, heads, dim, seed=93)
        a = rcp.rcp_kv_attention(q, cache, *tensors(starts, lengths, table))
        b = rcp.rcp_kv_attention(q, small, *tensors(starts, lengths, near))
        assert torch.equal(a, b)


@pytest.mark.parametrize("dim,kv_heads", [(64, 2), (128, 8)])
@pytest.mark.parametrize("low", [-11, -12, -14, -20, -22])
def test_prompt_values_of_unlike_blocks_side_by_side(dim, kv_heads, low):
    """Pages of 32, two of them in the prompt kernel's 64 keys, whose values' scales differ by 2^4 to 2^15 behind blocks of larger ones; queries look at
    keys of the small blocks alone, whose values have to come out as exactly as if the large ones were not there."""
    page, heads, length = 32, 4 * kv_heads, 1200
    new = 8000 // kv_heads // 4 + 40                                   # more rows than the kernel of few rows takes
    cache = random_cache(40, kv_heads, page, dim, seed=101, lo=-7, hi=-7)
    table = make_table([length], page, 40, seed=102)
    ids = table[0].long().to(DEV)
    cache.v_scale[ids] = 2.0 ** 8                                      # positions 0 .. 63
    cache.v_scale[ids[2::2]] = 2.0 ** (8 - 7)                          # from 64 on: the largest of 64 positions
    cache.v_scale[ids[3::2]] = 2.0 ** (8 + low)                        # and the other block of them
    value = (torch.arange(dim, device=DEV) % 126 + 1).to(torch.uint8)  # all positive codes, the same row for every token of a small block
    cache.v.view(torch.uint8)[ids[3::2]] = value
    key = torch.zeros(dim, device=DEV)
    key[0] = 448.0
    cache.k.view(torch.uint8).fill_(0)
    cache.k[ids[3::2]] = key.to(torch.float8_e4m3fn)                   # a score of 61 and more against zero: the others weigh 2^-88 at most
    q = torch.zeros(new, heads, dim, dtype=torch.float16, device=DEV)
    q[:, :, 0] = 200.0
    want, _ = ref.attention(q, cache, [0, new], [length], table, dim ** -0.5)
    exact = value.view(torch.float8_e4m3fn).double() * 2.0 ** (8 + low)
    # the other keys: fewer than 2^11 of magnitude 448 2^8 < 2^17 at 2^-88 of the weight
    assert bool(((want - exact).abs() <= 2.0 ** -60).all())
    got = rcp.rcp_kv_attention(q, cache, *tensors([0, new], [length], table))
    off = (got.double() - want).abs()
    # weights alike and a power of two: exact; sums of fewer than 2^10 terms in fp32 2^-13; the result to fp16
    assert bool((off <= (2.0 ** -11 + 2.0 ** -13) * want.abs() + 1.01 * 2.0 ** -25).all()), float((off / want.abs()).max())


@pytest.mark.parametrize("new,cached,page,dim", [([1, 1], [5, 64], 64, 128), ([1], [0], 32, 64), ([40, 3], [10, 0], 32, 64), ([100], [20], 128, 128)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_cuts_off_finite_magnitudes_too(new, cached, page, dim, interleaved):
    """Cosines and sines that carry a factor (as for longer contexts) make keys above 2^17, all of them finite: stored as 2^17."""
    lengths = [n + c for n, c in zip(new, cached)]
    cache = random_cache(10, 2, page, dim, seed=111)
    table = make_table(lengths, page, 10, seed=112)
    starts, T = starts_of(new), sum(new)
    k, v = (rand(T, 2, dim, seed=113 + i).clamp(-1, 1) for i in range(2))
    k[:, 0] *= 60000.0
    k[0, 1, 3] = 65504.0
    rope = 4.0 * ref.rope_table(table.shape[1] * page, dim)
    want, _ = ref.append(cache, k, v, starts, lengths, table, rope, interleaved)
    rcp.rcp_kv_append(k, v, cache, *tensors(starts, lengths, table), rope=rope, interleaved=interleaved, max_new=max(new))
    for name, g, w in zip(cache._fields, cache, want):
        assert same_bits(g, w), name
    stored = cache.k.float() * cache.k_scale[..., None, None]
    assert float(stored.abs().max()) == 2.0 ** 17


@pytest.mark.parametrize("new,max_new,length,heads,kv_heads", [(50, 20, 200, 4, 2), (9, 1, 300, 8, 2), (300, 265, 1300, 32, 8), (420, 270, 900, 32, 8)])
@pytest.mark.parametrize("page", [32, 64])
def test_slots_of_tokens_beyond_max_new_may_hold_anything(new, max_new, length, heads, kv_heads, page):
    """Tokens beyond max_new are not stored, so their slots may never have been written: NaN in them reaches no row."""
    dim = 64
    pages = -(-length // page) + 1
    cache = random_cache(pages, kv_heads, page, dim, seed=121)
    table = make_table([length], page, pages, seed=122)
    q = rand(new, heads, dim, seed=123)
    want, tol = ref.attention(q, cache, [0, new], [length], table, dim ** -0.5, max_new=max_new)
    for i in range(length - new + max_new, length):
        for t in (cache.k, cache.v):
            t.view(torch.uint8)[int(table[0, i // page]), :, i % page] = 0x7F
    out = torch.full(q.shape, math.nan, dtype=torch.float16, device=DEV)
    check_attention(rcp.rcp_kv_attention(q, cache, *tensors([0, new], [length], table), max_new=max_new, out=out), want, tol)


def attention_with_polls(polls, q, cache, starts, lengths, table, out, workspace, variant="prompt"):
    """rcp_kv_attention_variant with a limit of its own for the waits"""
    p = lambda t: t.data_ptr()
    pages, kv_heads, page, dim = cache.k.shape
    assert rcp.lib().rcp_kv_attention_variant(
        rcp.binding.ATTENTION_VARIANTS[variant], polls, p(q), q.stride(0), q.shape[0], q.shape[1], kv_heads, dim, dim ** -0.5, p(starts), p(lengths),
        p(table), table.shape[0], table.shape[1], 0, p(cache.k), p(cache.v), p(cache.k_scale), p(cache.v_scale), pages, page, p(out), p(workspace),
        torch.cuda.current_stream().cuda_stream) == 0
    return out


@pytest.mark.parametrize("dim", [64, 128])
def test_attention_that_gave_up_leaves_nan_and_a_status(dim):
    """Waits with no polls give up at once, with one poll some do: rows are NaN or right, the status says so, the kernel ends and the GPU goes on. The next
    calls on the workspace give NaN until it is cleared; sequences of the kernel of few rows are answered all the same."""
    page, heads, kv_heads = 64, 8, 2
    new, lengths = [300, 2, 40], [5000, 700, 300]
    pages = sum(-(-n // page) for n in lengths)
    cache = random_cache(pages, kv_heads, page, dim, seed=131)
    starts = starts_of(new, 1)
    args = tensors(starts, lengths, make_table(lengths, page, pages, seed=132))
    q, ws = rand(sum(new) + 2, heads, dim, seed=133), rcp.make_kv_workspace(DEV)
    mine = slice(starts[0], starts[-1])
    want = rcp.rcp_kv_attention(q, cache, *args, workspace=ws, variant="prompt")
    assert rcp.kv_attention_status(ws) == 0
    out = attention_with_polls(0, q, cache, *args, torch.zeros_like(want), ws)
    assert rcp.kv_attention_status(ws) in (3, 4, 5)
    assert bool(torch.isnan(out[mine]).all()) and not out[:1].any() and not out[-1:].any()
    # status set: in front of every wait
    out = rcp.rcp_kv_attention(q, cache, *args, workspace=ws, variant="prompt")
    assert bool(torch.isnan(out[mine]).all()) and not out[:1].any() and not out[-1:].any() and rcp.kv_attention_status(ws) in (3, 4, 5)
    # one poll a wait
    for _ in range(30):
        ws.zero_()
        out = attention_with_polls(1, q, cache, *args, torch.zeros_like(want), ws)
        bad = torch.isnan(out).any(-1)
        assert torch.equal(out[~bad], want[~bad]) and bool(torch.isnan(out[bad]).all()) and (rcp.kv_attention_status(ws) != 0 or not bool(bad.any()))
    ws.zero_()
    assert torch.equal(rcp.rcp_kv_attention(q, cache, *args, workspace=ws, variant="prompt"), want) and rcp.kv_attention_status(ws) == 0
    # both kernels in one call: rows of a key head up to 24 or 48 are the other kernel's
    heads, kv_heads, new, lengths = 32, 8, [300, 2], [1500, 1400]
    cache = random_cache(48, kv_heads, page, dim, seed=134)
    args = tensors(starts_of(new), lengths, make_table(lengths, page, 48, seed=135))
    q = rand(302, heads, dim, seed=136)
    want = rcp.rcp_kv_attention(q, cache, *args, workspace=ws)
    ws[0] = 3
    out = rcp.rcp_kv_attention(q, cache, *args, workspace=ws)
    assert bool(torch.isnan(out[:300]).all()) and torch.equal(out[300:], want[300:])
    # without a workspace of one's own, too, nothing looks like a result that is none
    assert torch.equal(rcp.rcp_kv_attention(q, cache, *args), want)


def test_calls_without_tokens():
    """A step in which no sequence has a new token: empty tensors, nothing stored, an empty result."""
    cache = random_cache(4, 2, 32, 64, seed=141)
    before = [t.clone() for t in cache]
    args = tensors([0, 0, 0], [20, 0], torch.tensor([[1], [2]], dtype=torch.int32))
    row = torch.empty(0, 8, 64, dtype=torch.float16, device=DEV)
    q, k, v = row[:, :4], row[:, 4:6], row[:, 6:]
    assert rcp.rcp_kv_append(k, v, cache, *args) is None
    for q_out in (None, torch.empty(0, 4, 64, dtype=torch.float16, device=DEV)):
        assert rcp.rcp_kv_append(k, v, cache, *args, rope=ref.rope_table(32, 64), q=q, q_out=q_out).shape == (0, 4, 64)
    for variant in ("auto", "split", "prompt"):
        assert rcp.rcp_kv_attention(q, cache, *args, variant=variant).shape == (0, 4, 64)
    assert all(same_bits(a, b) for a, b in zip(cache, before))
    assert rcp.rcp_kv_attention(rand(3, 4, 64), cache, *args).any().item() is False   # rows, all of them of no sequence

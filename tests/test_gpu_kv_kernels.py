"""Both attention kernels at the sizes and inputs where one of them can go wrong, whichever of them rcp_kv_attention would choose."""
import math
import threading

import pytest
import torch

import kv_reference as ref
import paper_2502_15779_b200 as rcp
from test_gpu_kv import ATTENTION, DEV, check_attention, make_table, rand, random_cache, starts_of, tensors

pytestmark = pytest.mark.gpu
KERNELS = pytest.mark.parametrize("kernel", ["split", "prompt"])


def run(kernel, q, cache, starts, lengths, table, **more):
    ws = rcp.make_kv_workspace(DEV)
    out = more.pop("out", None)
    if out is None:
        out = torch.full(q.shape, math.nan, dtype=torch.float16, device=DEV)
    got = rcp.rcp_kv_attention(q, cache, *tensors(starts, lengths, table), out=out, workspace=ws, variant=kernel, **more)
    assert rcp.kv_attention_status(ws) == 0
    return got


@KERNELS
@pytest.mark.parametrize("new,cached,heads,kv_heads,dim,page", ATTENTION)
def test_all_sizes(kernel, new, cached, heads, kv_heads, dim, page):
    lengths = [n + c for n, c in zip(new, cached)]
    pages = sum(-(-n // page) for n in lengths) + 2
    cache = random_cache(pages, kv_heads, page, dim, seed=21)
    table = make_table(lengths, page, pages, seed=22)
    for b, n in enumerate(lengths):   # slots behind a length may hold anything
        if n % page:
            for t in (cache.k, cache.v):
                t.view(torch.uint8)[int(table[b, n // page]), :, n % page:] = 0x7F
    starts, T = starts_of(new, 1), sum(new) + 4
    row = rand(T, heads + 3, dim, seed=23)
    row[:1], row[-3:] = math.nan, math.nan
    q = row[:, 1:1 + heads]
    check_attention(run(kernel, q, cache, starts, lengths, table), *ref.attention(q, cache, starts, lengths, table, dim ** -0.5))


@KERNELS
@pytest.mark.parametrize("page", [32, 64, 128])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("size", [0.0, 1e-3, 8.0, 300.0])
def test_flat_and_peaked_weights_under_unlike_scales(kernel, page, dim, size):
    """Scores all alike, ordinary, or so large that one key takes all; scales of neighbouring blocks that differ by many powers of two, so that the unit
    of the sums moves up and down."""
    heads, kv_heads, n, new = 8, 2, 700, 150
    pages = -(-n // page) + 1
    cache = random_cache(pages, kv_heads, page, dim, seed=31, lo=-20, hi=-4)
    cache.v_scale[::3] = 2.0 ** -40
    cache.v_scale[1::3] = 2.0 ** -2
    table = make_table([n], page, pages, seed=32)
    q = (rand(new, heads, dim, seed=33).float() * size).half()
    check_attention(run(kernel, q, cache, [0, new], [n], table), *ref.attention(q, cache, [0, new], [n], table, dim ** -0.5))


@KERNELS
@pytest.mark.parametrize("dim", [64, 128])
def test_scales_that_fall_and_rise(kernel, dim):
    """Every block's values 2^3 below, later 2^5 above the one in front: the unit of the sums has to follow, in both directions."""
    page, heads, kv_heads, n, new = 64, 8, 2, 64 * 24, 90
    cache = random_cache(24, kv_heads, page, dim, seed=34)
    table = make_table([n], page, 24, seed=35)
    steps = [9 - 3 * i for i in range(16)] + [-36 + 5 * i for i in range(8)]
    cache.v_scale[table[0].long().to(DEV)] = torch.exp2(torch.tensor(steps, dtype=torch.float32, device=DEV))[:, None]
    for last in (n, 64 * 12 + 5):
        q = rand(new, heads, dim, seed=36)
        check_attention(run(kernel, q, cache, [0, new], [last], table), *ref.attention(q, cache, [0, new], [last], table, dim ** -0.5))


@KERNELS
@pytest.mark.parametrize("new", [1, 40, 300])
def test_missing_pages_and_positions(kernel, new):
    page, dim, heads, kv_heads, width = 32, 64, 4, 2, 12
    cache = random_cache(20, kv_heads, page, dim, seed=41)
    table = torch.full((4, width), -1, dtype=torch.int32)
    table[0, ::2] = torch.arange(6, dtype=torch.int32)       # every second page is missing
    table[1] = 1 << 30                                       # all of them
    table[2] = torch.arange(6, 18, dtype=torch.int32)        # a length below the number of new tokens
    table[3] = torch.arange(6, 18, dtype=torch.int32)        # a length beyond the table
    lengths, starts = [380, 370, max(new - 3, 0), width * page + 2], starts_of([new] * 4)
    q = rand(4 * new, heads, dim, seed=42)
    check_attention(run(kernel, q, cache, starts, lengths, table), *ref.attention(q, cache, starts, lengths, table, dim ** -0.5))


@KERNELS
@pytest.mark.parametrize("new,max_new", [(50, 20), (300, 257)])
def test_more_tokens_than_max_new(kernel, new, max_new):
    page, dim, heads = 64, 64, 4
    lengths, starts = [new + 150, 90], [0, new, new + 3]
    cache = random_cache(12, 2, page, dim, seed=51)
    table = make_table(lengths, page, 12, seed=52)
    q = rand(new + 3, heads, dim, seed=53)
    want, tol = ref.attention(q, cache, starts, lengths, table, 0.1, max_new=max_new)
    check_attention(run(kernel, q, cache, starts, lengths, table, sm_scale=0.1, max_new=max_new), want, tol)


@KERNELS
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new", [1, 9, 100])
def test_a_bad_query_stays_alone_and_a_scale_of_zero_weighs_all_alike(kernel, dim, new):
    page, heads, kv_heads, n = 64, 8, 2, 400
    cache = random_cache(8, kv_heads, page, dim, seed=47)
    table = make_table([n], page, 8, seed=48)
    q = rand(new, heads, dim, seed=49)
    want, tol = ref.attention(q, cache, [0, new], [n], table, dim ** -0.5)
    q[0, 1, 3], q[new // 2, 6, 0], q[new - 1, 7, 9] = math.nan, math.inf, math.nan
    got = run(kernel, q, cache, [0, new], [n], table)
    fine = torch.ones(new, heads, dtype=torch.bool, device=DEV)
    for t, h in ((0, 1), (new // 2, 6), (new - 1, 7)):
        fine[t, h] = False
    assert bool(((got.double() - want).abs() <= tol)[fine].all())
    assert bool(torch.isnan(got[0, 1]).all()) and bool(torch.isnan(got[new - 1, 7]).all())
    q = rand(new, heads, dim, seed=50)
    check_attention(run(kernel, q, cache, [0, new], [n], table, sm_scale=0.0), *ref.attention(q, cache, [0, new], [n], table, 0.0))


@KERNELS
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("new,length", [(1, 5000), (150, 700)])
def test_in_the_place_of_the_queries(kernel, dim, new, length):
    page, heads, kv_heads = 64, 8, 2
    cache = random_cache(90, kv_heads, page, dim, seed=51)
    table = make_table([length], page, 90, seed=52)
    q = rand(new, heads, dim, seed=53)
    want = run(kernel, q.clone(), cache, [0, new], [length], table)
    assert torch.equal(run(kernel, q, cache, [0, new], [length], table, out=q), want)


@KERNELS
@pytest.mark.parametrize("heads,kv_heads", [(40, 1), (200, 1), (65, 1), (128, 2), (3, 3)])
@pytest.mark.parametrize("new", [1, 3])
def test_many_query_heads_of_a_key_head(kernel, heads, kv_heads, new):
    page, dim, lengths = 64, 128, [500, 64, 131]
    cache = random_cache(13, kv_heads, page, dim, seed=44)
    table = make_table(lengths, page, 13, seed=45)
    q, starts = rand(3 * new, heads, dim, seed=46), starts_of([new] * 3)
    check_attention(run(kernel, q, cache, starts, lengths, table), *ref.attention(q, cache, starts, lengths, table, dim ** -0.5))


@KERNELS
@pytest.mark.parametrize("new,cached,heads,kv_heads,dim", [([300], [129], 12, 4, 64), ([65, 1, 129], [3, 50, 200], 8, 2, 128), ([70], [0], 4, 1, 128)])
def test_short_prompts_many_times(kernel, new, cached, heads, kv_heads, dim):
    """A few tiles of keys, whose ends the kernel's warps reach in any order: no wait may give up and every run gives the same."""
    page, lengths = 64, [n + c for n, c in zip(new, cached)]
    pages = sum(-(-n // page) for n in lengths) + 1
    cache = random_cache(pages, kv_heads, page, dim, seed=68)
    args = tensors(starts_of(new), lengths, make_table(lengths, page, pages, seed=69))
    q, ws = rand(sum(new), heads, dim, seed=70), rcp.make_kv_workspace(DEV)
    first = rcp.rcp_kv_attention(q, cache, *args, workspace=ws, variant=kernel)
    bad = torch.zeros((), dtype=torch.int64, device=DEV)
    for _ in range(400):
        bad += (rcp.rcp_kv_attention(q, cache, *args, workspace=ws, variant=kernel) != first).sum()
    assert rcp.kv_attention_status(ws) == 0 and int(bad) == 0


@pytest.mark.parametrize("new,length,heads,kv_heads,choice", [
    (1, 3000, 32, 8, "split"), (12, 3000, 32, 8, "split"), (250, 3000, 32, 8, "split"), (251, 3000, 32, 8, "prompt"), (100, 900, 32, 8, "split"),
    (512, 900, 32, 8, "prompt"), (513, 2000, 32, 8, "prompt"), (2000, 3000, 4, 1, "split"), (2001, 3000, 4, 1, "prompt")])
def test_the_choice_of_one_sequence(new, length, heads, kv_heads, choice):
    """Which kernel a call gets, told by its bits (148 SMs)."""
    if torch.cuda.get_device_properties(0).multi_processor_count != 148:
        pytest.skip("thresholds of 148 SMs")
    page, dim = 64, 64
    pages = -(-length // page)
    cache = random_cache(pages, kv_heads, page, dim, seed=71)
    args = ([0, new], [length], make_table([length], page, pages, seed=72))
    q = rand(new, heads, dim, seed=73)
    split, prompt = run("split", q, cache, *args), run("prompt", q, cache, *args)
    assert not torch.equal(split, prompt)
    assert torch.equal(run("auto", q, cache, *args), split if choice == "split" else prompt)


def test_a_batch_of_prompts_and_single_tokens_gets_both_kernels():
    page, dim, heads, kv_heads = 64, 64, 32, 8
    new, lengths = [400, 1, 13, 12], [2000, 1500, 700, 80]
    pages = sum(-(-n // page) for n in lengths)
    cache = random_cache(pages, kv_heads, page, dim, seed=74)
    args = (starts_of(new), lengths, make_table(lengths, page, pages, seed=75))
    q = rand(sum(new), heads, dim, seed=76)
    prompt, auto = (run(k, q, cache, *args) for k in ("prompt", "auto"))
    # up to 48 rows of a key head are the split kernel's (whose last bits go by how its list of tiles is cut, so by the rest of the batch)
    for part, same in ((slice(0, 400), True), (slice(400, 401), False), (slice(401, 414), True), (slice(414, 426), False)):
        assert torch.equal(auto[part], prompt[part]) == same, part
    check_attention(auto, *ref.attention(q, cache, *args, dim ** -0.5))


def test_calls_from_several_host_threads():
    """Append, attention of both kernels and adapters from four host threads at once, each on a stream and buffers of its own: the results of calls in a row."""
    page, dim, heads, kv_heads = 64, 64, 32, 8
    jobs = []
    for i in range(4):
        new, lengths = ([1, 1, 1] if i % 2 else [300, 2, 9]), [2500 + 100 * i, 70, 300]
        pages = sum(-(-n // page) for n in lengths)
        cache = random_cache(pages, kv_heads, page, dim, seed=81 + i)
        args = tensors(starts_of(new), lengths, make_table(lengths, page, pages, seed=82 + i))
        T, M, N, rank = sum(new), (7, 97)[i % 2], 520, 16
        row = rand(T, heads + 2 * kv_heads, dim, seed=83 + i)
        x, a, b = rand(M, 512, seed=84 + i), rand(3, rank, 512, seed=85, std=0.04), rand(3, N, rank, seed=86)
        jobs.append(dict(cache=cache, args=args, row=row, rope=ref.rope_table(args[2].shape[1] * page, dim), x=x, a=a, b=b, q=torch.empty(T, heads, dim, dtype=torch.float16, device=DEV),
                         adapter=torch.arange(M, dtype=torch.int32, device=DEV) % 4 - 1, scaling=torch.ones(3, device=DEV), out=torch.empty(T, heads, dim, dtype=torch.float16, device=DEV),
                         y=torch.empty(M, N, dtype=torch.float16, device=DEV), ws=rcp.make_kv_workspace(DEV), lws=rcp.make_lora_workspace(M, rank, DEV), stream=torch.cuda.Stream()))

    def step(j):
        row = j["row"]
        rcp.rcp_kv_append(row[:, heads:heads + kv_heads], row[:, heads + kv_heads:], j["cache"], *j["args"], rope=j["rope"], q=row[:, :heads], q_out=j["q"])
        rcp.rcp_kv_attention(j["q"], j["cache"], *j["args"], out=j["out"], workspace=j["ws"])
        rcp.rcp_lora_add(j["x"], j["a"], j["b"], j["adapter"], j["scaling"], y=j["y"], workspace=j["lws"])

    for j in jobs:
        step(j)
        j["want"] = j["out"].clone(), j["y"].clone(), [t.clone() for t in j["cache"]]
        j["out"].zero_(), j["y"].zero_()
    torch.cuda.synchronize()
    errors = []

    def work(j):
        try:
            with torch.cuda.stream(j["stream"]):
                for _ in range(50):
                    step(j)
        except Exception as e:   # (an assertion in a thread would be lost)
            errors.append(e)

    threads = [threading.Thread(target=work, args=(j,)) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors, errors
    for j in jobs:
        out, y, cache = j["want"]
        assert torch.equal(j["out"], out) and torch.equal(j["y"], y) and rcp.kv_attention_status(j["ws"]) == 0
        assert all(torch.equal(g.view(torch.uint8), w.view(torch.uint8)) for g, w in zip(j["cache"], cache))

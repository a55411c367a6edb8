"""rcp_lora_add on the GPU against 64 bits, and a decoder layer's calls one after the other as a decode step makes them."""
import math

import pytest
import torch

import kv_reference as ref
import paper_2502_15779_b200 as rcp
from gen import synth

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def rand(*shape, seed=0, std=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randn(*shape, generator=g, device=DEV) * std).half()


def case(M, N, K, rank, adapters, seed=0):
    x = rand(M, K, seed=seed)
    a, b = rand(adapters, rank, K, seed=seed + 1, std=K ** -0.5), rand(adapters, N, rank, seed=seed + 2, std=0.5)
    base = rand(M, N, seed=seed + 3)
    g = torch.Generator(device=DEV).manual_seed(seed + 4)
    adapter = torch.randint(-1, adapters + 1, (M,), generator=g, device=DEV, dtype=torch.int32)
    adapter[0] = adapters - 1
    scaling = torch.rand(adapters, generator=g, device=DEV) * 2 - 0.5
    return x, a, b, adapter, scaling, base


def check(got, want, tol):
    off = (got.double() - want).abs()
    assert bool((off <= tol).all()), f"off by {float((off / tol).max()):.3f} of the bound"


SHAPES = [(1, 64, 64, 8, 1), (1, 10240, 8192, 16, 8), (1, 1, 128, 8, 3), (2, 33, 192, 24, 2), (3, 5003, 2624, 8, 2), (7, 300, 64, 128, 5),
          (16, 6144, 4096, 32, 48), (16, 999, 14336, 16, 1), (17, 130, 320, 40, 4), (31, 4097, 1088, 64, 3), (33, 64, 65536, 8, 2),
          (64, 513, 512, 16, 64), (65, 257, 1024, 128, 2), (100, 2048, 2048, 16, 3), (300, 1025, 704, 48, 7), (1000, 129, 256, 72, 2), (97, 546, 2944, 56, 4),
          (134, 704, 2880, 24, 9), (1100, 2057, 640, 112, 3)]


@pytest.mark.parametrize("M,N,K,rank,adapters", SHAPES)
@pytest.mark.parametrize("form", ["base", "none", "in place"])
def test_against_64_bits(M, N, K, rank, adapters, form):
    x, a, b, adapter, scaling, base = case(M, N, K, rank, adapters, seed=M + N)
    want, tol = ref.lora(x, a, b, adapter, scaling, None if form == "none" else base)
    y = base.clone() if form == "in place" else None
    got = rcp.rcp_lora_add(x, a, b, adapter, scaling, base=y if form == "in place" else base if form == "base" else None, y=y)
    check(got, want, tol)
    if form == "in place":
        assert got is y


@pytest.mark.parametrize("M", [1, 16, 200])
def test_requests_in_order_strided_rows_and_no_adapters(M):
    x, a, b, _, scaling, base = case(M, 777, 512, 16, 3, seed=5)
    wide = rand(M, 1000, seed=6)
    wide[:, 8:520] = x
    for adapter in (torch.arange(M, device=DEV, dtype=torch.int32) * 3 // M, torch.full((M,), -1, dtype=torch.int32, device=DEV),
                    torch.full((M,), 2, dtype=torch.int32, device=DEV), torch.full((M,), 1 << 30, dtype=torch.int32, device=DEV)):
        want, tol = ref.lora(x, a, b, adapter, scaling, base)
        check(rcp.rcp_lora_add(wide[:, 8:520], a, b, adapter, scaling, base=base), want, tol)


@pytest.mark.parametrize("M,N", [(3, 512), (100, 512), (130, 77)])
def test_results_that_start_between_sixteen_bytes(M, N):
    x, a, b, adapter, scaling, base = case(M, N, 256, 16, 3, seed=31)
    odd = [torch.empty(M * N + 1, dtype=torch.float16, device=DEV)[1:].view(M, N) for _ in range(2)]
    odd[0].copy_(base)
    want, tol = ref.lora(x, a, b, adapter, scaling, base)
    check(rcp.rcp_lora_add(x, a, b, adapter, scaling, base=odd[0], y=odd[1]), want, tol)
    check(rcp.rcp_lora_add(x, a, b, adapter, scaling, base=base, y=odd[1]), want, tol)
    check(rcp.rcp_lora_add(x, a, b, adapter, scaling, base=odd[0], y=odd[0]), want, tol)


def test_a_large_token_beside_a_small_one():
    """z of the prompt form is scaled a token: large and tiny activations side by side, sums beyond fp16's range."""
    M, N, K, R = 80, 200, 512, 32
    x, a, b, adapter, scaling, _ = case(M, N, K, R, 2, seed=33)
    x[::3] *= 2000.0
    x[1::3] *= 1e-4
    a *= 30.0
    b *= 1e-3
    want, tol = ref.lora(x, a, b, adapter, scaling, None)
    check(rcp.rcp_lora_add(x, a, b, adapter, scaling), want, tol)


def test_calls_on_several_streams():
    sets = []
    for i, (M, N) in enumerate(((1, 4096), (16, 1000), (200, 700))):
        args = case(M, N, 1024, 16, 4, seed=60 + i)
        sets.append((args, rcp.rcp_lora_add(*args[:5], base=args[5]), rcp.make_lora_workspace(M, 16, DEV), torch.empty(M, N, dtype=torch.float16, device=DEV),
                     torch.cuda.Stream()))
    torch.cuda.synchronize()
    for _ in range(10):
        for args, _, ws, y, st in sets:
            with torch.cuda.stream(st):
                rcp.rcp_lora_add(*args[:5], base=args[5], y=y, workspace=ws)
    torch.cuda.synchronize()
    for _, want, _, y, _ in sets:
        assert torch.equal(y, want)


def test_a_bad_number_stays_with_its_token():
    """NaN and infinity in one token's activations or one adapter's weights reach no other token, and a token without an adapter keeps
    its base bit for bit."""
    x, a, b, adapter, scaling, base = case(40, 200, 256, 16, 4, seed=9)
    adapter = torch.arange(40, device=DEV, dtype=torch.int32) % 5 - 1
    x[3, 7], x[8, 9], a[2, 3, 4] = math.nan, math.inf, math.nan
    got = rcp.rcp_lora_add(x, a, b, adapter, scaling, base=base)
    clean = [i for i in range(40) if i not in (3, 8) and int(adapter[i]) != 2]
    want, tol = ref.lora(x[clean], a[[0, 1, 3]], b[[0, 1, 3]], torch.tensor([{-1: -1, 0: 0, 1: 1, 3: 2}[int(adapter[i])] for i in clean], device=DEV),
                         scaling[[0, 1, 3]], base[clean])
    check(got[clean], want, tol)
    none = adapter < 0
    assert torch.equal(got[none], base[none])


def test_results_repeat_and_the_workspace_is_ready_again():
    for M, N, K in ((1, 4096, 4096), (16, 6144, 4096), (150, 1000, 2048)):
        x, a, b, adapter, scaling, base = case(M, N, K, 16, 4, seed=M)
        ws = rcp.make_lora_workspace(M, 16, DEV)
        first = rcp.rcp_lora_add(x, a, b, adapter, scaling, base=base, workspace=ws)
        rcp.rcp_lora_add(rand(M, K, seed=77), a, b, adapter, scaling, base=base, workspace=ws)
        for _ in range(20):
            assert torch.equal(rcp.rcp_lora_add(x, a, b, adapter, scaling, base=base, workspace=ws), first)


def test_captured_call_follows_its_inputs():
    x, a, b, adapter, scaling, base = case(9, 500, 1024, 32, 6, seed=3)
    y, ws = torch.empty_like(base), rcp.make_lora_workspace(9, 32, DEV)
    rcp.rcp_lora_add(x, a, b, adapter, scaling, base=base, y=y, workspace=ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rcp.rcp_lora_add(x, a, b, adapter, scaling, base=base, y=y, workspace=ws)
    for i in range(5):
        x.copy_(rand(9, 1024, seed=200 + i))
        adapter.copy_((torch.arange(9, device=DEV, dtype=torch.int32) * (i + 1)) % 7 - 1)
        graph.replay()
        check(y, *ref.lora(x, a, b, adapter, scaling, base))


def test_adapters_beyond_four_gibibytes():
    """Offsets into the adapters pass 32 bits."""
    M, N, K, rank = 3, 65536, 64, 128
    adapters = (1 << 32) // (2 * N * rank) + 3
    a = torch.zeros(adapters, rank, K, dtype=torch.float16, device=DEV)
    b = torch.zeros(adapters, N, rank, dtype=torch.float16, device=DEV)
    assert b.numel() * 2 > 1 << 32
    x = rand(M, K, seed=1)
    adapter = torch.tensor([adapters - 1, 0, adapters - 2], dtype=torch.int32, device=DEV)
    for i in adapter.tolist():
        a[i], b[i] = rand(rank, K, seed=10 + i), rand(N, rank, seed=20 + i)
    scaling = torch.ones(adapters, device=DEV)
    mine = adapter.long()
    want, tol = ref.lora(x, a[mine], b[mine], torch.arange(3, device=DEV), torch.ones(3, device=DEV), None)
    check(rcp.rcp_lora_add(x, a, b, adapter, scaling), want, tol)


@pytest.mark.parametrize("captured", [False, True])
def test_attention_half_of_a_decoder_layer(captured):
    """qkv projection (2-bit weights) with adapters, append with rotation, attention, output projection with adapters: two decode steps of a small
    batch, eager or one captured graph, each step against the plain forms fed with the library's own intermediate results."""
    B, heads, kv_heads, dim, page, K, rank = 5, 8, 2, 64, 32, 512, 16
    Nq = (heads + 2 * kv_heads) * dim
    layers = {}
    for name, N in (("qkv", Nq), ("o", K)):
        codes, lut = synth.make_layer(N, 512, 512, "uniform", 3 + N, DEV)
        layers[name] = dict(words=rcp.rcp_pack_weights(codes), lut=lut, N=N, a=rand(3, rank, 512, seed=N, std=0.04), b=rand(3, N, rank, seed=N + 1, std=0.05),
                            xq=torch.empty(B, 256, dtype=torch.uint8, device=DEV), scale=torch.empty(B, dtype=torch.float16, device=DEV),
                            ws=rcp.make_workspace(B, N, 512, DEV), lws=rcp.make_lora_workspace(B, rank, DEV),
                            plain=torch.empty(B, N, dtype=torch.float16, device=DEV), y=torch.empty(B, N, dtype=torch.float16, device=DEV))
    adapter = torch.tensor([0, -1, 2, 1, 0], dtype=torch.int32, device=DEV)
    scaling = torch.tensor([1.0, 0.5, 2.0], device=DEV)
    cache = rcp.make_kv_cache(20, kv_heads, dim, page, DEV)
    table = torch.arange(20, dtype=torch.int32).reshape(5, 4)
    lengths_now = [1, 32, 33, 100, 2]
    starts = torch.arange(B + 1, dtype=torch.int32, device=DEV)
    lengths, tab = torch.tensor(lengths_now, dtype=torch.int32, device=DEV), table.to(DEV)
    # what the sequences hold already
    held = [n - 1 for n in lengths_now]
    hs = torch.tensor([0] + held, dtype=torch.int32).cumsum(0).int()
    rcp.rcp_kv_append(rand(sum(held), kv_heads, dim, seed=1), rand(sum(held), kv_heads, dim, seed=2), cache, hs.to(DEV),
                      torch.tensor(held, dtype=torch.int32, device=DEV), tab)
    rope = ref.rope_table(4 * page, dim)
    x = rand(B, K, seed=4)
    q_rot, att = (torch.empty(B, heads, dim, dtype=torch.float16, device=DEV) for _ in range(2))
    kws = rcp.make_kv_workspace(DEV)

    def linear(layer, x):
        L = layers[layer]
        rcp.rcp_linear_w2a4(x, 512, 1.0, L["words"], L["lut"], y=L["plain"], xq=L["xq"], scale=L["scale"], workspace=L["ws"])
        return rcp.rcp_lora_add(x, L["a"], L["b"], adapter, scaling, base=L["plain"], y=L["y"], workspace=L["lws"])

    def step():
        row = linear("qkv", x).view(B, heads + 2 * kv_heads, dim)
        rcp.rcp_kv_append(row[:, heads:heads + kv_heads], row[:, heads + kv_heads:], cache, starts, lengths, tab, rope=rope, q=row[:, :heads],
                          q_out=q_rot, max_new=1)
        rcp.rcp_kv_attention(q_rot, cache, starts, lengths, tab, max_new=1, out=att, workspace=kws)
        linear("o", att.view(B, heads * dim))

    run = step
    if captured:
        saved = [t.clone() for t in cache]
        step()
        for t, w in zip(cache, saved):
            t.view(torch.uint8).copy_(w.view(torch.uint8))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        run = graph.replay
    for i in range(2):
        at = [n + i for n in lengths_now]
        lengths.copy_(torch.tensor(at, dtype=torch.int32))
        x.copy_(rand(B, K, seed=40 + i))
        before = rcp.KvCache(*(t.clone() for t in cache))
        run()
        q, o = layers["qkv"], layers["o"]
        check(q["y"], *ref.lora(x, q["a"], q["b"], adapter, scaling, q["plain"]))
        row = q["y"].view(B, heads + 2 * kv_heads, dim)
        want, want_q = ref.append(before, row[:, heads:heads + kv_heads], row[:, heads + kv_heads:], list(range(B + 1)), at, table, rope, False,
                                  row[:, :heads])
        assert torch.equal(q_rot, want_q)
        assert all(torch.equal(g.view(torch.uint8), w.view(torch.uint8)) for g, w in zip(cache, want))
        out, tol = ref.attention(q_rot, cache, list(range(B + 1)), at, table, dim ** -0.5)
        check(att, out, tol)
        check(o["y"], *ref.lora(att.view(B, -1), o["a"], o["b"], adapter, scaling, o["plain"]))


@pytest.mark.parametrize("M,N", [(64, 200), (65, 200), (130, 201)])
def test_ranks_of_unlike_size(M, N):
    """Rows of a whose z differ by 2^15 to 2^24 within a token, b scaled the other way: the small z make up as much of the result as the large ones, whether
    the tokens are few or many."""
    K, R = 512, 32
    x, a, b, adapter, scaling, _ = case(M, N, K, R, 2, seed=35)
    for r, e in enumerate((0, -15, -8, -24, 0, -20, -12, -18) * 4):
        a[:, r] = (a[:, r].float() * 2.0 ** (10 + e)).half()
        b[:, :, r] = (b[:, :, r].float() * 2.0 ** (-14 - e)).half()
    want, tol = ref.lora(x, a, b, adapter, scaling, None)
    check(rcp.rcp_lora_add(x, a, b, adapter, scaling), want, tol)


@pytest.mark.parametrize("M", [64, 65, 300])
def test_one_workspace_for_adapters_and_attention(M):
    """One zero-filled buffer, large enough for each, for the calls of a stream in turn: what the adapters leave there is not taken for attention's status
    or counters, and the other way round."""
    heads, kv_heads, dim, page = 32, 8, 64, 64
    x, a, b, adapter, scaling, base = case(M, 300, 512, 32, 5, seed=41)
    cache = rcp.make_kv_cache(300, kv_heads, dim, page, DEV)
    cases = []
    for lengths, new in (([9000], 1), ([1500, 40], 300), ([5000, 700, 3], 1)):
        lengths = [max(n, new) for n in lengths]
        need = [-(-n // page) for n in lengths]
        table = torch.full((len(lengths), max(need)), -1, dtype=torch.int32)
        for i, n in enumerate(need):
            table[i, :n] = torch.arange(n) + sum(need[:i])
        starts = torch.arange(len(lengths) + 1, dtype=torch.int32, device=DEV) * new
        cases.append((rand(len(lengths) * new, heads, dim, seed=42), cache, starts, torch.tensor(lengths, dtype=torch.int32, device=DEV), table.to(DEV)))
    ws = torch.zeros(max(rcp.make_kv_workspace(DEV).numel(), rcp.make_lora_workspace(M, 32, DEV).numel()), dtype=torch.uint8, device=DEV)
    k = rand(9000, kv_heads, dim, seed=43)
    rcp.rcp_kv_append(k, k, cache, *(torch.tensor(t, dtype=torch.int32, device=DEV) for t in ([0, 9000], [9000], [list(range(141))])))
    want_y = rcp.rcp_lora_add(x, a, b, adapter, scaling, base=base)
    wants = [rcp.rcp_kv_attention(*c) for c in cases]
    for _ in range(3):
        for c, want in zip(cases, wants):
            assert torch.equal(rcp.rcp_lora_add(x, a, b, adapter, scaling, base=base, workspace=ws), want_y)
            assert torch.equal(rcp.rcp_kv_attention(*c, workspace=ws), want)
    assert not ws[:256].any()


@pytest.mark.parametrize("M", [40, 97, 200])
@pytest.mark.parametrize("N", [200, 201])
@pytest.mark.parametrize("order", ["mixed", "runs"])
def test_a_bad_number_stays_with_its_token_or_adapter(M, N, order):
    """Few tokens and tiles of many, rows on 16 bytes and off them: NaN and infinity in a token's activations or an adapter's a or b reach no other request, rows
    without an adapter keep their base bit for bit, and nothing of an earlier call full of NaN is left in the workspace."""
    K, R, L = 256, 24, 5
    x, a, b, _, scaling, base = case(M, N, K, R, L, seed=9)
    i = torch.arange(M, device=DEV, dtype=torch.int32)
    adapter = i % (L + 1) - 1 if order == "mixed" else (i * (L + 1) // M).int() - 1
    ws = rcp.make_lora_workspace(M, R, DEV)
    nan = torch.full_like(x, math.nan)
    rcp.rcp_lora_add(nan, a, b, (i % L).int(), scaling, base=base, workspace=ws)
    bad_tokens = [int(t) for t in torch.nonzero(adapter == 0)[:, 0].tolist()[1:3]]
    x[bad_tokens[0], 7], x[bad_tokens[1], 9] = math.nan, math.inf
    a[2, 3, 4], b[3, :, 5] = math.nan, math.nan
    bad = (adapter == 2) | (adapter == 3)
    bad[bad_tokens] = True
    keep = torch.nonzero(~bad)[:, 0]
    ok = [0, 1, 4]
    names = torch.full((L + 1,), -1, device=DEV, dtype=torch.int32)
    names[ok] = torch.arange(3, device=DEV, dtype=torch.int32)
    for form in ("base", "none", "in place"):
        y = base.clone() if form == "in place" else None
        got = rcp.rcp_lora_add(x, a, b, adapter, scaling, base=y if y is not None else base if form == "base" else None, y=y, workspace=ws)
        want, tol = ref.lora(x[keep], a[ok], b[ok], names[adapter[keep].long()], scaling[ok], None if form == "none" else base[keep])
        check(got[keep], want, tol)
        none = adapter < 0
        assert torch.equal(got[none].view(torch.int16), (torch.zeros_like(base) if form == "none" else base)[none].view(torch.int16))


@pytest.mark.parametrize("M,adapters", [(65, 48), (130, 64), (200, 200)])
def test_many_tokens_with_adapters_of_their_own(M, adapters):
    """A batch of more tokens than the kernel for few takes, nearly every one with another adapter."""
    x, a, b, adapter, scaling, base = case(M, 640, 512, 16, adapters, seed=51)
    if M == adapters:
        adapter = torch.randperm(M, device=DEV).int()
    check(rcp.rcp_lora_add(x, a, b, adapter, scaling, base=base), *ref.lora(x, a, b, adapter, scaling, base))


def test_one_workspace_for_a_layer():
    """Linear calls, adapters of few and many tokens and attention of both kernels in turn on one zero-filled buffer."""
    heads, kv_heads, dim, page, K, N, rank = 8, 2, 64, 64, 512, 768, 16
    codes, lut = synth.make_layer(N, K, K, "uniform", 5, DEV)
    words = rcp.rcp_pack_weights(codes)
    cache = rcp.make_kv_cache(20, kv_heads, dim, page, DEV)
    k = rand(1200, kv_heads, dim, seed=1)
    table = torch.arange(19, dtype=torch.int32, device=DEV)[None]
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)
    rcp.rcp_kv_append(k, k, cache, i32(0, 1200), i32(1200), table)

    def linear(x, **ws):
        n = len(x)
        xq, scale = torch.empty(n, K // 2, dtype=torch.uint8, device=DEV), torch.empty(n, dtype=torch.float16, device=DEV)
        return rcp.rcp_linear_w2a4(x, K, 1.0, words, lut, xq=xq, scale=scale, **ws)

    def calls(**ws):
        out = []
        for M, new in ((1, 1), (16, 300), (70, 40)):
            x, a, b, adapter, scaling, _ = case(M, N, K, rank, 4, seed=M)
            base = torch.cat([linear(x[i:i + 16], **ws) for i in range(0, M, 16)])
            out.append(rcp.rcp_lora_add(x, a, b, adapter, scaling, base=base, **ws))
            for variant in ("split", "prompt"):
                out.append(rcp.rcp_kv_attention(rand(new, heads, dim, seed=new), cache, i32(0, new), i32(1200), table, variant=variant, **ws))
        return out

    one = torch.zeros(8 << 20, dtype=torch.uint8, device=DEV)
    want = calls()
    for _ in range(2):
        assert all(torch.equal(g, w) for g, w in zip(calls(workspace=one), want))
    assert not one[:256].any()

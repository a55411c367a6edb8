"""What the cache, attention and adapter calls refuse: by the library's checks (host only, no GPU) and by the binding's."""
import ctypes as C

import pytest
import torch

import paper_2502_15779_b200 as rcp

NULL, SHAPE, ALIGN, WORKSPACE, LIMIT = -1, -2, -3, -5, -8
P = 1 << 20   # an address that is never followed: every call below is refused before anything is launched


@pytest.fixture(scope="module")
def L():
    from paper_2502_15779_b200 import build
    build.build()
    return rcp.lib()


def call(fn, spec, **change):
    args = dict(spec)
    assert set(change) <= set(args), change
    args.update(change)
    return fn(*[C.c_void_p(v) if isinstance(v, str) is False and k in POINTERS else v for k, v in args.items()])


POINTERS = {"q", "k", "v", "rope", "starts", "lengths", "table", "k_cache", "v_cache", "k_scale", "v_scale", "q_out", "out", "workspace", "stream",
            "x", "a", "b", "adapter", "scaling", "base", "y"}
APPEND = dict(q=P, qs=512, k=P, ks=128, v=P, vs=128, tokens=0, heads=8, kv_heads=2, dim=64, rope=P, positions=256, rot=64, interleaved=0, starts=P,
              lengths=P, table=P, seqs=2, width=4, max_new=0, k_cache=P, v_cache=P, k_scale=P, v_scale=P, pages=9, page=64, q_out=P, stream=None)
ATTENTION = dict(q=P, qs=512, tokens=0, heads=8, kv_heads=2, dim=64, sm=0.125, starts=P, lengths=P, table=P, seqs=2, width=4, max_new=0, k_cache=P,
                 v_cache=P, k_scale=P, v_scale=P, pages=9, page=64, out=P, workspace=P, stream=None)
LORA = dict(x=P, xs=128, a=P, b=P, adapter=P, scaling=P, base=P, M=2, N=5, K=128, rank=16, adapters=3, y=P, workspace=P, stream=None)


def test_calls_without_tokens_are_fine(L):
    assert call(L.rcp_kv_append, APPEND) == 0
    assert call(L.rcp_kv_append, APPEND, q=None, q_out=None, rope=None) == 0
    assert call(L.rcp_kv_attention, ATTENTION) == 0


CACHE = [(NULL, dict(starts=None)), (NULL, dict(lengths=None)), (NULL, dict(table=None)), (NULL, dict(k_cache=None)), (NULL, dict(v_scale=None)),
         (SHAPE, dict(dim=96)), (SHAPE, dict(page=16)), (SHAPE, dict(page=96)), (SHAPE, dict(page=256)), (SHAPE, dict(heads=7)), (SHAPE, dict(heads=0)),
         (SHAPE, dict(kv_heads=0)), (SHAPE, dict(heads=1026, qs=1026 * 64)), (SHAPE, dict(tokens=-1)), (SHAPE, dict(seqs=0)), (SHAPE, dict(width=0)),
         (SHAPE, dict(pages=0)), (SHAPE, dict(max_new=-1)), (LIMIT, dict(seqs=1025)), (LIMIT, dict(tokens=(1 << 20) + 1)),
         (LIMIT, dict(width=(1 << 24) // 64 + 1)), (ALIGN, dict(k_cache=P + 8)), (ALIGN, dict(v_cache=P + 1)), (ALIGN, dict(starts=P + 2)),
         (ALIGN, dict(lengths=P + 1)), (ALIGN, dict(table=P + 2)), (ALIGN, dict(k_scale=P + 2)), (ALIGN, dict(v_scale=P + 1)),
         (SHAPE, dict(tokens=2, qs=504)), (SHAPE, dict(qs=516)), (SHAPE, dict(qs=-512)), (ALIGN, dict(q=P + 8))]


@pytest.mark.parametrize("status,change", CACHE + [
    (NULL, dict(k=None)), (NULL, dict(v=None)), (NULL, dict(q_out=None)), (NULL, dict(rope=None)), (SHAPE, dict(rot=72)), (SHAPE, dict(rot=80)),
    (SHAPE, dict(rot=0)), (SHAPE, dict(rot=24)), (SHAPE, dict(positions=255)), (SHAPE, dict(tokens=2, ks=120)), (SHAPE, dict(vs=132)),
    (ALIGN, dict(k=P + 8)), (ALIGN, dict(v=P + 2)), (ALIGN, dict(rope=P + 8)), (ALIGN, dict(q_out=P + 8))])
def test_append_refuses(L, status, change):
    assert call(L.rcp_kv_append, APPEND, **change) == status


@pytest.mark.parametrize("status,change", CACHE + [
    (NULL, dict(q=None)), (NULL, dict(out=None)), (WORKSPACE, dict(workspace=None)), (ALIGN, dict(workspace=P + 8)), (ALIGN, dict(out=P + 2)),
    (SHAPE, dict(sm=float("nan"))), (SHAPE, dict(sm=float("inf"))), (SHAPE, dict(sm=-1.0))])
def test_attention_refuses(L, status, change):
    assert call(L.rcp_kv_attention, ATTENTION, **change) == status


@pytest.mark.parametrize("status,change", [
    (NULL, dict(x=None)), (NULL, dict(a=None)), (NULL, dict(b=None)), (NULL, dict(adapter=None)), (NULL, dict(scaling=None)), (NULL, dict(y=None)),
    (WORKSPACE, dict(workspace=None)), (SHAPE, dict(M=0)), (SHAPE, dict(M=65536)), (SHAPE, dict(N=0)), (SHAPE, dict(K=96)), (SHAPE, dict(K=0)),
    (SHAPE, dict(K=65600, xs=65600)), (SHAPE, dict(rank=0)), (SHAPE, dict(rank=12)), (SHAPE, dict(rank=136)), (SHAPE, dict(adapters=0)),
    (SHAPE, dict(xs=120)), (SHAPE, dict(xs=132)), (ALIGN, dict(x=P + 8)), (ALIGN, dict(a=P + 8)), (ALIGN, dict(b=P + 2)), (ALIGN, dict(y=P + 1)),
    (ALIGN, dict(base=P + 1)), (ALIGN, dict(workspace=P + 4)), (ALIGN, dict(adapter=P + 1)), (ALIGN, dict(scaling=P + 2))])
def test_lora_refuses(L, status, change):
    assert call(L.rcp_lora_add, LORA, **change) == status


def test_workspace_sizes(L):
    assert rcp.lib().rcp_kv_attention_workspace_bytes() >= 16
    assert L.rcp_lora_workspace_bytes(0, 16) == L.rcp_lora_workspace_bytes(5, 12) == L.rcp_lora_workspace_bytes(70000, 16) == 0
    assert L.rcp_lora_workspace_bytes(5, 16) >= 16


def test_binding_refuses_host_tensors_and_other_types(L):
    cache = rcp.make_kv_cache(2, 1, 64, 32, "cpu")
    x = torch.zeros(1, 1, 64, dtype=torch.float16)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError, match="k: expected a CUDA tensor"):
        rcp.rcp_kv_append(x, x, cache, i, i[:1], i[None])
    with pytest.raises(TypeError, match="q: expected a CUDA tensor"):
        rcp.rcp_kv_attention(x, cache, i, i[:1], i[None])
    with pytest.raises(TypeError, match="x: expected a CUDA tensor"):
        rcp.rcp_lora_add(x[0], x, x, i[:1], torch.ones(1))


def test_binding_refuses_a_wrong_number_of_arguments(L):
    m = rcp.binding._native()
    for fn in (m.kv_append, m.kv_attention, m.lora_add):
        with pytest.raises(TypeError, match="expected .* arguments"):
            fn(1, 2)


@pytest.mark.gpu
def test_binding_refuses_wrong_shapes_on_the_gpu(L):
    dev = "cuda:0"
    cache = rcp.make_kv_cache(2, 2, 64, 32, dev)
    x = torch.zeros(3, 2, 64, dtype=torch.float16, device=dev)
    starts, lengths, table = (torch.tensor(t, dtype=torch.int32, device=dev) for t in ([0, 3], [3], [[0]]))
    ok = (starts, lengths, table)
    rcp.rcp_kv_append(x, x, cache, *ok)
    with pytest.raises(TypeError, match="without gaps"):
        rcp.rcp_kv_append(x.transpose(0, 1), x, cache, *ok)
    with pytest.raises(TypeError, match="float16"):
        rcp.rcp_kv_append(x.float(), x, cache, *ok)
    with pytest.raises(ValueError, match="k, v and the cache"):
        rcp.rcp_kv_append(x, x[:2], cache, *ok)
    with pytest.raises(ValueError, match="k, v and the cache"):
        rcp.rcp_kv_append(x[:, :1], x[:, :1], cache, *ok)
    with pytest.raises(ValueError, match="starts"):
        rcp.rcp_kv_append(x, x, cache, starts[:1], lengths, table)
    with pytest.raises(TypeError, match="block_table"):
        rcp.rcp_kv_append(x, x, cache, starts, lengths, table.long())
    with pytest.raises(ValueError, match="the cache's codes"):
        rcp.rcp_kv_append(x, x, cache._replace(v=cache.v[:1]), *ok)
    with pytest.raises(ValueError, match="rope"):
        rcp.rcp_kv_append(x, x, cache, *ok, rope=torch.zeros(32, 32, device=dev))
    with pytest.raises(rcp.RcpError, match="null"):
        rcp.rcp_kv_append(x, x, cache, *ok, q=x)                       # queries without a rotation
    with pytest.raises(ValueError, match="q, k and v"):
        rcp.rcp_kv_append(x, x, cache, *ok, rope=torch.zeros(32, 32, 2, device=dev), q=x[:2])
    with pytest.raises(ValueError, match="q_out"):
        rcp.rcp_kv_append(x, x, cache, *ok, rope=torch.zeros(32, 32, 2, device=dev), q=x, q_out=x[:2])
    with pytest.raises(rcp.RcpError, match="shape"):
        rcp.rcp_kv_append(x, x, cache, *ok, rope=torch.zeros(31, 32, 2, device=dev))
    with pytest.raises(ValueError, match="q and the cache"):
        rcp.rcp_kv_attention(torch.zeros(3, 4, 128, dtype=torch.float16, device=dev), cache, *ok)
    with pytest.raises(rcp.RcpError, match="shape"):
        rcp.rcp_kv_attention(torch.zeros(3, 3, 64, dtype=torch.float16, device=dev), cache, *ok)
    with pytest.raises(ValueError, match="workspace"):
        rcp.rcp_kv_attention(x, cache, *ok, workspace=torch.zeros(8, dtype=torch.uint8, device=dev))
    with pytest.raises(ValueError, match="out"):
        rcp.rcp_kv_attention(x, cache, *ok, out=x[:2])
    a, b = torch.zeros(2, 8, 64, dtype=torch.float16, device=dev), torch.zeros(2, 5, 8, dtype=torch.float16, device=dev)
    adapter, scaling = torch.zeros(3, dtype=torch.int32, device=dev), torch.ones(2, device=dev)
    xx = x[:, 0]
    assert rcp.rcp_lora_add(xx, a, b, adapter, scaling).shape == (3, 5)
    for bad in ((xx, a, b[:, :, :4].contiguous(), adapter, scaling), (xx, a[:1], b, adapter, scaling), (xx, a, b, adapter[:2], scaling),
                (xx, a, b, adapter, scaling[:1])):
        with pytest.raises(ValueError, match="x, a, b, adapter and scaling"):
            rcp.rcp_lora_add(*bad)
    with pytest.raises(ValueError, match="base"):
        rcp.rcp_lora_add(xx, a, b, adapter, scaling, base=torch.zeros(2, 5, dtype=torch.float16, device=dev))


VARIANT = -7


@pytest.mark.parametrize("status,change", [
    (VARIANT, dict(variant=3)), (VARIANT, dict(variant=-1)), (SHAPE, dict(polls=-2)), (SHAPE, dict(polls=(1 << 18) + 1)),
    # more rows, or more tiles of them, than the split kernel counts
    (VARIANT, dict(variant=1, tokens=15001, qs=512)), (VARIANT, dict(variant=1, tokens=1 << 20, max_new=15001, qs=512)),
    (VARIANT, dict(variant=1, tokens=1536, heads=1024, kv_heads=1024, qs=65536)),
    (NULL, dict(q=None)), (WORKSPACE, dict(workspace=None)), (SHAPE, dict(dim=96))])
def test_attention_of_a_chosen_kernel_refuses(L, status, change):
    assert call(L.rcp_kv_attention_variant, dict(variant=0, polls=-1, **ATTENTION), **change) == status


def test_binding_refuses_an_unknown_attention_kernel(L):
    x = torch.zeros(1, 1, 64, dtype=torch.float16)
    with pytest.raises(KeyError):
        rcp.rcp_kv_attention(x, rcp.make_kv_cache(2, 1, 64, 32, "cpu"), x, x, x, out=x, workspace=x, variant="best")


@pytest.mark.parametrize("N", [(1 << 30) + 1, (1 << 31) - 1])
@pytest.mark.parametrize("M", [2, 65])
def test_lora_refuses_columns_that_its_indexes_cannot_pass(L, M, N):
    """The kernels step through a row some thousand columns at a time, so that an index may go that far beyond its end."""
    assert call(L.rcp_lora_add, LORA, M=M, N=N) == LIMIT

"""Caches and biases whose tensors get another storage: a call takes the memory that they have then, or refuses."""
import pytest
import torch

from paper_2511_18871_amd import binding as B


def test_a_cache_is_looked_at_again():
    k, v = torch.zeros(4, 2, 16, 64), torch.zeros(4, 2, 16, 64)
    cache = B.KvCache(k, v)
    for tensor, name in ((k, "k"), (v, "v")):
        tensor.data = torch.ones(4, 2, 16, 64)
        struct = cache._ref.contents
        assert getattr(struct, name) == tensor.data_ptr() and struct.n_pages == 4
    other = torch.zeros(9, 2, 16, 64)
    for bad in (other, other[:4, :, :, ::2], torch.zeros(4, 2, 16, 64).bfloat16(), torch.zeros(4, 16, 2, 64).transpose(1, 2)):
        cache = B.KvCache(torch.zeros(4, 2, 16, 64), torch.zeros(4, 2, 16, 64))
        cache.v.data = bad
        with pytest.raises(B.SpAttnError) as e:
            cache._ref
        assert e.value.status == B.SP_ERR_INVALID_ARG
    cache = B.KvCache(torch.zeros(4, 2, 16, 64), torch.zeros(4, 2, 16, 64))
    cache.k.resize_(2, 2, 16, 64)                       # the same memory, fewer pages
    with pytest.raises(B.SpAttnError):
        cache._ref


@pytest.mark.parametrize("view", [lambda t: t.transpose(1, 2), lambda t: t.flatten().view(torch.bfloat16)[:t.numel()].view(t.shape)])
def test_other_views_of_the_same_memory(view):
    cache = B.KvCache(torch.zeros(4, 16, 16, 64), torch.zeros(4, 16, 16, 64))
    cache.v.data = view(cache.v.data)
    assert cache.v.data_ptr() == cache._struct.v and cache.v.shape == (4, 16, 16, 64)
    with pytest.raises(B.SpAttnError):
        cache._ref


def test_a_bias_is_looked_at_again():
    rules = B.LogitRules(bias=torch.zeros(40))
    rules.bias.data = torch.ones(40)
    rules._fits(40, -1)
    assert rules._ref.contents.bias == rules.bias.data_ptr()
    rules.bias = None
    rules._fits(40, -1)
    assert rules._ref.contents.bias is None


@pytest.mark.gpu
def test_calls_follow_the_tensors():
    gen = torch.Generator().manual_seed(2)
    k, v, x = (torch.randn(*s, generator=gen).cuda() for s in ((4, 2, 16, 64), (4, 2, 16, 64), (1, 2, 64)))
    cache, tables, lens = B.KvCache(k, v), torch.tensor([[1, 3]], dtype=torch.int32).cuda(), torch.tensor([17], dtype=torch.int32).cuda()
    old = k.data_ptr()
    first = B.sp_attn_decode(cache, x, None, None, None, tables, lens, 0.1)
    keep_k, keep_v = k.detach(), v.detach()             # the first storages live on
    k.data, v.data = torch.randn(4, 2, 16, 64, generator=gen).cuda(), torch.randn(4, 2, 16, 64, generator=gen).cuda()
    assert k.data_ptr() != old
    keep_k, keep_v, before = keep_k.clone(), keep_v.clone(), (keep_k, keep_v)
    o, lse = B.sp_attn_decode(cache, x, None, None, None, tables, lens, 0.1)
    want = B.sp_attn_decode(B.KvCache(k, v), x, None, None, None, tables, lens, 0.1)
    assert torch.equal(o, want[0]) and torch.equal(lse, want[1]) and not torch.equal(o, first[0])
    B.sp_attn_cache_append(cache, x, x, tables, lens, 1e4)
    assert torch.equal(before[0], keep_k) and torch.equal(before[1], keep_v) and torch.equal(v[3, :, 1], x[0])
    z, none = torch.randn(2, 40, generator=gen).cuda(), (None,) * 4
    rules = B.LogitRules(bias=torch.zeros(40).cuda())
    rules.bias.data = torch.full((40,), 2.0).cuda()
    assert torch.equal(B.sp_attn_adjust_logits(z, rules, None, *none), z + 2.0)

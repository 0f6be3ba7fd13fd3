"""Appending to the paged cache on the GPU, element by element against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import rollout_oracle as ro
from paper_2511_18871_amd import binding as B
from tests.rollout import HALF_STEP, check, make_tables, numpy64

pytestmark = pytest.mark.gpu
BASE = 10000.0


def make(dtype, d, hq, hkv, page, lens, new_lens, seed=3, fused=True):
    gen = torch.Generator().manual_seed(seed)
    T = sum(new_lens)
    tables, pages = make_tables(gen, [max(a, 0) + b for a, b in zip(lens, new_lens)], page)
    qkv = torch.randn(T, (hq + 2 * hkv) * d, generator=gen).to(dtype).cuda()
    q, k, v = qkv.split([hq * d, hkv * d, hkv * d], dim=1)
    q, k, v = q.unflatten(1, (hq, d)), k.unflatten(1, (hkv, d)), v.unflatten(1, (hkv, d))
    if not fused:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    kc = torch.randn(pages, hkv, page, d, generator=gen).to(dtype).cuda()
    vc = torch.randn(pages, hkv, page, d, generator=gen).to(dtype).cuda()
    return q, k, v, kc, vc, tables


def compare(q, k, v, kc0, vc0, kc, vc, tables, lens, new_lens, base, q_out, k_out, lens_out, dtype):
    rk, rv, rq, rko, rl = ro.cache_append(numpy64(kc0), numpy64(vc0), numpy64(q), numpy64(k), numpy64(v), new_lens, tables.tolist(), lens, base, BASE)
    half = HALF_STEP[dtype] if dtype == torch.bfloat16 else 0.0
    # a pair (a, b) turns by a float32 angle in [-pi, pi] (2^-23 off), by a sine and cosine of 2 units and two products each:
    # 2^-20 (|a| + |b|) in all; then one rounding
    def size(x):
        x = np.abs(numpy64(x))
        d = x.shape[-1]
        return np.tile(x[..., :d // 2] + x[..., d // 2:], 2)
    active = np.repeat(np.array(lens) >= 0, new_lens)
    for name, got, ref, x in (("q_out", q_out, rq, q), ("k_out", k_out, rko, k)):
        if got is not None:
            check(name, numpy64(got)[active], ref[active], half * np.abs(ref[active]) + 2.0 ** -20 * size(x)[active])
    assert np.array_equal(numpy64(vc), rv)
    big = 2 * np.abs(numpy64(k)).max() if k.shape[0] else 0.0
    same = rk == numpy64(kc0)
    assert np.array_equal(numpy64(kc)[same], rk[same])               # what no token falls on is left as it was
    check("k_cache", kc, rk, half * np.abs(rk) + 2.0 ** -20 * big)
    assert lens_out.tolist() == rl.tolist()


SHAPES = [(torch.bfloat16, 128, 28, 4), (torch.bfloat16, 64, 5, 1), (torch.float32, 64, 2, 2), (torch.float32, 128, 8, 2), (torch.bfloat16, 128, 40, 8)]


@pytest.mark.parametrize("dtype,d,hq,hkv", SHAPES)
@pytest.mark.parametrize("page", [16, 64, 256])
def test_one_token_each(dtype, d, hq, hkv, page):
    lens = [0, 1, 15, 16, 17, 255, 256, 300, -1]
    new = [1] * len(lens)
    q, k, v, kc, vc, tables = make(dtype, d, hq, hkv, page, lens, new)
    base = [0, 5, 100, 16000, 3, 0, 1, 2, 9]
    kc0, vc0 = kc.clone(), vc.clone()
    q_out = torch.full(q.shape, 7.0, dtype=dtype, device="cuda")
    q_out, lens_out = B.sp_attn_cache_append(B.KvCache(kc, vc), k, v, tables.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), BASE, q=q,
                                             pos_base=torch.tensor(base, dtype=torch.int32).cuda(), q_out=q_out)
    torch.cuda.synchronize()
    compare(q, k, v, kc0, vc0, kc, vc, tables, lens, new, base, q_out, None, lens_out, dtype)
    assert torch.all(q_out[-1] == 7.0)                               # the sequence that takes no part


@pytest.mark.parametrize("dtype,d,hq,hkv", SHAPES)
def test_ragged_prompts(dtype, d, hq, hkv):
    lens, new = [0, 7, 0, 30, -1, 64], [33, 0, 1, 50, 4, 17]
    q, k, v, kc, vc, tables = make(dtype, d, hq, hkv, 32, lens, new, fused=False)
    kc0, vc0 = kc.clone(), vc.clone()
    k_out = torch.full(k.shape, 5.0, dtype=dtype, device="cuda")
    q_out, lens_out = B.sp_attn_cache_append(B.KvCache(kc, vc), k, v, tables.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), BASE, q=q,
                                             new_lens=new, k_out=k_out)
    torch.cuda.synchronize()
    compare(q, k, v, kc0, vc0, kc, vc, tables, lens, new, None, q_out, k_out, lens_out, dtype)
    assert torch.all(k_out[84:88] == 5.0)


def test_more_sequences_than_a_launch_holds():
    lens, new = [i % 40 for i in range(1600)], [i % 3 for i in range(1600)]
    q, k, v, kc, vc, tables = make(torch.bfloat16, 64, 2, 1, 16, lens, new)
    kc0, vc0 = kc.clone(), vc.clone()
    q_out, lens_out = B.sp_attn_cache_append(B.KvCache(kc, vc), k, v, tables.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), BASE, q=q, new_lens=new)
    torch.cuda.synchronize()
    compare(q, k, v, kc0, vc0, kc, vc, tables, lens, new, None, q_out, None, lens_out, torch.bfloat16)


def test_bad_pages_and_full_tables_store_nothing():
    lens, new = [14, 30, 3], [6, 5, 2]
    q, k, v, kc, vc, tables = make(torch.float32, 64, 2, 2, 16, lens, new)
    tables[0, 1] = kc.shape[0]            # behind the cache
    tables[2, 0] = -5
    tables = tables[:, :2].contiguous()   # sequence 1: two of its five tokens find room
    kc0, vc0 = kc.clone(), vc.clone()
    q_out, lens_out = B.sp_attn_cache_append(B.KvCache(kc, vc), k, v, tables.cuda(), torch.tensor(lens, dtype=torch.int32).cuda(), BASE, q=q, new_lens=new)
    torch.cuda.synchronize()
    compare(q, k, v, kc0, vc0, kc, vc, tables, lens, new, None, q_out, None, lens_out, torch.float32)
    assert lens_out.tolist() == [20, 32, 5]


def test_far_positions_in_place_and_without_q():
    lens, new = [5, 2], [3, 2]
    q, k, v, kc, vc, tables = make(torch.float32, 128, 3, 1, 16, lens, new, fused=False)
    kc0, vc0, q0, k0 = kc.clone(), vc.clone(), q.clone(), k.clone()
    base = [2 ** 31 - 9, 1 << 20]
    dev = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    _, lens_out = B.sp_attn_cache_append(B.KvCache(kc, vc), k, v, tables.cuda(), dev(lens), BASE, q=q, new_lens=new, pos_base=dev(base), q_out=q, k_out=k)
    torch.cuda.synchronize()
    # theta and the product are float64: 2^31 radians are 2^-21 off
    rk, rv, rq, rko, rl = ro.cache_append(numpy64(kc0), numpy64(vc0), numpy64(q0), numpy64(k0), numpy64(v), new, tables.tolist(), lens, base, BASE)
    for got, ref in ((q, rq), (k, rko), (kc, rk)):
        check("rotated", got, ref, 4e-6 * 8)
    q1, l1 = B.sp_attn_cache_append(B.KvCache(kc0, vc0), k0, v, tables.cuda(), dev(lens), BASE, new_lens=new, pos_base=dev(base))
    torch.cuda.synchronize()
    assert q1 is None and torch.equal(kc0, kc) and torch.equal(vc0, vc) and torch.equal(l1, lens_out)


def test_nothing_new():
    _, _, _, kc, vc, tables = make(torch.float32, 64, 2, 2, 16, [3, 4], [0, 0])
    empty = torch.empty(0, 2, 64, device="cuda")
    q_out, lens_out = B.sp_attn_cache_append(B.KvCache(kc, vc), empty, empty, tables.cuda(), torch.tensor([3, 4], dtype=torch.int32).cuda(), BASE, q=empty, new_lens=[0, 0])
    assert q_out.shape == (0, 2, 64) and lens_out.tolist() == [3, 4]


def test_offsets_beyond_32_bits():
    """A cache of more than 2^32 elements (8.6 GB each): the last pages are reached."""
    pages, hkv, page, d = 2 ** 20 + 16, 2, 16, 128
    kc, vc = (torch.zeros(pages, hkv, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    gen = torch.Generator().manual_seed(1)
    k, v, q = (torch.randn(2, h, d, generator=gen).bfloat16().cuda() for h in (hkv, hkv, 4))
    tables = torch.tensor([[pages - 1], [pages - 2]], dtype=torch.int32).cuda()
    lens = torch.tensor([3, 15], dtype=torch.int32).cuda()
    cache = B.KvCache(kc, vc)
    q_out, lens_out = B.sp_attn_cache_append(cache, k, v, tables, lens, BASE, q=q)
    o, lse = B.sp_attn_decode(cache, q_out, None, None, None, tables, lens_out, 0.1)
    torch.cuda.synchronize()
    assert torch.equal(vc[pages - 1, :, 3], v[0]) and torch.equal(vc[pages - 2, :, 15], v[1])
    assert torch.count_nonzero(vc[: 1 << 19].view(torch.int16)).item() == 0
    small = B.KvCache(kc[-2:].clone(), vc[-2:].clone())
    o2, lse2 = B.sp_attn_decode(small, q_out, None, None, None, torch.tensor([[1], [0]], dtype=torch.int32).cuda(), lens_out, 0.1)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)


def test_on_another_stream_and_replayed():
    """A captured append follows the lengths that the device holds at the replay."""
    lens, new = [3, 20], [1, 1]
    q, k, v, kc, vc, tables = make(torch.bfloat16, 128, 4, 2, 16, [40, 40], new)
    cache, tables = B.KvCache(kc, vc), tables.cuda()
    lens_d = torch.tensor(lens, dtype=torch.int32).cuda()
    lens_out, q_out = torch.zeros_like(lens_d), torch.empty(2, 4, 128, dtype=torch.bfloat16, device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    B.sp_attn_cache_append(cache, k, v, tables, lens_d, BASE, q=q, q_out=q_out, lens_out=lens_out, stream=stream)
    stream.synchronize()
    first = (q_out.clone(), kc.clone())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.sp_attn_cache_append(cache, k, v, tables, lens_d, BASE, q=q, q_out=q_out, lens_out=lens_out)
    kc.copy_(kc * 0)
    for step in range(3):
        graph.replay()
        torch.cuda.synchronize()
        have = (lens_d + 1).tolist()
        assert lens_out.tolist() == have
        if step == 0:
            assert torch.equal(q_out, first[0]) and torch.equal(kc[tables[0, 0].item(), :, 3], first[1][tables[0, 0].item(), :, 3])
        eager = B.sp_attn_cache_append(B.KvCache(kc.clone(), vc.clone()), k, v, tables, lens_d, BASE, q=q)
        assert torch.equal(eager[0], q_out)
        lens_d.copy_(lens_out)

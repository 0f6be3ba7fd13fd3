"""Attention of one new token per sequence on the GPU, element by element against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import rollout_oracle as ro
from paper_2511_18871_amd import binding as B
from tests.rollout import check, decode_bounds, make_tables, numpy64

pytestmark = pytest.mark.gpu


def make(dtype, d, hq, hkv, page, prompts, Gs, resp, seed=5):
    gen = torch.Generator().manual_seed(seed)
    tables, pages = make_tables(gen, prompts + resp, page)
    kc, vc = (torch.randn(pages, hkv, page, d, generator=gen).to(dtype) for _ in range(2))
    q = torch.randn(len(resp), hq, d, generator=gen).to(dtype)
    return q, kc, vc, tables[:len(prompts)].contiguous(), tables[len(prompts):].contiguous()


def dev32(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def run_and_check(q, kc, vc, Gs, pt, prompts, rt, resp, scale):
    d = q.shape[2]
    o, lse = B.sp_attn_decode(B.KvCache(kc.cuda(), vc.cuda()), q.cuda(), Gs, None if pt is None else pt.cuda(), None if pt is None else dev32(prompts),
                              None if rt is None else rt.cuda(), dev32(resp), scale)
    o2, lse2 = B.sp_attn_decode(B.KvCache(kc.cuda(), vc.cuda()), q.cuda(), Gs, None if pt is None else pt.cuda(), None if pt is None else dev32(prompts),
                                None if rt is None else rt.cuda(), dev32(resp), scale)
    torch.cuda.synchronize()
    assert torch.equal(o, o2) and torch.equal(lse, lse2)                # bitwise repeatable
    groups = [1] * len(resp) if Gs is None else Gs
    ref, rlse, weight, reach, count = ro.decode(numpy64(kc), numpy64(vc), numpy64(q), groups, None if pt is None else pt.tolist(), prompts,
                                                None if rt is None else rt.tolist(), resp, scale)
    tol_o, tol_lse = decode_bounds(ref, rlse, weight, reach, count, d, q.dtype)
    check("lse", lse, rlse, tol_lse)
    check("o", o, ref, tol_o)
    return o, lse


TYPES = [(torch.bfloat16, 128), (torch.bfloat16, 64), (torch.float32, 128), (torch.float32, 64)]


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("page", [16, 32, 64, 128, 256])
def test_ragged_groups(dtype, d, page):
    prompts, Gs = [70, 0, 129, 16, 1], [3, 2, 0, 4, 1]
    resp = [1, 17, 64, 200, 31, 0, 33, 65, 128, 127]
    run_and_check(*(lambda q, kc, vc, pt, rt: (q, kc, vc, Gs, pt, prompts, rt, resp, 0.11))(*make(dtype, d, 4, 2, page, prompts, Gs, resp)))


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("hq,hkv", [(1, 1), (7, 7), (28, 4), (40, 8), (32, 8), (64, 1), (6, 3)])
def test_head_layouts(dtype, d, hq, hkv):
    prompts, Gs, resp = [90, 33], [5, 2], [3, 40, 17, 1, 70, 64, 9]
    q, kc, vc, pt, rt = make(dtype, d, hq, hkv, 16, prompts, Gs, resp)
    run_and_check(q, kc, vc, Gs, pt, prompts, rt, resp, 0.09)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("members", [1, 4, 5, 8, 9, 16, 17, 32, 33, 70])
def test_rows_of_a_group(dtype, d, members):
    """Row blocks of every size, with a prompt that several workgroups share."""
    prompts, resp = [700], [1 + 7 * i % 50 for i in range(members)]
    q, kc, vc, pt, rt = make(dtype, d, 8, 2, 64, prompts, [members], resp)
    run_and_check(q, kc, vc, [members], pt, prompts, rt, resp, 0.1)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("length", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 511, 513, 1000, 5000])
def test_lengths_of_one_sequence(dtype, d, length):
    q, kc, vc, _, rt = make(dtype, d, 4, 1, 32, [], [1], [length])
    run_and_check(q, kc, vc, None, None, None, rt, [length], 0.125)


def test_prompt_alone_and_rows_without_a_key():
    q, kc, vc, pt, rt = make(torch.bfloat16, 128, 4, 2, 16, [50, 0, 7], [2, 2, 3], [0, 3, 0, 0, 5, 0, 2])
    resp = [0, 3, 0, 0, 5, -1, 2]
    o, lse = run_and_check(q, kc, vc, [2, 2, 3], pt, [50, 0, 7], rt, resp, 0.1)
    for s in (2, 3, 5):
        assert torch.all(o[s] == 0) and torch.all(torch.isneginf(lse[:, s]))
    run_and_check(q, kc, vc, [2, 2, 3], pt, [50, 0, 7], None, [0, 0, 0, 0, 0, -1, 0], 0.1)


def test_bad_pages_are_not_followed_and_lengths_are_cut():
    prompts, Gs, resp = [100, 40], [2, 3], [20, 60, 33, 1, 80]
    for dtype, d in TYPES:
        q, kc, vc, pt, rt = make(dtype, d, 4, 2, 16, prompts, Gs, resp)
        pt[0, 2], pt[0, 6], pt[1, 0] = -1, kc.shape[0], 2 ** 31 - 1
        rt[1, 1], rt[4, 4], rt[3, 0] = -2 ** 31, kc.shape[0] + 7, -3
        run_and_check(q, kc, vc, Gs, pt, [1000, -4], rt, [20, 10 ** 6, 33, 1, 80], 0.1)


def test_what_lies_behind_a_length_does_not_matter():
    """NaN and infinities behind the last key of a page, in pages of others and in the padding of tables."""
    prompts, Gs, resp = [37, 0], [2, 1], [5, 50, 18]
    for dtype, d in TYPES:
        q, kc, vc, pt, rt = make(dtype, d, 4, 2, 16, prompts, Gs, resp)
        want = run_and_check(q, kc, vc, Gs, pt, prompts, rt, resp, 0.1)
        used = torch.zeros(kc.shape[0], 16, dtype=torch.bool)
        for table, lens in ((pt, prompts), (rt, resp)):
            for row, n in zip(table, lens):
                for j in range(n):
                    used[row[j // 16], j % 16] = True
        hole = ~used[:, None, :, None]
        for bad in (float("nan"), float("inf")):
            o, lse = B.sp_attn_decode(B.KvCache(torch.where(hole, bad, kc).to(dtype).cuda(), torch.where(hole, bad, vc).to(dtype).cuda()), q.cuda(), Gs,
                                      pt.cuda(), dev32(prompts), rt.cuda(), dev32(resp), 0.1)
            assert torch.equal(o, want[0]) and torch.equal(lse, want[1])


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("factor", [1e-3, 8.0, 40.0])
def test_scales_of_scores(dtype, d, factor):
    """From even weights to rows that one key decides; the largest score may come late."""
    prompts, Gs, resp = [300], [3], [100, 1, 260]
    q, kc, vc, pt, rt = make(dtype, d, 8, 2, 64, prompts, Gs, resp)
    kc[rt[2, 3], :, 40] *= 6
    run_and_check(q * factor, kc, vc, Gs, pt, prompts, rt, resp, 1 / d ** 0.5)


def test_many_groups_take_their_table_from_memory():
    n = 900
    prompts, resp = [i % 21 for i in range(n)], [i % 9 for i in range(n)]
    q, kc, vc, pt, rt = make(torch.bfloat16, 64, 2, 1, 16, prompts, [1] * n, resp)
    run_and_check(q, kc, vc, [1] * n, pt, prompts, rt, resp, 0.1)


@pytest.mark.parametrize("dtype,d", TYPES)
def test_more_rows_than_the_chip_holds_waves(dtype, d):
    """Rows with one chunk and with many side by side in a wave, rows without a key among them, an incomplete last wave."""
    Gs = [7] * 43
    prompts, resp = [(i * 37) % 90 for i in range(43)], [(i * 11) % 40 for i in range(301)]
    prompts[5], prompts[6], resp[42], resp[43], resp[300] = 900, 0, 0, -1, 2100
    q, kc, vc, pt, rt = make(dtype, d, 28, 4, 32, prompts, Gs, [max(n, 0) for n in resp])
    run_and_check(q, kc, vc, Gs, pt, prompts, rt, resp, 0.1)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_more_lists_than_a_workgroup_holds(dtype):
    Gs = [(i * 7) % 9 for i in range(1100)]
    n = sum(Gs)
    assert n + len(Gs) > 4096
    prompts, resp = [(i * 5) % 40 for i in range(1100)], [(i * 13) % 19 for i in range(n)]
    prompts[700], resp[3000] = 600, 333
    q, kc, vc, pt, rt = make(dtype, 64, 6, 1, 16, prompts, Gs, resp)
    run_and_check(q, kc, vc, Gs, pt, prompts, rt, resp, 0.125)


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.float32, 64)])
def test_pages_beyond_32_bits(dtype, d):
    """Pages whose offsets pass 2^31 elements and 2^32 bytes, beside the first ones."""
    prompts, Gs, resp = [600], [6], [40, 300, 1, 0, 77, 513]
    q, kc, vc, pt, rt = (x.cuda() for x in make(dtype, d, 8, 2, 64, prompts, Gs, resp))
    want = B.sp_attn_decode(B.KvCache(kc, vc), q, Gs, pt, dev32(prompts), rt, dev32(resp), 0.1)
    n, of_page = kc.shape[0], kc[0].numel()
    far = (2 ** 31 + 2 ** 28) // of_page
    big = [torch.zeros(far + n, *kc.shape[1:], dtype=dtype, device="cuda") for _ in range(2)]
    for c, b in zip((kc, vc), big):
        b[far:] = c
        b[:n] = c
    assert far * of_page > 2 ** 31 and big[0].numel() * big[0].element_size() > 2 ** 32
    for pages, resp_pages in ((pt + far, rt + far), (pt, rt + far), (pt + far, rt)):
        got = B.sp_attn_decode(B.KvCache(*big), q, Gs, pages.to(torch.int32), dev32(prompts), resp_pages.to(torch.int32), dev32(resp), 0.1)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_replayed_with_other_lengths_and_workspaces_shared():
    """Two captured graphs on one workspace, replayed in turn with other lengths, eager calls on it in between."""
    prompts, Gs, resp = [200, 90], [5, 3], [64] * 8
    q, kc, vc, pt, rt = (x.cuda() for x in make(torch.bfloat16, 128, 8, 2, 16, prompts, Gs, resp))
    cache, pl, rl = B.KvCache(kc, vc), dev32(prompts), dev32(resp)
    ws = torch.empty(B.decode_workspace_bytes(2, 8, 8, 2, 128, B.SP_BF16), dtype=torch.uint8, device="cuda")
    outs, graphs = [], []
    B.sp_attn_decode(cache, q, Gs, pt, pl, rt, rl, 0.1, workspace=ws)
    torch.cuda.synchronize()
    for tables in ((pt, pl), (None, None)):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(B.sp_attn_decode(cache, q, Gs, *tables, rt, rl, 0.1, workspace=ws))
        graphs.append((graph, tables))
    for step in range(4):
        rl.copy_(dev32([(13 * step + 9 * i) % 65 for i in range(8)]))
        pl.copy_(dev32([200 - 60 * step, 30 * step]))
        for (graph, tables), (o, lse) in zip(graphs, outs):
            graph.replay()
            torch.cuda.synchronize()
            eo, el = B.sp_attn_decode(cache, q, Gs, *tables, rt, rl, 0.1)
            assert torch.equal(o, eo) and torch.equal(lse, el), step
            B.sp_attn_decode(cache, q, Gs, pt, pl, rt, rl, 0.2, workspace=ws)


def test_on_another_stream_into_given_outputs():
    prompts, Gs, resp = [64], [4], [10, 20, 30, 0]
    q, kc, vc, pt, rt = (x.cuda() for x in make(torch.bfloat16, 128, 8, 2, 16, prompts, Gs, resp))
    cache = B.KvCache(kc, vc)
    want = B.sp_attn_decode(cache, q, Gs, pt, dev32(prompts), rt, dev32(resp), 0.1)
    stream = torch.cuda.Stream()
    guard = torch.full((6, 8, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.empty(8, 4, device="cuda")
    pl, rl = dev32(prompts), dev32(resp)
    stream.wait_stream(torch.cuda.current_stream())
    B.sp_attn_decode(cache, q, Gs, pt, pl, rt, rl, 0.1, o=guard[1:5], lse=lse, stream=stream)
    free = B.sp_attn_decode(cache, q, Gs, pt, pl, rt, rl, 0.1, stream=stream)
    stream.synchronize()
    assert torch.equal(guard[1:5], want[0]) and torch.equal(lse, want[1])
    assert torch.equal(free[0], want[0]) and torch.equal(free[1], want[1])
    assert torch.all(guard[0] == 3.0) and torch.all(guard[5] == 3.0)
    B.sp_attn_decode(cache, q, Gs, pt, pl, rt, rl, 0.1, o=q)            # in place
    assert torch.equal(q, want[0])


def test_reserve_of_a_forward_is_given_up():
    """A decode step on the workspace of a forward leaves no reserve that a backward could take for the forward's."""
    torch.manual_seed(0)
    T, hq, hkv, d = 70, 4, 2, 128
    q, k, v, do = (torch.randn(T, h, d, device="cuda").bfloat16() for h in (hq, hkv, hkv, hq))
    ws = torch.empty(1 << 24, dtype=torch.uint8, device="cuda")
    o, lse = B.sp_attn_fwd(q, k, v, 50, [20], 0.1, workspace=ws)
    with_reserve = B.sp_attn_bwd(q, k, v, o, lse, do, 50, [20], 0.1, workspace=ws)
    o, lse = B.sp_attn_fwd(q, k, v, 50, [20], 0.1, workspace=ws)
    cache_k = torch.randn(4, hkv, 64, d, device="cuda").bfloat16()
    B.sp_attn_decode(B.KvCache(cache_k, cache_k), q[:1], None, None, None, dev32([[0, 1]]), dev32([100]), 0.1, workspace=ws)
    without = B.sp_attn_bwd(q, k, v, o, lse, do, 50, [20], 0.1, workspace=ws)
    fresh = B.sp_attn_bwd(q, k, v, o, lse, do, 50, [20], 0.1, workspace=torch.empty(1 << 24, dtype=torch.uint8, device="cuda"))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(without, fresh))
    assert not all(torch.equal(a, b) for a, b in zip(with_reserve, fresh))

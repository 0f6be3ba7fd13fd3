"""bf16 attention of one new token per sequence: what is lost is the rounding of o, as if the weights had 32 bits."""
import numpy as np
import pytest
import torch

from oracle import rollout_oracle as ro
from paper_2511_18871_amd import binding as B
from tests.rollout import check, decode_bounds, make_tables, numpy64

pytestmark = pytest.mark.gpu


def dev32(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


# lists of a wave with one and with two row tiles, shared ones with one to three
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv,prompts,Gs,resp", [
    (4, 1, [], [], [700]), (24, 1, [40], [1], [90]), (28, 4, [130, 1], [3, 2], [5, 40, 1, 64, 33]), (8, 2, [300], [16], list(range(1, 17))),
    (40, 8, [500], [24], [7 * i % 41 for i in range(24)]), (40, 8, [200], [33], [i % 5 for i in range(33)])])
def test_weights_keep_their_bits(d, hq, hkv, prompts, Gs, resp):
    gen = torch.Generator().manual_seed(31)
    tables, pages = make_tables(gen, prompts + resp, 16)
    kc, vc = (torch.randn(pages, hkv, 16, d, generator=gen).bfloat16() for _ in range(2))
    q = torch.randn(len(resp), hq, d, generator=gen).bfloat16()
    pt, rt = (tables[:len(prompts)].contiguous() if prompts else None), tables[len(prompts):].contiguous()
    scale = 1 / d ** 0.5
    o, lse = B.sp_attn_decode(B.KvCache(kc.cuda(), vc.cuda()), q.cuda(), Gs or None, None if pt is None else pt.cuda(), dev32(prompts) if prompts else None,
                              rt.cuda(), dev32(resp), scale)
    ref, rlse, weight, reach, count = ro.decode(numpy64(kc), numpy64(vc), numpy64(q), Gs or [1], None if pt is None else pt.tolist(), prompts, rt.tolist(), resp, scale)
    # as in float32 but for: a weight's second part is below 2^-7 of it and off by 2^-8 of that; and one rounding of o
    tol_o, tol_lse = decode_bounds(ref, rlse, weight, reach, count, d, torch.float32)
    check("lse", lse, rlse, tol_lse)
    check("o", o, ref, tol_o + weight * 2.0 ** -15 + np.abs(ref) * 2.0 ** -8)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("members", [1, 20])                    # a list of a wave, a shared one
def test_keys_without_weight_add_nothing(d, members):
    """The largest values, under keys whose weights are below what float32 holds."""
    gen = torch.Generator().manual_seed(d)
    kc, vc = (torch.randn(3, 1, 64, d, generator=gen).bfloat16() for _ in range(2))
    q = torch.randn(members, 2, d, generator=gen).bfloat16()
    q[:, :, 0], kc[:, 0, :, 0] = 100.0, 1.0
    kc[1, 0, 7, 0] = -100.0                                     # 2e4 times the scale below the others
    vc[1, 0, 7] = 0
    args = (q.cuda(), [members], dev32([[0, 1, 2]]), dev32([150]), None, dev32([0] * members), 0.1)
    want = B.sp_attn_decode(B.KvCache(kc.cuda(), vc.cuda()), *args)
    vc[1, 0, 7] = torch.finfo(torch.bfloat16).max
    got = B.sp_attn_decode(B.KvCache(kc.cuda(), vc.cuda()), *args)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])

"""Scores of any magnitude that float32 holds: attention of one new token per sequence against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import rollout_oracle as ro
from paper_2511_18871_amd import binding as B
from tests.rollout import HALF_STEP, U24, check, make_tables, numpy64

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.bfloat16, 64), (torch.float32, 128), (torch.float32, 64)])
@pytest.mark.parametrize("power", [0, 12, 30, 60, 100])
@pytest.mark.parametrize("hq,hkv,prompts,Gs,resp", [(4, 1, [70], [1], [500]), (8, 2, [300], [24], [i % 9 for i in range(24)])])
def test_large_scores(dtype, d, power, hq, hkv, prompts, Gs, resp):
    """Small whole numbers times a power of two: every score is exact, and equal ones share a row's weight."""
    gen = torch.Generator().manual_seed(power)
    tables, pages = make_tables(gen, prompts + resp, 16)
    kc = torch.randint(-2, 3, (pages, hkv, 16, d), generator=gen).to(dtype)
    kc[::2] = kc[0]                                      # the same keys again, in other chunks
    vc = torch.randn(pages, hkv, 16, d, generator=gen).to(dtype)
    q = (torch.randint(-2, 3, (len(resp), hq, d), generator=gen).double() * 2.0 ** power).to(dtype)
    pt, rt = tables[:1].contiguous(), tables[1:].contiguous()
    dev32 = lambda x: torch.tensor(x, dtype=torch.int32).cuda()
    o, lse = B.sp_attn_decode(B.KvCache(kc.cuda(), vc.cuda()), q.cuda(), Gs, pt.cuda(), dev32(prompts), rt.cuda(), dev32(resp), 1.0)
    ref, rlse, weight, _, count = ro.decode(numpy64(kc), numpy64(vc), numpy64(q), Gs, pt.tolist(), prompts, rt.tolist(), resp, 1.0)
    # no score is rounded; an exponential: its argument's rounding (weights that count: above e^-100), 4 units; sums: n / 16 + 64 units; scaling by
    # 1: 4 units of lse; bf16: 2^-15 of the weights
    unit = (110 + 4 + 64 + count / 16) * U24
    check("lse", lse, rlse, unit + 4 * U24 * np.abs(np.where(np.isfinite(rlse), rlse, 0.0)))
    lost = 2.0 ** -15 if dtype == torch.bfloat16 else 0.0
    check("o", o, ref, weight * (2 * unit[:, None, None] + lost) + np.abs(ref) * HALF_STEP[dtype] + 1e-37)

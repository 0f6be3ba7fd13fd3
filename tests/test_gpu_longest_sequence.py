"""Sequences as long as an int32 length can say, over a table that names one page again and again."""
import math

import pytest
import torch

from paper_2511_18871_amd import binding as B

pytestmark = pytest.mark.gpu
LONGEST = 2 ** 31 - 64


def dev32(*x):
    return torch.tensor(x, dtype=torch.int32).cuda()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("members", [1, 40])                    # a list of a wave, a shared one
def test_decode(dtype, members):
    """Every key is the same but for those behind the longest length, which are NaN."""
    if dtype is torch.float32 and members > 1:
        members = 2
    gen = torch.Generator().manual_seed(1)
    k, v = (torch.randn(1, 1, 1, 64, generator=gen).expand(2, 1, 256, 64).contiguous() for _ in range(2))
    k[1, 0, 192:], v[1, 0, 192:] = float("nan"), float("nan")
    table = torch.zeros(1, 2 ** 31 // 256, dtype=torch.int32, device="cuda")
    table[0, -1] = 1
    q = torch.randn(members, 1, 64, generator=gen).to(dtype)
    k, v = k.to(dtype), v.to(dtype)
    scale = 1 / 64
    o, lse = B.sp_attn_decode(B.KvCache(k.cuda(), v.cuda()), q.cuda(), [members], table, dev32(2 ** 31 - 1), None, dev32(*[0] * members), scale)
    score = scale * (q[:, 0].double() @ k[0, 0, 0].double())
    # sums of equal terms: 2^18 of a lane one by one, 2^-24 of the sum so far each, then those of lanes and chunks
    assert (lse[0].cpu().double() - score - math.log(LONGEST)).abs().max() <= 2.0 ** -24 * 2 ** 18
    assert (o[:, 0].cpu().double() - v[0, 0, 0].double()).abs().max() <= 2 * 2.0 ** -24 * 2 ** 18 * v[0].double().abs().max()


def test_append():
    k, v = (torch.zeros(3, 1, 256, 64, device="cuda") for _ in range(2))
    table = torch.zeros(4, 2 ** 31 // 256 + 1, dtype=torch.int32, device="cuda")
    table[:, -2], table[:, -1] = 1, 2
    x = torch.full((4, 1, 64), 3.0, device="cuda")
    _, now = B.sp_attn_cache_append(B.KvCache(k, v), x, x, table, dev32(LONGEST - 1, LONGEST, 2 ** 31 - 1, -1), 1e4)
    assert now.tolist() == [LONGEST, LONGEST, 2 ** 31 - 1, -1]
    assert v.nonzero()[:, :3].unique(dim=0).tolist() == [[1, 0, 191]] and torch.all(v[1, 0, 191] == 3)

"""Scores of any magnitude that float32 holds: attention of drafted tokens, in lists of few rows and of many, against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import rollout_oracle as ro
from paper_2511_18871_amd import binding as B
from tests.branching import dev32, mask_words, random_trees
from tests.rollout import HALF_STEP, U24, check, make_tables, numpy64

pytestmark = pytest.mark.gpu


FEW, EIGHT_WAVES, FOUR_WAVES = (8, 2, 70, 300, 6), (16, 4, 0, 2900, 200), (16, 4, 0, 8100, 90)


@pytest.mark.parametrize("dtype,d,hq,hkv,prompt,ahead,n", [(torch.float32, 64, *FEW)] + [(torch.bfloat16, d, *x) for d in (128, 64) for x in (FEW, EIGHT_WAVES, FOUR_WAVES)])
@pytest.mark.parametrize("power", [30, 100])
def test_large_scores(dtype, d, power, hq, hkv, prompt, ahead, n):
    """Small whole numbers times a power of two: every score is exact, and equal ones share a row's weight."""
    gen = torch.Generator().manual_seed(power)
    tables, pages = make_tables(gen, [prompt, ahead + n], 16)
    kc = torch.randint(-2, 3, (pages, hkv, 16, d), generator=gen).to(dtype)
    kc[::2] = kc[0]                                      # the same keys again, in other chunks
    vc = torch.randn(pages, hkv, 16, d, generator=gen).to(dtype)
    q = (torch.randint(-2, 3, (n, hq, d), generator=gen).double() * 2.0 ** power).to(dtype)
    rows, (pt, rt) = random_trees(gen, [n]), (tables[:1].contiguous(), tables[1:].contiguous())
    o, lse = B.sp_attn_tree_decode(B.KvCache(kc.cuda(), vc.cuda()), q.cuda(), [1], [n], mask_words(rows, -(-n // 32)).cuda(), pt.cuda(), dev32([prompt]), rt.cuda(),
                                   dev32([ahead + n]), 1.0)
    ref, rlse, weight, _, count = ro.tree_decode(numpy64(kc), numpy64(vc), numpy64(q), [1], [n], rows, pt.tolist(), [prompt], rt.tolist(), [ahead + n], 1.0)
    # no score is rounded; an exponential: its argument's rounding (weights that count: above e^-100), 4 units; sums: n / 16 + 64 units; scaling by
    # 1: 4 units of lse.  bf16: o is sum p (1 + e) v / sum p (1 + e) with |e| <= 2^-8 in lists of many rows, off by sum p e (v - o), 2^-8 (sum p |v| + |o|) at most
    unit = (110 + 4 + 64 + count / 16) * U24
    check("lse", lse, rlse, unit + 4 * U24 * np.abs(rlse))
    lost = 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
    check("o", o, ref, weight * (2 * unit[:, None, None] + lost) + np.abs(ref) * (HALF_STEP[dtype] + lost) + 1e-37)

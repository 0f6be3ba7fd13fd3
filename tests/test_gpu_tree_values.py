"""Infinite and NaN values ahead of the drafted tokens of long lists: every row sees them, wherever the work is cut."""
import pytest
import torch

from paper_2511_18871_amd import binding as B
from tests.branching import dev32
from tests.test_gpu_tree import make

pytestmark = pytest.mark.gpu


def check_values(d, hq, hkv, prompt, ahead, n, seen):
    """seen: (in the prompt, token) of values that all rows see, each in a kv head and an element of its own."""
    q, kc, vc, pt, rt, rows, mask = make(torch.bfloat16, d, hq, hkv, 16, [prompt], [n], [ahead + n])
    args = (q.cuda(), [1], [n], mask.cuda(), pt.cuda(), dev32([prompt]), rt.cuda(), dev32([ahead + n]), 0.1)
    cache_k = kc.cuda()
    clean, clean_lse = B.sp_attn_tree_decode(B.KvCache(cache_k, vc.cuda()), *args)
    for bad in (float("nan"), float("inf"), -float("inf")):
        v2, want = vc.clone(), torch.zeros(n, hq, d, dtype=torch.bool)
        for i, (in_prompt, j) in enumerate(seen):
            head, e = i % hkv, 7 + 11 * i
            v2[(pt if in_prompt else rt)[0, j // 16], head, j % 16, e] = bad
            want[:, head * (hq // hkv):(head + 1) * (hq // hkv), e] = True
        o, lse = (x.cpu() for x in B.sp_attn_tree_decode(B.KvCache(cache_k, v2.cuda()), *args))
        hit = o[want]
        assert torch.all(hit.isnan() if bad != bad else hit == bad), (bad, seen)
        # The others but for another order of their sums: both are rounded to bf16, by 2^-8 of a value at most, and float32 sums of weights times values below 8 are
        # off by some 2^-20 of these.
        assert torch.allclose(o[~want].double(), clean.cpu()[~want].double(), rtol=2.0 ** -7, atol=2e-5)
        assert torch.allclose(lse, clean_lse.cpu(), rtol=1e-5, atol=1e-5)


def places(base):
    """The last key ahead of the first 64 keys with drafted tokens, the first and last of the 64 ahead of these, and the last key that is no drafted token."""
    first = base // 64 * 64
    return [(False, j) for j in sorted({first - 1, first - 64, first - 65, base - 1})]


# Runs of four units of 64 keys, or of seven: the first with drafted tokens is at every place of one
@pytest.mark.parametrize("d,hq,hkv,n", [(128, 16, 4, 200), (64, 16, 4, 200), (128, 32, 8, 200), (128, 16, 4, 256)])
@pytest.mark.parametrize("ahead", [2628 + 64 * i for i in range(8)])
@pytest.mark.parametrize("prompt", [0, 100])
def test_ahead_of_the_drafted_tokens_in_eight_waves(d, hq, hkv, n, ahead, prompt):
    check_values(d, hq, hkv, prompt, ahead, n, places(ahead))


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("ahead", [8004 + 64 * i for i in range(8)])
def test_ahead_of_the_drafted_tokens_in_four_waves(d, ahead):
    check_values(d, 16, 4, 0, ahead, 90, places(ahead))


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("prompt", [2600 + 64 * i for i in range(8)])
@pytest.mark.parametrize("ahead", [0, 20, 64])
def test_the_end_of_a_prompt_ahead_of_the_drafted_tokens(d, prompt, ahead):
    seen = [(True, prompt - 1), (True, prompt // 64 * 64 - 1), (True, prompt // 64 * 64 - 65)] + ([(False, ahead - 1)] if ahead else [])
    check_values(d, 16, 4, prompt, ahead, 200, seen)

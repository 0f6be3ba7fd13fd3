"""Log-probabilities of packs so large that a workgroup takes several rows, against float64."""
import numpy as np
import pytest
import torch

from paper_2511_18871_amd import binding as B
from tests.rollout import HALF_STEP, U24, check, numpy64

pytestmark = pytest.mark.gpu


def response_rows(prompt_lens, Gs, resp_lens):
    rows, at, r = [], 0, 0
    for p, members in zip(prompt_lens, Gs):
        n = sum(resp_lens[r:r + members])
        rows += range(at + p, at + p + n)
        at, r = at + p + n, r + members
    return np.array(rows)


@pytest.mark.parametrize("dtype,vocab", [(torch.float32, 61), (torch.bfloat16, 1003), (torch.bfloat16, 8200)])         # two waves, eight
def test_rows_without_rules_between_short_prompts(dtype, vocab):
    """Prompts of one and three tokens, so that a workgroup's next response row follows an odd number of others, and nothing to count."""
    groups = 1100
    prompts, Gs = [1 + 2 * (i % 2) for i in range(groups)], [1 + i % 3 for i in range(groups)]
    resp = [1 + (5 * i) % 4 for i in range(sum(Gs))]
    T = sum(prompts) + sum(resp)
    assert T >= 3 * 2048                                 # runs of three rows or more
    gen = torch.Generator().manual_seed(3)
    z = (3 * torch.randn(T, vocab, generator=gen)).to(dtype)
    labels = torch.randint(0, vocab, (T,), generator=gen, dtype=torch.int32)
    g = torch.randn(T, generator=gen)
    temperature = 0.75
    rules = B.LogitRules(temperature=temperature)
    zc, yc, gc = z.cuda(), labels.cuda(), g.cuda()
    logp, lse = B.sp_attn_adjusted_logprob_fwd(zc, yc, yc, rules, prompts, Gs, resp)
    dz = B.sp_attn_adjusted_logprob_bwd(zc, yc, yc, lse, gc, rules, prompts, Gs, resp)
    for _ in range(3):
        again = B.sp_attn_adjusted_logprob_fwd(zc, yc, yc, rules, prompts, Gs, resp)
        assert torch.equal(again[0], logp) and torch.equal(again[1], lse)
    rows = response_rows(prompts, Gs, resp)
    other = np.setdiff1d(np.arange(T), rows)
    assert torch.all(logp[other] == 0) and torch.all(lse[other] == 0) and torch.all(dz[other] == 0)
    want = numpy64(z)[rows] / temperature
    top = want.max(1, keepdims=True)
    L = (top + np.log(np.exp(want - top).sum(1, keepdims=True)))
    y = numpy64(labels)[rows].astype(int)
    # an element: 12 units; an exponential: its argument's rounding (weights that count: above e^-100) and 4 units; a sum of V terms by 128 threads or
    # more: V / 128 + 32 units; the logarithm and its sum: 4 units of L
    size = np.abs(want).max(1)
    tol = U24 * (12 * size + 110 + 4 + 32 + vocab / 128 + 4 * np.maximum(1.0, np.abs(L[:, 0])))
    check("lse", numpy64(lse)[rows], L[:, 0], tol)
    picked = want[np.arange(len(rows)), y] - L[:, 0]
    check("logp", numpy64(logp)[rows], picked, tol + U24 * (12 * size + np.abs(picked)))
    grad = -np.exp(want - L)
    grad[np.arange(len(rows)), y] += 1
    scale = numpy64(g)[rows][:, None] / temperature
    rel = (tol + 12 * U24 * size + 130 * U24)[:, None]
    half = HALF_STEP[dtype] if dtype == torch.bfloat16 else U24
    check("dlogits", numpy64(dz)[rows], grad * scale, np.abs(scale) * (np.exp(want - L) * rel + np.abs(grad) * (half + 4 * U24)) + 1e-37)

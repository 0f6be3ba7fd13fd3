"""Log-probabilities and gradients of rows whose values are large throughout, such as those that an added mask leaves nothing of."""
import math

import pytest
import torch

from paper_2511_18871_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [100, 9000, 40000])
@pytest.mark.parametrize("rules", [(1.0, 0.0, 0.0, 0.7), (1.0, 0.0, 0.0, 0.9), (1.3, 0.0, 0.0, 1.3), (1.0, 0.0, 0.0, 1.0)])
def test_rows_of_one_large_value(dtype, vocab, rules):
    """No weight is above 1: z' is rounded like the largest one of its row, which L is not below."""
    values = [s * x for x in (1e9, 1.1e9, 1e12, 3.3e15, 1e30) for s in (-1, 1)] + [-1e9, -1e30]
    T, prompts, Gs, resp = 1 + len(values), [1], [1], [len(values)]
    z = torch.tensor([0.0] + values)[:, None].repeat(1, vocab)
    z[-1, 3:], z[-2, 7] = -2e30, -9e8                    # a few above the others
    z = z.to(dtype)
    labels = torch.full((T,), 5, dtype=torch.int32)
    labels[-1], labels[-2] = 1, 7
    tokens = torch.full((T,), 50, dtype=torch.int32)
    g = torch.ones(T).cuda()
    r = B.LogitRules(*rules)
    zc, yc, tc = z.cuda(), labels.cuda(), tokens.cuda()
    logp, lse = B.sp_attn_adjusted_logprob_fwd(zc, yc, tc, r, prompts, Gs, resp)
    dz = B.sp_attn_adjusted_logprob_bwd(zc, yc, tc, lse, g, r, prompts, Gs, resp).double().cpu()
    logp, lse = logp.double().cpu(), lse.double().cpu()
    assert torch.isfinite(logp).all() and torch.isfinite(lse).all() and torch.isfinite(dz).all()
    assert (logp <= 0).all()
    # each rounding of L is 2^-24 of it; the history's one id may stand far above or below the others
    assert (logp[1:] >= -math.log(vocab) - 3 * 2.0 ** -24 * lse[1:].abs()).all() or rules[0] != 1.0
    step = max(rules[0], 1 / rules[0]) / rules[3]
    assert (dz.abs() <= step * (1 + 2.0 ** -8)).all()

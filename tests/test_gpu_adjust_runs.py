"""Log-probabilities of packs so large that a workgroup takes several rows, against float64."""
import numpy as np
import pytest
import torch

from oracle import rollout_oracle as ro
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


def history_and_oracle(t, z, tokens, prompts, Gs, resp, rules, bias, allowed):
    """(z', its slope, magnitudes) of response row t."""
    at, r = 0, 0
    for p, members in zip(prompts, Gs):
        start = at + p
        for n in resp[r:r + members]:
            if start <= t < start + n:
                return ro.adjust_row(numpy64(z[t]), tokens[at:at + p].tolist(), tokens[start:t].tolist(), rules, bias, allowed)
            start += n
        at, r = start, r + members
    raise AssertionError("not a response row")


# one slice of eight waves; three, four and five slices; gradients above and below what is stored past the caches
@pytest.mark.parametrize("dtype,vocab,groups", [(torch.bfloat16, 8201, 44), (torch.float32, 30000, 48), (torch.bfloat16, 70003, 15), (torch.bfloat16, 100003, 14), (torch.float32, 131072, 11)])
def test_several_rows_of_several_slices(dtype, vocab, groups):
    """Every row as in a call of its group alone, whose workgroups take one row each; a sample of rows against float64; the gradient in place."""
    gen = torch.Generator().manual_seed(vocab)
    prompts, Gs = [4 + 9 * (i % 3) for i in range(groups)], [2 + i % 3 for i in range(groups)]
    resp = [(53 * i) % 67 for i in range(sum(Gs))]
    T = sum(prompts) + sum(resp)
    assert T * -(-vocab // 32768) >= 2 * 2048                       # runs of two rows or more
    dev = torch.Generator(device="cuda").manual_seed(vocab)
    z = (3 * torch.randn(T, vocab, generator=dev, device="cuda")).to(dtype)
    u = torch.rand(T, generator=gen, dtype=torch.float64)
    tokens = (vocab * u ** 4).to(torch.int32).clamp_(max=vocab - 1)
    allowed = torch.rand(T, (vocab + 31) // 32, 32, generator=dev, device="cuda") < 0.8
    mask = (allowed.long() * (1 << torch.arange(32, device="cuda"))).sum(2).to(torch.int32)
    t64 = tokens.long().cuda()
    word, bit = (t64 // 32)[:, None], (1 << (t64 % 32)).to(torch.int32)[:, None]
    mask.scatter_(1, word, mask.gather(1, word) | bit)
    allowed.view(T, -1).scatter_(1, t64[:, None], True)
    bias, g = torch.randn(vocab, generator=gen), torch.randn(T, generator=gen).cuda()
    numbers = (1.3, 0.4, 0.25, 0.7)
    rules, tc = B.LogitRules(*numbers, bias=bias.cuda()), tokens.cuda()

    def both(z, tokens, mask, g, *pack, dlogits=None):
        logp, lse = B.sp_attn_adjusted_logprob_fwd(z, tokens, tokens, rules, *pack, mask=mask)
        return logp, lse, B.sp_attn_adjusted_logprob_bwd(z, tokens, tokens, lse, g, rules, *pack, mask=mask, dlogits=dlogits, flags=B.SP_FLAG_ZERO_PROMPT_ROWS)

    logp, lse, dz = both(z, tc, mask, g, prompts, Gs, resp)
    at, r = 0, 0
    for p, members in zip(prompts, Gs):
        lens = resp[r:r + members]
        rows = slice(at, at + p + sum(lens))
        alone = both(z[rows].clone(), tc[rows].clone(), mask[rows].clone(), g[rows].clone(), [p], [members], lens)
        assert torch.equal(alone[0], logp[rows]) and torch.equal(alone[1], lse[rows]) and torch.equal(alone[2], dz[rows]), at
        at, r = rows.stop, r + members
    response = response_rows(prompts, Gs, resp)
    sample = response[::max(1, len(response) // 12)][:14]
    for t in sample.tolist():
        want, slope, size = history_and_oracle(t, z, tokens, prompts, Gs, resp, numbers, bias.double().numpy(), allowed[t].flatten()[:vocab].cpu().numpy())
        top = want.max()
        L = top + np.log(np.exp(want - top).sum())
        # as above, with the rules' own operations in the 12 units; 512 threads share a slice
        off = 12 * U24 * size[np.isfinite(want)].max()
        tol = off + U24 * (110 + 4 + 32 + vocab / 512 + 4 * max(1.0, abs(L)))
        y = int(tokens[t])
        assert abs(lse[t].item() - L) <= tol and abs(logp[t].item() - (want[y] - L)) <= tol + off + U24 * abs(want[y] - L)
        pick = np.zeros(vocab)
        pick[y] = 1
        p = np.exp(want - L)
        scale = g[t].item() * slope
        half = HALF_STEP[dtype] if dtype == torch.bfloat16 else U24
        check(f"dlogits {t}", numpy64(dz[t]), (pick - p) * scale, np.abs(scale) * (p * (off + tol + 130 * U24) + np.abs(pick - p) * (half + 4 * U24)) + 1e-37)
    in_place = both(z, tc, mask, g, prompts, Gs, resp, dlogits=z)[2]
    assert in_place.data_ptr() == z.data_ptr() and torch.equal(in_place, dz)

"""The rollout calls together, as a program uses them: prompts enter the cache, responses grow token by token, their logits are
adjusted, and training then sees on the pack what the rollout saw."""
import numpy as np
import pytest
import torch

from oracle import rope_oracle, sp_attn_oracle
from paper_2511_18871_amd import binding as B
from tests.rollout import numpy64

pytestmark = pytest.mark.gpu
BASE = 10000.0


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.float32, 64)])
@pytest.mark.parametrize("graphed", [False, True])
def test_tokens_one_by_one_give_the_rows_of_the_pack(dtype, d, graphed):
    """Rows of sp_attn_fwd on the packed group against rows that appends and decode steps produced."""
    hq, hkv, page, prompts, Gs, steps = 8, 2, 16, [37, 20], [3, 2], 19
    n, scale = sum(Gs), 1 / d ** 0.5
    rl = [steps] * n
    T = sum(prompts) + steps * n
    gen = torch.Generator().manual_seed(2)
    q, k, v = (torch.randn(T, h, d, generator=gen).to(dtype).cuda() for h in (hq, hkv, hkv))
    first = []                                                 # first packed row of every response, and the prompts' rows
    prompt_rows, at = [], 0
    for p, members in zip(prompts, Gs):
        prompt_rows += range(at, at + p)
        first += [at + p + steps * i for i in range(members)]
        at += p + steps * members
    # training side: rope and attention over the pack
    qr, kr = B.sp_attn_rope_qk(q, k, prompts, Gs, rl, BASE)
    o_pack, lse_pack = B.sp_attn_fwd_batched(qr, kr, v, prompts, Gs, rl, scale)
    # rollout side
    cache = B.KvCache(*(torch.zeros(2 * 3 + n * 2, hkv, page, d, dtype=dtype, device="cuda") for _ in range(2)))
    order = torch.randperm(2 * 3 + n * 2, generator=gen).to(torch.int32)
    pt, rt = order[:6].view(2, 3).cuda(), order[6:].view(n, 2).cuda()
    zero = torch.zeros(2, dtype=torch.int32, device="cuda")
    rows = torch.tensor(prompt_rows).cuda()
    k_out = torch.empty(len(prompt_rows), hkv, d, dtype=dtype, device="cuda")
    q_out, prompt_lens = B.sp_attn_cache_append(cache, k[rows], v[rows], pt, zero, BASE, q=q[rows], new_lens=prompts, k_out=k_out)
    assert torch.equal(q_out, qr[rows]) and torch.equal(k_out, kr[rows]) and prompt_lens.tolist() == prompts
    base = torch.tensor([p for p, members in zip(prompts, Gs) for _ in range(members)], dtype=torch.int32).cuda()
    lens, lens_next = torch.zeros(n, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    step_q, step_k, step_v = (torch.empty(n, h, d, dtype=dtype, device="cuda") for h in (hq, hkv, hkv))

    def step():
        rotated, _ = B.sp_attn_cache_append(cache, step_k, step_v, rt, lens, BASE, q=step_q, pos_base=base, lens_out=lens_next)
        out = B.sp_attn_decode(cache, rotated, Gs, pt, prompt_lens, rt, lens_next, scale)
        lens.copy_(lens_next)
        return rotated, out

    if graphed:
        side = torch.cuda.Stream()
        lens.zero_()
        with torch.cuda.stream(side):
            step()
        side.synchronize()
        lens.zero_()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            result = step()
    for i in range(steps):
        at = torch.tensor(first).cuda() + i
        for buf, x in ((step_q, q), (step_k, k), (step_v, v)):
            buf.copy_(x[at])
        if graphed:
            graph.replay()
        else:
            result = step()
        torch.cuda.synchronize()
        rotated, (o, lse) = result
        assert torch.equal(rotated, qr[at])
        # both sides are within 2^-8 of a weighted mean of |v| below 6 twice over (weights and output rounded); float32 within 1e-5
        tol = 2 * 2 * 2.0 ** -8 if dtype == torch.bfloat16 else 1e-5
        assert (o.float() - o_pack[at].float()).abs().max().item() <= tol * 2
        assert (lse - lse_pack[:, at]).abs().max().item() <= 2e-5
    assert lens.tolist() == [steps] * n


def test_a_step_over_a_padded_batch():
    """Sequences that have ended ride along with a negative length: nothing of theirs is written, their rows are zero."""
    d, hq, hkv, n = 128, 4, 2, 4
    gen = torch.Generator().manual_seed(6)
    kc, vc = (torch.randn(9, hkv, 16, d, generator=gen).bfloat16().cuda() for _ in range(2))
    q, k, v = (torch.randn(n, h, d, generator=gen).bfloat16().cuda() for h in (hq, hkv, hkv))
    tables = torch.tensor([[0, 1], [2, 3], [4, 5], [-1, -1]], dtype=torch.int32).cuda()
    lens = torch.tensor([16, -1, 3, -5], dtype=torch.int32).cuda()
    k0 = kc.clone()
    cache = B.KvCache(kc, vc)
    q_out, now = B.sp_attn_cache_append(cache, k, v, tables, lens, BASE, q=q, q_out=torch.zeros_like(q))
    o, lse = B.sp_attn_decode(cache, q_out, [2, 2], torch.tensor([[6], [7]], dtype=torch.int32).cuda(), torch.tensor([10, 16], dtype=torch.int32).cuda(), tables, now, 0.1)
    torch.cuda.synchronize()
    assert now.tolist() == [17, -1, 4, -5]
    changed = (kc != k0).flatten(1).any(1).nonzero().flatten().tolist()
    assert changed == [1, 4]
    assert torch.all(o[[1, 3]] == 0) and torch.all(torch.isneginf(lse[:, [1, 3]])) and torch.isfinite(lse[:, [0, 2]]).all()


def test_sampled_under_rules_and_trained_under_the_same():
    """The log-probabilities of tokens drawn from adjusted logits step by step are those that training forms on the pack, and the
    gradient of the policy objective arrives at the raw logits."""
    vocab, prompts, Gs, steps = 300, [6, 4], [2, 1], 7
    n, rl = 3, [7, 7, 7]
    T = sum(prompts) + steps * n
    gen = torch.Generator().manual_seed(9)
    logits = (2 * torch.randn(T, vocab, generator=gen)).cuda()
    tokens = torch.randint(0, vocab, (T,), generator=gen, dtype=torch.int32).cuda()
    group_first = [0, prompts[0] + 2 * steps]
    first = [prompts[0], prompts[0] + steps, group_first[1] + prompts[1]]
    prompt_tokens = torch.zeros(2, 6, dtype=torch.int32, device="cuda")
    for g, p in enumerate(prompts):
        prompt_tokens[g, :p] = tokens[group_first[g]:group_first[g] + p]
    plens = torch.tensor(prompts, dtype=torch.int32).cuda()
    rules = B.LogitRules(1.2, 0.3, 0.2, 0.9)
    resp_tokens, resp_lens = torch.zeros(n, steps, dtype=torch.int32, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
    drawn = torch.zeros(T, device="cuda")
    u = torch.rand(steps, n, vocab, generator=gen).cuda()
    for i in range(steps):
        at = torch.tensor(first).cuda() + i
        z = B.sp_attn_adjust_logits(logits[at], rules, Gs, prompt_tokens, plens, resp_tokens, resp_lens)
        token = (z - torch.log(-torch.log(u[i]))).argmax(1)
        drawn[at] = torch.log_softmax(z.double(), 1).gather(1, token[:, None])[:, 0].float()
        resp_tokens[:, i] = token.int()
        resp_lens += 1
        tokens[at] = token.int()
    logp, lse = B.sp_attn_adjusted_logprob_fwd(logits, tokens, tokens, rules, prompts, Gs, rl)
    assert (logp - drawn).abs().max().item() <= 1e-5
    adv = torch.tensor([0.5, -1.0, 0.25]).cuda()
    loss, g = B.sp_attn_grpo_loss(logp, drawn, drawn, adv, prompts, Gs, rl)
    dz = B.sp_attn_adjusted_logprob_bwd(logits, tokens, tokens, lse, g, rules, prompts, Gs, rl)
    # a step along a random direction changes the loss by the gradient's share of it
    way = torch.randn(T, vocab, generator=gen).cuda()
    def loss_at(eps):
        lp, _ = B.sp_attn_adjusted_logprob_fwd(logits + eps * way, tokens, tokens, rules, prompts, Gs, rl)
        return B.sp_attn_grpo_loss(lp, drawn, drawn, adv, prompts, Gs, rl)[0].double().item()
    eps = 2.0 ** -8
    slope = (loss_at(eps) - loss_at(-eps)) / (2 * eps)
    want = (dz.double() * way.double()).sum().item()
    # third-order term eps^2 / 6 |way|^3-like, and losses off by 1e-6 over 2 eps
    assert abs(slope - want) <= 1e-3 * max(1.0, abs(want))

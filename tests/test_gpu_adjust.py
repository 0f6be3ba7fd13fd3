"""Adjusted logits, their log-probabilities and the gradient on the GPU, element by element against the fp64 oracle."""
import numpy as np
import pytest
import torch

from oracle import rollout_oracle as ro
from paper_2511_18871_amd import binding as B
from tests.rollout import HALF_STEP, U24, check, numpy64

pytestmark = pytest.mark.gpu
RULES = {"all": (1.3, 0.4, 0.25, 0.7), "none": (1.0, 0.0, 0.0, 1.0), "repetition": (0.8, 0.0, 0.0, 1.0), "counts": (1.0, -0.3, 0.6, 1.5)}


def random_mask(gen, rows, vocab, share=0.5, stride=None):
    words = stride or -(-vocab // 32)
    bits = torch.rand(rows, words, 32, generator=gen) < share
    weights = (1 << torch.arange(32, dtype=torch.int64))
    return (bits.long() * weights).sum(2).to(torch.int32)


def some_tokens(gen, shape, vocab):
    u = torch.rand(shape, generator=gen, dtype=torch.float64)
    return (vocab * u ** 3).to(torch.int32).clamp_(max=vocab - 1)


def adjust_case(dtype, vocab, Gs, prompts, resp, seed, masked=True, biased=True, extra=0):
    gen = torch.Generator().manual_seed(seed)
    n = len(resp)
    z = (3 * torch.randn(n, vocab + extra, generator=gen)).to(dtype)
    pt = some_tokens(gen, (len(prompts), max(1, max(prompts, default=1))), vocab)
    rt = some_tokens(gen, (n, max(1, max(resp))), vocab)
    return z, pt, rt, random_mask(gen, n, vocab) if masked else None, torch.randn(vocab, generator=gen) if biased else None


def dev32(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def adjust_oracle(z, pt, rt, mask, bias, Gs, prompts, resp, rules):
    vocab = z.shape[1]
    allowed = None if mask is None else ro.unpack_mask(mask.numpy(), vocab)
    out, sizes, s = [], [], 0
    for g, members in enumerate(Gs):
        for _ in range(members):
            o, _, size = ro.adjust_row(numpy64(z[s]), pt[g, :max(0, prompts[g])].tolist() if pt is not None else [], rt[s, :max(0, resp[s])].tolist() if rt is not None else [],
                                       rules, None if bias is None else numpy64(bias), None if allowed is None else allowed[s])
            out.append(o)
            sizes.append(size)
            s += 1
    return np.array(out), np.array(sizes)


def adjust_bound(ref, size, dtype):
    """Five float32 operations on what went into an element, with reciprocals in place of two divisions: 12 units; then one rounding."""
    return 12 * U24 * size + (HALF_STEP[dtype] if dtype == torch.bfloat16 else U24) * np.abs(np.where(np.isfinite(ref), ref, 0.0)) + 1e-37


@pytest.mark.parametrize("rules", list(RULES))
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("vocab", [1, 7, 8, 31, 1000, 1003, 5003])
def test_adjust(rules, dtype, vocab):
    Gs, prompts, resp = [2, 0, 3, 1], [9, 4, 0, 40], [0, 3, 60, 1, 17, 300]
    z, pt, rt, mask, bias = adjust_case(dtype, vocab, Gs, prompts, resp, 7)
    out = B.sp_attn_adjust_logits(z.cuda(), B.LogitRules(*RULES[rules], bias=bias.cuda()), Gs, pt.cuda(), dev32(prompts), rt.cuda(), dev32(resp), mask=mask.cuda())
    ref, size = adjust_oracle(z, pt, rt, mask, bias, Gs, prompts, resp, RULES[rules])
    check("adjusted", out, ref, adjust_bound(ref, size, dtype))


@pytest.mark.parametrize("vocab", [32768, 32769, 70001, 151936])
def test_adjust_many_slices(vocab):
    Gs, prompts, resp = [1, 2], [500, 20], [40, 700, 0]
    z, pt, rt, mask, bias = adjust_case(torch.bfloat16, vocab, Gs, prompts, resp, 8)
    out = B.sp_attn_adjust_logits(z.cuda(), B.LogitRules(*RULES["all"], bias=bias.cuda()), Gs, pt.cuda(), dev32(prompts), rt.cuda(), dev32(resp), mask=mask.cuda())
    ref, size = adjust_oracle(z, pt, rt, mask, bias, Gs, prompts, resp, RULES["all"])
    check("adjusted", out, ref, adjust_bound(ref, size, torch.bfloat16))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_adjust_strides_in_place_and_without_parts(dtype):
    vocab, Gs, prompts, resp = 1003, [2, 1], [12, 5], [6, 0, 33]
    z, pt, rt, mask, bias = adjust_case(dtype, vocab, Gs, prompts, resp, 9, extra=13)
    rules = RULES["all"]
    for use_p, use_r, use_m, use_b in ((1, 1, 1, 1), (0, 1, 0, 1), (1, 0, 1, 0), (0, 0, 0, 0)):
        whole = z.cuda()
        view = whole[:, :vocab]
        p, r, m, b = (pt if use_p else None), (rt if use_r else None), (mask if use_m else None), (bias if use_b else None)
        out = B.sp_attn_adjust_logits(view, B.LogitRules(*rules, bias=None if b is None else b.cuda()), Gs, None if p is None else p.cuda(),
                                      dev32(prompts) if use_p else None, None if r is None else r.cuda(), dev32(resp) if use_r else None,
                                      mask=None if m is None else m.cuda(), out=view)
        assert out.data_ptr() == whole.data_ptr() and torch.equal(whole[:, vocab:].cpu(), z[:, vocab:])
        ref, size = adjust_oracle(z[:, :vocab], p, r, m, b, Gs, prompts, resp, rules)
        check("adjusted", out, ref, adjust_bound(ref, size, dtype))


def test_adjust_ids_and_lengths_out_of_range_and_special_values():
    vocab = 200
    z = torch.zeros(3, vocab)
    z[0, :4] = torch.tensor([float("nan"), float("inf"), -float("inf"), -0.0])
    z[1, 5], z[1, 6] = float("nan"), float("inf")
    z[2] = torch.finfo(torch.float32).min
    pt = torch.tensor([[3, -1, vocab, 2 ** 31 - 1, -2 ** 31, 5]], dtype=torch.int32)
    rt = torch.tensor([[1, 2, 199, 199], [5, 6, 6, -7], [0, 0, 0, 0]], dtype=torch.int32)
    mask = torch.full((3, 7), -1, dtype=torch.int32)
    mask[1, 0] = ~((1 << 5) | (1 << 6))                              # NaN and infinity in masked places
    out = B.sp_attn_adjust_logits(z.cuda(), B.LogitRules(2.0, 0.5, 0.25, 1.0), [3], pt.cuda(), dev32([100]), rt.cuda(), dev32([4, 100, -3]), mask=mask.cuda()).cpu()
    assert torch.isnan(out[0, 0]) and out[0, 1] == float("inf") and out[0, 2] == -float("inf") and out[0, 3] == 0 and out[0, 199] == -1.0
    assert torch.all(torch.isneginf(out[1, 5:7])) and torch.all(out[1, :5] == 0) and torch.all(out[1, 7:] == 0)
    assert out[2, 0] == torch.finfo(torch.float32).min and out[2, 3] == -float("inf") and out[2, 5] == -float("inf")


def test_adjust_counts_that_end_at_15_bits():
    vocab, n = 64, 40000
    rt = torch.zeros(2, n, dtype=torch.int32)
    rt[0, 39990:] = 9
    rt[1] = 3
    rt[1, :32766] = 2
    pt = torch.tensor([[0, 1, 2, 3]], dtype=torch.int32)
    z = torch.zeros(2, vocab)
    out = B.sp_attn_adjust_logits(z.cuda(), B.LogitRules(1.0, 0.0, 1.0, 1.0), [2], pt.cuda(), dev32([4]), rt.cuda(), dev32([n, n])).cpu()
    assert out[0, 0] == -32767 and out[0, 9] == -10 and torch.count_nonzero(out[0]) == 2
    assert out[1, 2] == -32766 and out[1, 3] == -(n - 32766) and torch.count_nonzero(out[1]) == 2


def test_adjust_more_groups_and_rows_than_a_launch_holds():
    """Groups beyond a kernel argument, and rows beyond a grid's second dimension, with empty groups in between."""
    vocab = 16
    Gs = [i % 3 for i in range(2000)] + [33000, 0, 2]
    n = sum(Gs)
    gen = torch.Generator().manual_seed(4)
    pt = torch.randint(0, vocab, (len(Gs), 2), generator=gen, dtype=torch.int32)
    group = torch.repeat_interleave(torch.arange(len(Gs)), torch.tensor(Gs))
    z = torch.randn(n, vocab, generator=gen)
    out = B.sp_attn_adjust_logits(z.cuda(), B.LogitRules(2.0), Gs, pt.cuda(), torch.full((len(Gs),), 2, dtype=torch.int32).cuda(), None, None).cpu()
    seen = torch.zeros(n, vocab, dtype=torch.bool).scatter_(1, pt[group].long(), True)
    assert torch.equal(out, torch.where(seen, torch.where(z > 0, z / 2, z * 2), z))


PACKS = {
    "ragged": ([5, 0, 3], [3, 2, 0], [4, 0, 7, 2, 9]),
    "one_group": ([17], [6], [3, 1, 0, 8, 2, 5]),
    "no_prompt": ([0], [2], [6, 3]),
    "long": ([40], [3], [70, 1, 33]),
}


def pack_case(pack, vocab, dtype, seed, share=0.6):
    pl, Gs, rl = PACKS[pack]
    T = sum(pl) + sum(rl)
    gen = torch.Generator().manual_seed(seed)
    z = (3 * torch.randn(T, vocab, generator=gen)).to(dtype)
    tokens = some_tokens(gen, (T,), vocab)
    labels = tokens.clone()
    mask = random_mask(gen, T, vocab, share)
    for t in range(T):
        mask[t, labels[t] // 32] |= (1 << int(labels[t] % 32)) - (1 << 32 if labels[t] % 32 == 31 else 0)
    return pl, Gs, rl, z, tokens, labels, mask, torch.randn(vocab, generator=gen), torch.randn(T, generator=gen)


def logprob_check(pl, Gs, rl, z, tokens, labels, mask, bias, g, rules, own=False, in_place=False):
    vocab, dtype = z.shape[1], z.dtype
    allowed = None if mask is None else ro.unpack_mask(mask.numpy(), vocab)
    rows, rlogp, rlse, rdz, size = ro.adjusted_logprob(numpy64(z), labels.tolist(), tokens.tolist(), numpy64(g), rules, pl, Gs, rl,
                                                       None if bias is None else numpy64(bias), allowed, own)
    T = z.shape[0]
    flags = B.SP_FLAG_OWN_TOKEN if own else 0
    r = B.LogitRules(*rules, bias=None if bias is None else bias.cuda())
    zc, yc, tc, mc = z.cuda(), labels.cuda(), tokens.cuda(), None if mask is None else mask.cuda()
    logp0, lse0, dz0 = torch.full((T,), 5.0, device="cuda"), torch.full((T,), 6.0, device="cuda"), torch.full_like(zc, 3.0)
    logp, lse = B.sp_attn_adjusted_logprob_fwd(zc, yc, tc, r, pl, Gs, rl, mask=mc, flags=flags, logp=logp0, lse=lse0)
    dz = B.sp_attn_adjusted_logprob_bwd(zc, yc, tc, lse, g.cuda(), r, pl, Gs, rl, mask=mc, flags=flags, dlogits=dz0)
    zeroed = B.sp_attn_adjusted_logprob_bwd(zc, yc, tc, lse, g.cuda(), r, pl, Gs, rl, mask=mc, flags=flags)
    again = B.sp_attn_adjusted_logprob_fwd(zc, yc, tc, r, pl, Gs, rl, mask=mc, flags=flags)
    other = np.setdiff1d(np.arange(T), rows)
    resp = torch.tensor(rows)
    assert torch.all(logp.cpu()[other] == 5.0) and torch.all(lse.cpu()[other] == 6.0) and torch.all(dz.cpu()[other] == 3.0)
    assert torch.all(zeroed.cpu()[other] == 0) and torch.equal(zeroed.cpu()[resp], dz.cpu()[resp])
    assert torch.equal(again[0].cpu()[resp], logp.cpu()[resp]) and torch.equal(again[1].cpu()[resp], lse.cpu()[resp])
    assert torch.all(again[0].cpu()[other] == 0) and torch.all(again[1].cpu()[other] == 0)
    # an adjusted element is 12 units of what went into it off; an exponential of a difference adds the argument's rounding (weights that count:
    # above e^-100) and 4 units; a sum of V terms, which 512 threads share, V / 512 + 32 units; the logarithm and its sum 4 units of lse
    z_off = 12 * U24 * size
    lse_tol = z_off + U24 * (110 + 4 + 32 + vocab / 512) + 4 * U24 * np.maximum(1.0, np.abs(np.where(np.isfinite(rlse), rlse, 0.0)))
    check("lse", numpy64(lse)[rows], rlse, lse_tol)
    check("logp", numpy64(logp)[rows], rlogp, lse_tol + z_off + U24 * np.abs(np.where(np.isfinite(rlogp), rlogp, 0.0)))
    rel = (z_off + lse_tol + 130 * U24)[:, None]
    top = np.abs(g.numpy().astype(np.float64))[rows][:, None] * max(1.0, rules[0], 1 / rules[0]) / rules[3]
    check("dlogits", numpy64(dz)[rows], rdz, np.abs(rdz) * ((HALF_STEP[dtype] if dtype == torch.bfloat16 else 0.0) + 2 * rel) + rel * top * np.minimum(1.0, np.abs(rdz) / top + 1e-3) + 1e-37)
    if in_place:
        B.sp_attn_adjusted_logprob_bwd(zc, yc, tc, lse, g.cuda(), r, pl, Gs, rl, mask=mc, flags=flags, dlogits=zc)
        assert torch.equal(zc.cpu()[resp], dz.cpu()[resp]) and torch.equal(zc.cpu()[other], z[other])
    return logp, lse, dz


@pytest.mark.parametrize("pack", list(PACKS))
@pytest.mark.parametrize("dtype,vocab", [(torch.bfloat16, 4096), (torch.float32, 1000), (torch.bfloat16, 1003), (torch.float32, 37)])
def test_logprob(pack, dtype, vocab):
    pl, Gs, rl, z, tokens, labels, mask, bias, g = pack_case(pack, vocab, dtype, 11)
    logprob_check(pl, Gs, rl, z, tokens, labels, mask, bias, g, RULES["all"], in_place=True)


def test_logprob_several_rows_to_a_workgroup():
    """More rows than the chip takes at once, of a vocabulary that one workgroup has to itself, and prompts between them."""
    gen = torch.Generator().manual_seed(17)
    vocab, pl, Gs, rl = 61, [700, 1, 30], [5, 4, 9], [(97 * i) % 700 + 1 for i in range(18)]
    T = sum(pl) + sum(rl)
    z, tokens = 3 * torch.randn(T, vocab, generator=gen), some_tokens(gen, (T,), vocab)
    mask = random_mask(gen, T, vocab, 0.7)
    logprob_check(pl, Gs, rl, z, tokens, some_tokens(gen, (T,), vocab), mask, torch.randn(vocab, generator=gen), torch.randn(T, generator=gen), RULES["all"])


@pytest.mark.parametrize("dtype,vocab", [(torch.bfloat16, 8192), (torch.float32, 8193), (torch.bfloat16, 20000), (torch.float32, 32768), (torch.bfloat16, 32769)])
def test_logprob_either_side_of_a_workgroups_sizes(dtype, vocab):
    pl, Gs, rl, z, tokens, labels, mask, bias, g = pack_case("ragged", vocab, dtype, 12)
    logprob_check(pl, Gs, rl, z, tokens, labels, mask, bias, g, RULES["all"])


@pytest.mark.parametrize("rules", list(RULES))
@pytest.mark.parametrize("own", [False, True])
def test_logprob_rules_and_own_token(rules, own):
    pl, Gs, rl, z, tokens, labels, mask, bias, g = pack_case("long", 500, torch.float32, 12)
    logprob_check(pl, Gs, rl, z, tokens, labels, mask if own else None, None if own else bias, g, RULES[rules], own=own)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_logprob_many_slices(dtype):
    pl, Gs, rl, z, tokens, labels, mask, bias, g = pack_case("one_group", 70001, dtype, 13)
    logprob_check(pl, Gs, rl, z, tokens, labels, mask, bias, g, RULES["all"])


def test_logprob_runs_that_cross_segments():
    """Packs of so many tokens that a workgroup's run of rows holds several responses and a prompt's end."""
    PACKS["crossing"] = ([31, 2] * 20, [9, 3] * 20, [3, 5, 0, 1, 9, 2, 4, 30, 7, 11, 0, 6] * 20)
    pl, Gs, rl, z, tokens, labels, mask, bias, g = pack_case("crossing", 40, torch.float32, 14)
    logprob_check(pl, Gs, rl, z, tokens, labels, mask, bias, g, RULES["all"])
    big = [30] * 60, [40] * 60, [3, 1] * 1200
    PACKS["crossing"] = big
    pl, Gs, rl, z, tokens, labels, mask, bias, g = pack_case("crossing", 33, torch.bfloat16, 15)
    logprob_check(pl, Gs, rl, z, tokens, labels, mask, bias, g, RULES["all"])


def test_logprob_without_rules_is_the_ordinary_one():
    pl, Gs, rl, z, tokens, labels, _, _, g = pack_case("ragged", 4096, torch.bfloat16, 16)
    zc, yc = z.cuda(), labels.cuda()
    a = B.sp_attn_adjusted_logprob_fwd(zc, yc, tokens.cuda(), B.LogitRules(), pl, Gs, rl)
    b = B.sp_attn_logprob_fwd(zc, yc, pl, Gs, rl)
    assert torch.allclose(a[0], b[0], rtol=0, atol=4e-6) and torch.allclose(a[1], b[1], rtol=0, atol=4e-6)


def test_logprob_rows_that_allow_nothing_and_odd_labels():
    pl, Gs, rl, z, tokens, labels, mask, _, g = pack_case("one_group", 100, torch.float32, 17)
    mask[20] = 0                                         # nothing allowed
    mask[21, labels[21] // 32] = 0                       # the label masked
    labels[22], labels[23] = -1, 100
    z[24] = -float("inf")                                # nothing left by value
    z[25, :3] = float("nan")                             # NaN and infinity in masked places
    z[25, 3] = float("inf")
    mask[25, 0] = mask[25, 0] & ~15
    labels[25] = 50
    mask[25, 1] = -1
    z[26] = torch.finfo(torch.float32).min               # the lowest value throughout
    mask[26] = -1
    allowed = ro.unpack_mask(mask.numpy(), 100)
    zz = torch.where(torch.tensor(allowed), z, 0.0).contiguous()
    logp, lse, dz = logprob_check(pl, Gs, rl, zz, tokens, labels, mask, None, g, (1.0, 0.0, 0.0, 1.0))
    r = B.LogitRules()
    logp2, lse2 = B.sp_attn_adjusted_logprob_fwd(z.cuda(), labels.cuda(), tokens.cuda(), r, pl, Gs, rl, mask=mask.cuda())
    dz2 = B.sp_attn_adjusted_logprob_bwd(z.cuda(), labels.cuda(), tokens.cuda(), lse2, g.cuda(), r, pl, Gs, rl, mask=mask.cuda())
    assert torch.equal(logp2[17:], logp[17:]) and torch.equal(lse2[17:], lse[17:]) and torch.equal(dz2[17:], dz[17:])
    assert all(logp2[t].item() == -float("inf") for t in (20, 21, 22, 23, 24)) and lse2[20].item() == lse2[24].item() == -float("inf")
    assert torch.all(dz2[20] == 0) and torch.all(dz2[24] == 0) and torch.isfinite(dz2[25]).all()


def test_logprob_long_response_saturates_its_counts():
    n, vocab = 33000, 8
    pl, Gs, rl = [1], [1], [n]
    tokens = torch.ones(n + 1, dtype=torch.int32)
    z = torch.zeros(n + 1, vocab)
    logp, lse = B.sp_attn_adjusted_logprob_fwd(z.cuda(), tokens.cuda(), tokens.cuda(), B.LogitRules(frequency=1e-4), pl, Gs, rl)
    c = np.minimum(np.arange(n), ro.COUNT_MAX) * np.float64(np.float32(1e-4))
    want = np.log(vocab - 1 + np.exp(-c))
    assert np.abs(numpy64(lse)[1:] - want).max() < 1e-5 and np.abs(numpy64(logp)[1:] + c + want).max() < 1e-5


def test_logprob_captured_and_replayed():
    pl, Gs, rl, z, tokens, labels, mask, bias, g = (x.cuda() if torch.is_tensor(x) else x for x in pack_case("long", 40000, torch.bfloat16, 18))
    rules = B.LogitRules(*RULES["all"], bias=bias)
    def both():
        logp, lse = B.sp_attn_adjusted_logprob_fwd(z, labels, tokens, rules, pl, Gs, rl, mask=mask)
        return logp, lse, B.sp_attn_adjusted_logprob_bwd(z, labels, tokens, lse, g, rules, pl, Gs, rl, mask=mask)
    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for step in range(3):
        z.copy_(torch.randn_like(z, dtype=torch.float32) * (1 + step))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, both()):
            assert torch.equal(a, b), step

"""CPU pins of the rollout oracle: against the oracles of the pack, autograd, differences and hand-made cases."""
import numpy as np
import pytest
import torch

from oracle import loss_oracle, rollout_oracle as ro, rope_oracle, sp_attn_oracle


def test_decode_is_the_last_row_of_the_pack():
    rng = np.random.default_rng(1)
    prompt, lens, hq, hkv, d, page = 21, [5, 1, 9], 4, 2, 16, 16
    T = prompt + sum(lens)
    q, k, v = (rng.standard_normal((T, h, d)) for h in (hq, hkv, hkv))
    o, lse = sp_attn_oracle.sp_attn_fwd(q, k, v, prompt, lens, 0.2)
    kc, vc = np.zeros((8, hkv, page, d)), np.zeros((8, hkv, page, d))
    pt, rt = [[4, 1]], [[0, 2], [3, 5], [7, 6]]
    start = prompt + np.cumsum([0] + lens[:-1])
    for cache, x in ((kc, k), (vc, v)):
        for j in range(prompt):
            cache[pt[0][j // page], :, j % page] = x[j]
        for r in range(3):
            for j in range(lens[r]):
                cache[rt[r][j // page], :, j % page] = x[start[r] + j]
    last = start + np.array(lens) - 1
    got, glse, weight, _, count = ro.decode(kc, vc, q[last], [3], pt, [prompt], rt, lens, 0.2)
    assert np.allclose(got, o[last], atol=1e-12) and np.allclose(glse, lse[:, last], atol=1e-12)
    assert count.tolist() == [prompt + n for n in lens] and np.all(weight >= np.abs(got) - 1e-12)


def test_append_turns_as_the_rotation_over_the_pack():
    rng = np.random.default_rng(2)
    prompt, lens, d = 6, [3, 2], 8
    T = prompt + sum(lens)
    x, v = rng.standard_normal((T, 2, d)), rng.standard_normal((T, 2, d))
    want = rope_oracle.rope_rotate(x, rope_oracle.positions_batched([prompt], [2], lens), 100.0)
    kc, vc = np.zeros((4, 2, 4, d)), np.zeros((4, 2, 4, d))
    kc, vc, _, k_out, n = ro.cache_append(kc, vc, x[:prompt], x[:prompt], v[:prompt], [prompt], [[2, 0]], [0], None, 100.0)
    assert np.allclose(k_out, want[:prompt]) and np.allclose(kc[2].transpose(1, 0, 2), want[:4]) and np.allclose(kc[0].transpose(1, 0, 2)[:2], want[4:6])
    for i in range(2):          # response tokens one at a time
        rows = [prompt + i, prompt + 3 + i]
        kc, vc, q_out, _, n = ro.cache_append(kc, vc, x[rows], x[rows], v[rows], [1, 1], [[1], [3]], [i, i], [prompt, prompt], 100.0)
        assert np.allclose(q_out, want[rows]) and n.tolist() == [i + 1, i + 1]
        assert np.allclose(vc[3, :, i], v[rows[1]])


def test_adjust_by_hand():
    z = np.array([2.0, -2.0, 0.0, 1.0, 4.0])
    out, slope, _ = ro.adjust_row(z, [0, 1], [1, 3, 3], (2.0, 0.5, 0.25, 2.0), bias=np.array([0, 0, 0, 1.0, 0]), allowed=np.array([1, 1, 1, 1, 0], bool))
    assert out.tolist() == [0.5, (-4 - 0.25 - 0.5) / 2, 0.0, (1.0 - 0.5 - 0.5) / 2, -np.inf]
    assert slope.tolist() == [0.25, 1.0, 0.5, 0.25, 0.0]


def adjusted_torch(z, prompt, generated, rules, bias, allowed):
    """The rules once more, for whole rows and for autograd."""
    rho, presence, frequency, temperature = rules
    counts = torch.bincount(torch.tensor(generated, dtype=torch.long), minlength=len(z)).double()
    seen = (counts + torch.bincount(torch.tensor(prompt, dtype=torch.long), minlength=len(z))) > 0
    a = z + bias
    a = torch.where(seen, torch.where(a > 0, a / rho, a * rho), a)
    return ((a - frequency * counts - presence * (counts > 0).double()) / temperature).masked_fill(~allowed, -torch.inf)


@pytest.mark.parametrize("own", [False, True])
def test_logprob_and_gradient_against_autograd_and_differences(own):
    rng = np.random.default_rng(3)
    pl, Gs, rl, V = [4, 0], [2, 1], [3, 2, 5], 12
    T = sum(pl) + sum(rl)
    z, bias, g = rng.standard_normal((T, V)) * 2, rng.standard_normal(V), rng.standard_normal(T)
    tokens = rng.integers(0, V, T).tolist()
    allowed = rng.random((T, V)) < 0.8
    allowed[np.arange(T), tokens] = True
    rules = (1.5, 0.3, 0.2, 0.6)
    args = (tokens, tokens, g, rules, pl, Gs, rl, bias, allowed, own)
    rows, logp, lse, grad, _ = ro.adjusted_logprob(z, *args)
    starts = {4: (0, 4), 7: (0, 4), 9: (9, 9)}
    total, zt = 0.0, torch.tensor(z, requires_grad=True)
    for i, t in enumerate(rows):
        s = max(x for x in starts if x <= t)
        p0, p1 = starts[s]
        row = adjusted_torch(zt[t], tokens[p0:p1], tokens[s:t + int(own)], rules, torch.tensor(bias), torch.tensor(allowed[t]))
        lp = torch.log_softmax(row, 0)[tokens[t]]
        assert abs(lp.item() - logp[i]) < 1e-12 and abs(torch.logsumexp(row, 0).item() - lse[i]) < 1e-12
        total = total + g[t] * lp
    total.backward()
    assert np.allclose(zt.grad.numpy()[rows], grad, atol=1e-12)
    eps = 1e-6
    for _ in range(20):
        t, v = rng.choice(rows), rng.integers(0, V)
        up, down = z.copy(), z.copy()
        up[t, v] += eps
        down[t, v] -= eps
        f = lambda x: float((ro.adjusted_logprob(x, *args)[1] * g[rows]).sum())
        assert abs((f(up) - f(down)) / (2 * eps) - grad[list(rows).index(t), v]) < 1e-6


def test_no_rules_give_the_ordinary_log_probability():
    rng = np.random.default_rng(4)
    pl, Gs, rl, V = [3], [2], [4, 1], 9
    z, y, g = rng.standard_normal((8, V)), rng.integers(0, V, 8), rng.standard_normal(8)
    idx = loss_oracle.response_index(pl, Gs, rl)
    logp, lse = loss_oracle.logprob_fwd(z, y, idx)
    rows, lp, L, grad, _ = ro.adjusted_logprob(z, y.tolist(), y.tolist(), g, (1.0, 0.0, 0.0, 1.0), pl, Gs, rl)
    assert np.allclose(lp, logp[rows]) and np.allclose(L, lse[rows]) and np.allclose(grad, loss_oracle.logprob_bwd(z, y, g, idx)[rows])


def test_mask_bits():
    words = np.array([[0x80000001, 0x2]], dtype=np.uint32)
    assert np.flatnonzero(ro.unpack_mask(words, 40)[0]).tolist() == [0, 31, 33]
    assert np.flatnonzero(ro.unpack_mask(words.view(np.int32), 40)[0]).tolist() == [0, 31, 33]

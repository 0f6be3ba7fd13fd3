"""Pins of the oracle of branching sequences, on what it has to agree with: rows of one token at a time, and the same tokens appended anew."""
import numpy as np
import torch

from oracle import rollout_oracle as ro
from tests.branching import random_trees
from tests.rollout import make_tables

RNG = np.random.default_rng(3)


def setup(seed, prompts, resp, page=16, hq=4, hkv=2, d=8):
    gen = torch.Generator().manual_seed(seed)
    tables, pages = make_tables(gen, prompts + resp, page)
    kc, vc = (torch.randn(pages, hkv, page, d, generator=gen).double().numpy() for _ in range(2))
    return gen, kc, vc, tables[:len(prompts)].tolist(), tables[len(prompts):].tolist()


def test_a_chain_is_its_tokens_one_by_one():
    prompts, Gs, new, resp = [21, 0], [2, 1], [3, 1, 5], [9, 30, 5]
    gen, kc, vc, pt, rt = setup(1, prompts, resp)
    q = torch.randn(sum(new), 4, 8, generator=gen).double().numpy()
    o, lse, *_ = ro.tree_decode(kc, vc, q, Gs, new, None, pt, prompts, rt, resp, 0.3)
    t = 0
    for s, n in enumerate(new):
        for i in range(n):
            g = 0 if s < 2 else 1
            one, one_lse, *_ = ro.decode(kc, vc, q[t:t + 1], [1], [pt[g]], [prompts[g]], [rt[s]], [resp[s] - n + i + 1], 0.3)
            assert np.allclose(o[t], one[0], atol=1e-13) and np.allclose(lse[:, t], one_lse[:, 0], atol=1e-13)
            t += 1


def test_a_row_of_a_tree_is_its_path_kept():
    """Attention of a drafted token equals that of the last token of a sequence that kept its path."""
    prompts, resp, n = [19], [40], 12
    gen, kc, vc, pt, rt = setup(2, prompts, resp)
    rows = random_trees(gen, [n])
    q = torch.randn(n, 4, 8, generator=gen).double().numpy()
    o, lse, *_ = ro.tree_decode(kc, vc, q, [1], [n], rows, pt, prompts, rt, resp, 0.3)
    for t, path in enumerate(rows):
        (k2, v2), now = ro.cache_keep([kc[None], vc[None]], rt, [resp[0] - n], [path], [len(path)])
        assert now == [resp[0] - n + len(path)]
        one, one_lse, *_ = ro.decode(k2[0], v2[0], q[t:t + 1], [1], pt, prompts, rt, now, 0.3)
        assert np.allclose(o[t], one[0], atol=1e-13) and np.allclose(lse[:, t], one_lse[:, 0], atol=1e-13)


def test_fits_and_forks_count_their_pages():
    refs, page, rng = [0] * 30, 16, np.random.default_rng(4)
    tables, lens = [[-1] * 6 for _ in range(5)], [0] * 5
    for _ in range(40):
        lens = [int(x) for x in rng.integers(0, 90, 5)]
        refs, tables, missing = ro.pages_fit(refs, page, tables, lens)
        held = [p for t in tables for p in t if p >= 0]
        assert all(refs[p] == held.count(p) for p in range(30)) and missing == sum(-(-n // page) for n in lens) - len(held)
    cache = rng.standard_normal((2, 30, 1, page, 2))
    refs, tables, _ = ro.pages_fit(refs, page, tables, [20, 33, 0, 16, 5])
    children = [[-1] * 6 for _ in range(4)]
    caches, refs, children, lens = ro.cache_fork([cache], refs, [1, 0, 7, 1], tables, [20, 33, 0, 16, 5], children, [-3] * 4)
    held = [p for t in tables + children for p in t if p >= 0]
    assert all(refs[p] == held.count(p) for p in range(30)) and lens == [33, 20, -3, 33]
    for s, parent in ((0, 1), (1, 0), (3, 1)):
        for j in range(lens[s]):
            assert np.array_equal(caches[0][:, children[s][j // page], :, j % page], cache[:, tables[parent][j // page], :, j % page])

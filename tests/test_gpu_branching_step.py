"""Drafted tokens, kept ones, fitted tables and forks together, as a rollout uses them; and drafted trees at the sizes where the work is split otherwise."""
import pytest
import torch

from oracle import rollout_oracle as ro
from paper_2511_18871_amd import binding as B
from tests.branching import dev32, mask_words, random_trees
from tests.rollout import check, decode_bounds, numpy64
from tests.test_gpu_tree import make, run_and_check

pytestmark = pytest.mark.gpu
BASE = 10000.0


class Rollout:
    """Sequences in groups that share a prompt, over a paged cache of several layers whose pages are counted."""

    def __init__(self, dtype, d, hq, hkv, page, prompts, members, n_layers=2, pages=200, width=24, seed=3):
        self.gen = torch.Generator().manual_seed(seed)
        self.dtype, self.d, self.hq, self.hkv, self.page, self.prompts, self.n = dtype, d, hq, hkv, page, prompts, len(prompts) * members
        self.Gs, self.scale = [members] * len(prompts), d ** -0.5
        self.k, self.v = (torch.zeros(n_layers, pages, hkv, page, d, dtype=dtype, device="cuda") for _ in range(2))
        self.layers = [B.KvCache(self.k[i], self.v[i]) for i in range(n_layers)]
        self.all = B.KvLayers(self.k, self.v)
        self.refs, self.lens = dev32([0] * pages), dev32([0] * self.n)
        self.tables, self.other = dev32([[-1] * width] * self.n), dev32([[-1] * width] * self.n)
        self.pt, self.pl = dev32([[-1] * width] * len(prompts)), dev32(prompts)
        self.base = dev32([prompts[s // members] for s in range(self.n)])
        B.sp_attn_pages_fit(self.refs, page, self.pt, self.pl)
        for layer in self.layers:
            self.append(layer, self.tokens(sum(prompts)), self.pt, dev32([0] * len(prompts)), prompts, None)

    def tokens(self, n):
        return [torch.randn(n, h, self.d, generator=self.gen).to(self.dtype).cuda() for h in (self.hkv, self.hkv, self.hq)]

    def append(self, layer, kvq, tables, lens, new, pos_base):
        k, v, q = kvq
        return B.sp_attn_cache_append(layer, k, v, tables, lens, BASE, q=q, new_lens=new, pos_base=pos_base)[0]

    def step(self, drafts, index, depth, mask, kept, n_kept, parents):
        """One step: places, drafted tokens, their attention, the kept ones, what is left over given back, and the sequences that go on."""
        S, n = self.n, index.shape[0] // self.n
        out = [B.sp_attn_pages_fit(self.refs, self.page, self.tables, self.lens + n)]
        seq = torch.arange(S, device="cuda").repeat_interleave(n)
        grown = self.lens + n
        for layer, kvq in zip(self.layers, drafts):
            q = self.append(layer, kvq, self.tables[seq], self.lens[seq] + index, None, self.base[seq] + depth - index)
            out += [q, *B.sp_attn_tree_decode(layer, q, self.Gs, [n] * S, mask, self.pt, self.pl, self.tables, grown, self.scale)]
        self.lens.copy_(B.sp_attn_cache_keep(self.all, self.tables, self.lens, kept, n_kept))
        out.append(B.sp_attn_pages_fit(self.refs, self.page, self.tables, self.lens))
        out.append(B.sp_attn_cache_fork(self.all, self.refs, parents, self.tables, self.lens, self.other))
        out.append(B.sp_attn_pages_fit(self.refs, self.page, self.tables, torch.zeros_like(self.lens)))
        self.tables.copy_(self.other)
        self.other.fill_(-1)
        self.lens.copy_(out[-2])
        return out


def drafted(r, n, rng_seed):
    """A step's random trees of n tokens per sequence: (tokens of each layer, their numbers, depths, masks as lists and words, kept paths, their lengths, parents)."""
    gen = torch.Generator().manual_seed(rng_seed)
    rows = random_trees(gen, [n] * r.n)
    paths = [rows[s * n + int(torch.randint(0, n, (1,), generator=gen))] for s in range(r.n)]
    if rng_seed % 2:
        paths[0] = []
    members = r.Gs[0]
    parents = [s // members * members + int(torch.randint(0, members, (1,), generator=gen)) for s in range(r.n)]
    return ([r.tokens(r.n * n) for _ in r.layers], list(range(n)) * r.n, [len(x) - 1 for x in rows], rows, paths, parents)


@pytest.mark.parametrize("dtype,d,hq,hkv,page", [(torch.bfloat16, 128, 8, 2, 16), (torch.bfloat16, 64, 4, 4, 32), (torch.float32, 64, 6, 2, 16)])
def test_a_rollout_that_branches(dtype, d, hq, hkv, page):
    """Against the oracle's attention, and a second cache to which the kept tokens are appended one by one."""
    n = 6
    r = Rollout(dtype, d, hq, hkv, page, [37, 0, 16], 3)
    # what each sequence holds, as the numbers of its appended tokens, and those tokens as a cache without drafts has them
    plain = [Rollout(dtype, d, hq, hkv, page, [0], 1, pages=24) for _ in range(r.n)]
    for i in range(5):
        kvq, index, depth, rows, paths, parents = drafted(r, n, i)
        before = r.lens.tolist()
        mask = mask_words(rows, 1).cuda()
        tables_before_keep = []
        kept = dev32([p + [0] * (n - len(p)) for p in paths])
        # the oracle sees the cache as the drafted tokens leave it: recorded by a copy between the calls
        seen = []
        inner = B.sp_attn_cache_keep
        def keep(*a, **k):
            tables_before_keep.append(r.tables.tolist())
            seen.append([(numpy64(r.k[x]), numpy64(r.v[x])) for x in range(len(r.layers))])
            return inner(*a, **k)
        B.sp_attn_cache_keep = keep
        try:
            out = r.step(kvq, dev32(index), dev32(depth), mask, kept, dev32([len(p) for p in paths]), dev32(parents))
        finally:
            B.sp_attn_cache_keep = inner
        torch.cuda.synchronize()
        assert out[0].item() == 0
        for x in range(len(r.layers)):
            q, o, lse = out[1 + 3 * x:4 + 3 * x]
            ref, rlse, weight, reach, count = ro.tree_decode(*seen[0][x], numpy64(q), r.Gs, [n] * r.n, rows, r.pt.tolist(), r.prompts, tables_before_keep[0],
                                                             [b + n for b in before], r.scale)
            tol_o, tol_lse = decode_bounds(ref, rlse, weight, reach, count, d, dtype)
            check("lse", lse, rlse, tol_lse)
            check("o", o, ref, tol_o)
        # the plain caches
        for s, p in enumerate(plain):
            have = before[s]
            lens = dev32([have + len(paths[s])])
            B.sp_attn_pages_fit(p.refs, page, p.tables, lens)
            for j, node in enumerate(paths[s]):
                for x, layer in enumerate(p.layers):
                    at = slice(s * n + node, s * n + node + 1)
                    p.append(layer, [t[at] for t in kvq[x]], p.tables, dev32([have + j]), None, r.base[s:s + 1].contiguous())
            p.lens = lens
        copies = [(p.k.clone(), p.v.clone(), p.tables.clone(), p.refs.clone(), p.lens) for p in plain]
        for s, p in enumerate(plain):
            p.k[:], p.v[:], p.tables, p.refs, p.lens = (*copies[parents[s]][:2], *(t.clone() for t in copies[parents[s]][2:]))
        # the same tokens in every layer, and every page counted as often as tables hold it
        held = [0] * r.refs.shape[0]
        for table in r.tables.tolist() + r.pt.tolist():
            for x in table:
                if x >= 0:
                    held[x] += 1
        assert r.refs.tolist() == held and torch.all(r.other == -1)
        for s, p in enumerate(plain):
            length = p.lens.item()
            assert r.lens[s].item() == length
            j = torch.arange(length, device="cuda")
            for mine, want in ((r.k, p.k), (r.v, p.v)):
                got = mine[:, r.tables[s, j // page].long(), :, j % page]
                assert torch.equal(got, want[:, p.tables[0, j // page].long(), :, j % page])
            assert (r.tables[s] >= 0).sum().item() == -(-length // page)


def test_a_step_in_a_graph():
    """Captured once, replayed with other drafts, with eager steps of a second rollout between the replays."""
    n = 5
    make_one = lambda: Rollout(torch.bfloat16, 128, 8, 2, 16, [20, 33], 4, seed=9)
    eager, graphed = make_one(), make_one()
    def inputs(r, i):
        kvq, index, depth, rows, paths, parents = drafted(r, n, i)
        return kvq, [dev32(index), dev32(depth), mask_words(rows, 1).cuda(), dev32([p + [0] * (n - len(p)) for p in paths]), dev32([len(p) for p in paths]), dev32(parents)]
    kvq, args = inputs(graphed, 100)
    inputs(eager, 100)                                                  # (both draw the same tokens from here on)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = graphed.step(kvq, *args)
    for i in range(5):
        more, other = inputs(graphed, i)
        for a, b in zip(args + [t for x in kvq for t in x], other + [t for x in more for t in x]):
            a.copy_(b)
        more, other = inputs(eager, i)
        want = eager.step(more, *other)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        for name in ("k", "v", "refs", "tables", "lens"):
            assert torch.equal(getattr(eager, name), getattr(graphed, name)), name


# groups, their sequences, prompts, tokens ahead, drafted tokens, heads
SPLITS = [
    ("chain behind a long response, workgroups of eight waves", [1], [0], [3900], [256], 8, 2),
    ("long lists of many rows, prompt ahead of each response", [4, 4], [700, 650], [200, 1, 0, 90, 130, 17, 31, 64], [40] * 8, 32, 8),
    ("the same with groups of other sizes: prompts by themselves", [5, 3], [700, 650], [200, 1, 0, 90, 130, 17, 31, 64], [40] * 8, 32, 8),
    ("a long prompt that many sequences share", [24], [4000], [(31 * i) % 70 for i in range(24)], [1 + i % 4 for i in range(24)], 28, 4),
    ("short prompts of many sequences", [16] * 6, [64 + 21 * i for i in range(6)], [(7 * i) % 40 for i in range(96)], [3] * 96, 28, 4),
    ("groups of one", [1] * 20, [(97 * i) % 600 for i in range(20)], [(13 * i) % 90 for i in range(20)], [9] * 20, 16, 4),
    ("one long prompt and one none", [2, 2], [5000, 0], [3, 700, 600, 0], [30, 64, 1, 20], 16, 8),
]


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.bfloat16, 64), (torch.float32, 64)])
@pytest.mark.parametrize("case", SPLITS, ids=lambda c: c[0].replace(" ", "_"))
def test_every_split_of_the_work(dtype, d, case):
    _, Gs, prompts, ahead, new, hq, hkv = case
    if d == 64:                                                         # half the rows, and pages of another size
        new = [(n + 1) // 2 for n in new]
    resp = [a + n for a, n in zip(ahead, new)]
    *x, rows, mask = make(dtype, d, hq, hkv, 64 if d == 64 else 16, prompts, new, resp, seed=d)
    run_and_check(*x, rows, mask, Gs, new, prompts, resp, d ** -0.5)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("n,ahead,prompt", [(200, 2900, 100), (300, 2500, 0), (40, 60, 300)])
def test_values_that_are_not_finite_in_long_lists(bad, n, ahead, prompt):
    """A drafted token's value reaches the rows that see it, in its element and heads, and no other."""
    prompts, new, resp = [prompt], [n], [ahead + n]
    q, kc, vc, pt, rt, rows, _ = make(torch.bfloat16, 128, 16, 4, 16, prompts, new, resp)
    rows = [sorted(set([0, i] + ([5] if i % 3 else []))) for i in range(n)]
    mask = mask_words(rows, -(-n // 32)).cuda()
    def call(v):
        return B.sp_attn_tree_decode(B.KvCache(kc.cuda(), v.cuda()), q.cuda(), [1], new, mask, pt.cuda(), dev32(prompts), rt.cuda(), dev32(resp), 0.1)
    clean, clean_lse = call(vc)
    v2, j = vc.clone(), ahead + 5
    v2[rt[0, j // 16], 2, j % 16, 77] = bad
    o, lse = call(v2)
    changed = torch.zeros(n, 16, 128, dtype=torch.bool)
    for t in range(n):
        changed[t, 8:12, 77] = 5 in rows[t]
    assert torch.equal(lse, clean_lse) and torch.equal(o.cpu()[~changed], clean.cpu()[~changed])
    hit = o.cpu()[changed]
    assert torch.all(hit.isnan()) if bad != bad else torch.all(hit == bad)


def test_two_calls_at_once():
    """Two streams, each with its own workspace, over the same cache; and one stream after the other with one workspace."""
    prompts, Gs, new, resp = [700, 90], [4, 4], [16] * 8, [90, 40, 16, 300, 200, 31, 64, 77]
    q, kc, vc, pt, rt, _, mask = make(torch.bfloat16, 128, 28, 4, 16, prompts, new, resp)
    cache, q, pt, rt, mask, pl, rl = B.KvCache(kc.cuda(), vc.cuda()), q.cuda(), pt.cuda(), rt.cuda(), mask.cuda(), dev32(prompts), dev32(resp)
    args = (Gs, new, mask, pt, pl, rt, rl, 0.1)
    want = [B.sp_attn_tree_decode(cache, x, *args) for x in (q, -q)]
    size = B.tree_decode_workspace_bytes(2, 8, q.shape[0], 28, 4, 128, B.SP_BF16)
    rooms = [torch.empty(size, dtype=torch.uint8, device="cuda") for _ in range(2)]
    outs = [(torch.empty_like(q), torch.empty_like(want[0][1])) for _ in range(2)]
    inputs, streams = (q, -q), [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for x, (o, lse), room, s in zip(inputs, outs, rooms, streams):
            B.sp_attn_tree_decode(cache, x, *args, o=o, lse=lse, workspace=room, stream=s)
    torch.cuda.synchronize()
    for (o, lse), (wo, wl) in zip(outs, want):
        assert torch.equal(o, wo) and torch.equal(lse, wl)
    for x, (wo, wl) in list(zip(inputs, want)) * 3:
        o, lse = B.sp_attn_tree_decode(cache, x, *args, workspace=rooms[0])
        assert torch.equal(o, wo) and torch.equal(lse, wl)


@pytest.mark.parametrize("d", [128, 64])
def test_rows_without_a_key_in_long_lists(d):
    """Many rows to a workgroup, some of which see nothing, one key, or the last one only."""
    new, resp = [1024, 40], [1024, 70]
    q, kc, vc, _, rt, _, _ = make(torch.bfloat16, d, 8, 1, 32, [0], new, resp, words=32)
    rows = [[] if i % 5 == 0 else [1023] if i % 5 == 1 else [i] if i % 5 == 2 else list(range(i % 7, 1024, 61)) for i in range(1024)] + [[] for _ in range(40)]
    o, lse = run_and_check(q, kc, vc, None, rt, rows, mask_words(rows, 32), None, new, None, resp, d ** -0.5)
    assert torch.all(o[:1024:5] == 0) and torch.all(torch.isneginf(lse[:, :1024:5])) and torch.isfinite(lse[:, 1024:]).all()


def test_long_tables_of_short_sequences():
    """The work is split by what tables hold; here lengths are far below that, or negative, or beyond."""
    Gs, prompts, new = [4, 4], [1500, 1500], [40] * 8
    q, kc, vc, pt, rt, rows, mask = make(torch.bfloat16, 128, 32, 8, 16, prompts, new, [900] * 8)
    for prompt_lens, resp in (([3, 0], [40, 41, 39, -1, 77, 0, 900, 1000]), ([-5, 1500], [-1] * 8), ([1500, 17], [1, 2, 900, 40, -7, 64, 65, 300])):
        run_and_check(q, kc, vc, pt, rt, rows, mask, Gs, new, prompt_lens, resp, 0.1)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_long_lists_do_not_see_what_is_masked(bad):
    """Neither key nor value of a drafted token matters to the rows that do not see it, in workgroups of four waves and of eight."""
    for n, ahead in ((200, 1500), (300, 3900)):
        new, resp = [n, n], [ahead + n, ahead]
        q, kc, vc, _, rt, _, _ = make(torch.bfloat16, 128, 16, 4, 16, [0], new, resp)
        rows = [sorted({0, i, i // 2} - {2, n - 1}) for i in range(n)] * 2
        args = (q.cuda(), None, new, mask_words(rows, -(-n // 32)).cuda(), None, None, rt.cuda(), dev32(resp), 0.1)
        clean, clean_lse = B.sp_attn_tree_decode(B.KvCache(kc.cuda(), vc.cuda()), *args)
        for s in range(2):
            for j in (resp[s] - n + 2, resp[s] - 1):
                kc[rt[s, j // 16], :, j % 16] = bad
                vc[rt[s, j // 16], :, j % 16] = bad
        o, lse = B.sp_attn_tree_decode(B.KvCache(kc.cuda(), vc.cuda()), *args)
        assert torch.equal(o, clean) and torch.equal(lse, clean_lse) and torch.isfinite(lse).all()


@pytest.mark.parametrize("n,ahead,prompt", [(200, 2900, 100), (300, 3900, 0)])
def test_large_scores_in_long_lists(n, ahead, prompt):
    """Scores far apart and far from 0, which rise along the list: rows take new references again and again."""
    prompts, new, resp = [prompt], [n], [ahead + n]
    q, kc, vc, pt, rt, rows, mask = make(torch.bfloat16, 128, 8, 2, 16, prompts, new, resp)
    q, kc = q.abs(), kc * 8
    for j in range(0, ahead, 50):
        kc[rt[0, j // 16], :, j % 16] = kc[rt[0, j // 16], :, j % 16].abs() * (j / ahead)
    run_and_check(q, kc, vc, pt, rt, rows, mask, [1], new, prompts, resp, 1.0)


@pytest.mark.parametrize("where", ["prompt", "ahead"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_keys_and_values_that_all_rows_of_long_lists_see(where, bad):
    """A value's element reaches its heads' rows in its place, a NaN key makes their rows NaN."""
    n, ahead, prompt = 200, 2900, 100
    q, kc, vc, pt, rt, _, _ = make(torch.bfloat16, 128, 16, 4, 16, [prompt], [n], [ahead + n])
    page, at = (pt[0, 2], 7) if where == "prompt" else (rt[0, 100], 3)
    def call(k, v):
        return B.sp_attn_tree_decode(B.KvCache(k.cuda(), v.cuda()), q.cuda(), [1], [n], None, pt.cuda(), dev32([prompt]), rt.cuda(), dev32([ahead + n]), 0.1)
    clean, clean_lse = call(kc, vc)
    v2 = vc.clone()
    v2[page, 1, at, 9] = bad
    o, lse = call(kc, v2)
    hit = o[:, 4:8, 9]
    assert torch.equal(lse, clean_lse) and (torch.all(hit.isnan()) if bad != bad else torch.all(hit == bad))
    o[:, 4:8, 9] = clean[:, 4:8, 9]
    assert torch.equal(o, clean)
    if bad != bad:
        k2 = kc.clone()
        k2[page, 1, at, 9] = bad
        o, lse = call(k2, vc)
        assert torch.all(o[:, 4:8].isnan()) and torch.all(lse[4:8].isnan())
        assert torch.equal(o[:, :4], clean[:, :4]) and torch.equal(o[:, 8:], clean[:, 8:]) and torch.equal(lse[:4], clean_lse[:4])


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("case", SPLITS, ids=lambda c: c[0].replace(" ", "_"))
def test_in_place_at_every_split(d, case):
    """o may be q: rows that one worker finishes by itself among them."""
    _, Gs, prompts, ahead, new, hq, hkv = case
    resp = [a + n for a, n in zip(ahead, new)]
    q, kc, vc, pt, rt, _, mask = make(torch.bfloat16, d, hq, hkv, 16, prompts, new, resp, seed=d)
    cache, q = B.KvCache(kc.cuda(), vc.cuda()), q.cuda()
    args = (Gs, new, mask.cuda(), pt.cuda(), dev32(prompts), rt.cuda(), dev32(resp), d ** -0.5)
    want, want_lse = B.sp_attn_tree_decode(cache, q, *args)
    for _ in range(3):
        mine = q.clone()
        o, lse = B.sp_attn_tree_decode(cache, mine, *args, o=mine)
        assert torch.equal(o, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("Gs,n,table", [([1] * 70, 32, 640), ([2, 1] * 25, 32, 700), ([33, 33], 64, 2304), ([1] * 66, 64, 2304), ([3] * 30, 40, 1100)])
@pytest.mark.parametrize("d", [128, 64])
def test_many_lists_of_many_rows(Gs, n, table, d):
    """More lists than lanes, each of many rows, in workgroups of four waves and of eight; most of the sequences are far shorter than their tables."""
    gen = torch.Generator().manual_seed(table + d)
    S, G = sum(Gs), len(Gs)
    new = [n] * S if Gs[0] != 2 else [n - s % 3 for s in range(S)]
    held = [n + (table - n if s % 12 == 5 else int(torch.randint(0, 90, (1,), generator=gen))) for s in range(S)]
    prompts = [table if g % 20 == 3 else int(torch.randint(0, 70, (1,), generator=gen)) for g in range(G)]
    q, kc, vc, pt, rt, rows, mask = make(torch.bfloat16, d, 8, 2, 64, prompts, new, held)
    resp = [-1 if s % 17 == 9 else x for s, x in enumerate(held)]
    run_and_check(q, kc, vc, pt, rt, rows, mask, Gs, new, prompts, resp, d ** -0.5)


@pytest.mark.parametrize("new", [300, 120])
def test_long_lists_beyond_32_bit_offsets(new):
    """Pages far behind the first 4 GB of a cache, in lists of many rows."""
    d, hkv, page, n_pages = 128, 8, 256, 10000
    kc, vc = (torch.empty(n_pages, hkv, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    gen = torch.Generator().manual_seed(3)
    used = [9999, 3, 8700, 9000, 9998, 5001, 8193, 7777, 9001, 42]
    small_k, small_v = (torch.randn(10, hkv, page, d, generator=gen).bfloat16().cuda() for _ in range(2))
    kc[used], vc[used] = small_k, small_v
    q = torch.randn(new, 16, d, generator=gen).bfloat16().cuda()
    near = B.KvCache(small_k, small_v)
    for prompt, resp in ((used[:2], used[2:]), (used[:1], used[1:])):
        at = [used.index(p) for p in resp]
        lens = dev32([256 * len(prompt) - 3]), dev32([256 * len(resp) - 9])
        far = B.sp_attn_tree_decode(B.KvCache(kc, vc), q, [1], [new], None, dev32([prompt]), lens[0], dev32([resp]), lens[1], 0.1)
        want = B.sp_attn_tree_decode(near, q, [1], [new], None, dev32([list(range(len(prompt)))]), lens[0], dev32([at]), lens[1], 0.1)
        assert torch.equal(far[0], want[0]) and torch.equal(far[1], want[1]) and torch.isfinite(far[1]).all()

"""Measured cases of the operators of branching rollouts: attention of drafted tokens that form trees over the paged
cache, keeping the accepted ones, forking sequences, and fitting tables of pages to their sequences' lengths.

``listed()`` names the cases, ``draw(rng)`` makes one more of the same ranges, ``prepare`` makes a case's inputs
from a seed, ``run`` is one pass, ``work`` the bytes and operations that a pass cannot do without and ``exact``
the results in 64 bits.  ``own`` chooses between the operators in elementary torch operations and this
repository's entry points."""
import math

import torch

own = False

DEVICE = "cuda" if torch.cuda.is_available() else "cpu"
HEADS = ((28, 4), (32, 8), (40, 8))
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- the cases ---------------------------------------------------------------------------------------------

def _stream(seed):
    """Endless 32-bit numbers."""
    state = seed * 2654435761 % 2 ** 32 or 1
    while True:
        state ^= state << 13 & 0xffffffff
        state ^= state >> 17
        state ^= state << 5 & 0xffffffff
        yield state


def _lens(count, lo, hi, seed):
    """`count` lengths of lo .. hi."""
    numbers = _stream(seed)
    return [lo + next(numbers) % (hi - lo + 1) for _ in range(count)]


def _tree(groups, prompt_lo, prompt_hi, members, resp_lo, resp_hi, new_lo, new_hi, hq, hkv, page=64, dtype="bf16", d=128, chain=False, pack_seed=1):
    return dict(op="tree", groups=groups, prompt_lo=prompt_lo, prompt_hi=prompt_hi, members=members, resp_lo=resp_lo, resp_hi=resp_hi,
                new_lo=new_lo, new_hi=new_hi, hq=hq, hkv=hkv, page=page, dtype=dtype, head_dim=d, chain=chain, pack_seed=pack_seed)


def _keep(layers, seqs, cached_lo, cached_hi, nodes, kept_lo, kept_hi, hkv, page=64, dtype="bf16", d=128, pack_seed=1):
    return dict(op="keep", layers=layers, seqs=seqs, cached_lo=cached_lo, cached_hi=cached_hi, nodes=nodes, kept_lo=kept_lo,
                kept_hi=kept_hi, hkv=hkv, page=page, dtype=dtype, head_dim=d, pack_seed=pack_seed)


def _fork(layers, parents, cached_lo, cached_hi, children, hkv, page=64, dtype="bf16", d=128, pack_seed=1):
    return dict(op="fork", layers=layers, parents=parents, cached_lo=cached_lo, cached_hi=cached_hi, children=children, hkv=hkv, page=page,
                dtype=dtype, head_dim=d, pack_seed=pack_seed)


def _fit(seqs, cached_lo, cached_hi, nodes, page, spare, pack_seed=1):
    return dict(op="fit", seqs=seqs, cached_lo=cached_lo, cached_hi=cached_hi, nodes=nodes, page=page, spare=spare, pack_seed=pack_seed)


def listed():
    named = {
        # a tree of 8 drafted tokens of one sequence without a shared prompt: latency
        "tree_one_sequence": _tree(1, 0, 0, 1, 1000, 1000, 8, 8, 28, 4),
        # one GRPO group of a 7B-class model, trees of 16 at answers of different lengths
        "tree_single_group": _tree(1, 1024, 1024, 8, 1, 256, 16, 16, 28, 4),
        # 32 short answers to a 16K prompt, trees of 8
        "tree_extreme_sharing": _tree(1, 16384, 16384, 32, 64, 256, 8, 8, 40, 8),
        # grade-school maths at 1K context: many groups of a short prompt and 16 answers, 3 to 5 drafted tokens each
        "tree_many_short_answers": _tree(64, 64, 192, 16, 96, 416, 3, 5, 28, 4, page=16),
        # chunks of 192 to 256 tokens that follow 4K to 8K of their own: a chain, no mask
        "chain_chunks": _tree(4, 0, 0, 1, 4000, 8000, 192, 256, 32, 8, page=128, chain=True),
        # the float32 path on a small ragged batch
        "tree_small_f32": _tree(3, 0, 333, 5, 1, 200, 1, 7, 4, 2, page=16, dtype="f32", d=64),
        # accepted tokens of one group's step, in all layers of a small model
        "keep_step": _keep(12, 8, 64, 400, 16, 1, 8, 2, page=64),
        # many sequences with long accepted paths out of trees of 64
        "keep_batch": _keep(16, 128, 1, 200, 64, 8, 40, 4, page=16),
        # two answers continued four times each
        "fork_step": _fork(12, 2, 100, 500, 8, 2, page=64),
        # beams of many groups, pages of 128
        "fork_batch": _fork(8, 16, 64, 900, 128, 8, page=128),
        # a step's turnover of pages: 32 sequences give back what was rejected, finished ones all, and take room for new drafts
        "fit_step": _fit(32, 64, 2048, 16, 64, 100),
        # the same of 1024 sequences on pages of 16
        "fit_batch": _fit(1024, 96, 4000, 64, 16, 5000),
    }
    return [dict(case, name=name) for name, case in named.items()]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _spread(rng, lo, hi):
    """A range of lengths whose upper end is drawn over the logarithm."""
    top = _log_int(rng, lo, hi)
    return max(lo, int(top * rng.uniform(0.2, 1.0))), top


def draw(rng):
    """One more case of the ranges the listed ones stand for."""
    while True:
        op = rng.choice(("tree", "tree", "tree", "keep", "fork", "fit"))
        seed = rng.randint(1, 10 ** 6)
        hq, hkv = rng.choice(HEADS)
        dtype, d = rng.choice((("bf16", 128), ("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 128)))
        page = rng.choice((16, 32, 64, 128, 256))
        if op == "tree":
            prompt = (0, 0) if rng.random() < 0.25 else _spread(rng, 16, 16384)
            resp, new = _spread(rng, 1, 12000), _spread(rng, 1, 256)
            if dtype == "f32":
                hq, hkv = rng.choice(((4, 2), (4, 4), (28, 4)))
            case = _tree(_log_int(rng, 1, 64), *prompt, _log_int(rng, 1, 32), *resp, *new, hq, hkv, page, dtype, d, rng.random() < 0.3, seed)
            longest = prompt[1] + resp[1] + new[1]
            seqs = case["groups"] * case["members"]
            w = work(case)
            fits = (w["bytes"] <= 1e9 and w["flops"] <= (1e11 if dtype == "bf16" else 1e10) and seqs * longest * hkv * d <= 5e8
                    and seqs * new[1] * hq * longest <= 4e8 and seqs * new[1] <= 8000)
        elif op == "keep":
            lo, hi = _spread(rng, 1, 1000)
            nodes = _log_int(rng, 2, 256)
            most = rng.randint(1, nodes)
            case = _keep(_log_int(rng, 1, 32), _log_int(rng, 1, 256), lo, hi, nodes, rng.randint(0, most), most, hkv, page, dtype, d, seed)
            room = case["seqs"] * (-(-(hi + nodes) // page) + 1) * page
            fits = case["layers"] * room * hkv * d <= 1.2e8
        elif op == "fork":
            lo, hi = _spread(rng, 1, 2000)
            parents = _log_int(rng, 1, 64)
            case = _fork(_log_int(rng, 1, 32), parents, lo, hi, min(256, parents * _log_int(rng, 1, 16)), hkv, page, dtype, d, seed)
            room = (parents * (-(-hi // page)) + case["children"] + 4) * page
            fits = case["layers"] * room * hkv * d <= 3e8
        else:
            lo, hi = _spread(rng, 16, 16000)
            case = _fit(_log_int(rng, 1, 1024), lo, hi, _log_int(rng, 1, 256), page, _log_int(rng, 1, 20000), seed)
            fits = case["seqs"] * hi / page <= 4e5
        if fits:
            return case


def _groups(case):
    """(prompt length, [(tokens ahead of the drafted ones, drafted ones) of each sequence]) of each group of a tree case."""
    n, k = case["groups"], case["members"]
    prompts = _lens(n, case["prompt_lo"], case["prompt_hi"], case["pack_seed"])
    resp = _lens(n * k, case["resp_lo"], case["resp_hi"], case["pack_seed"] + 77)
    new = _lens(n * k, case["new_lo"], case["new_hi"], case["pack_seed"] + 154)
    own_tokens = list(zip(resp, new))
    return [(p, own_tokens[g * k:(g + 1) * k]) for g, p in enumerate(prompts)]


def _ancestor_sets(case):
    """For each sequence and each of its drafted tokens, an integer whose bit m says whether it sees the drafted token m: its own
    bit and those on the way to the root.  The parent of a token is one of the four ahead of it, as in a narrow tree."""
    numbers = _stream(case["pack_seed"] + 231)
    found = []
    for _, members in _groups(case):
        for _, n in members:
            sets = []
            for i in range(n):
                parent = i - 1 if case["chain"] or i < 2 else i - 1 - next(numbers) % min(4, i)
                sets.append((sets[parent] if i else 0) | 1 << i)
            found.append(sets)
    return found


def _cached(case):
    return _lens(case["seqs" if "seqs" in case else "parents"], case["cached_lo"], case["cached_hi"], case["pack_seed"])


def _pages(tokens, page):
    return -(-tokens // page)


def work(case):
    """Bytes and operations that one pass cannot do without: every input read once, every output written once."""
    e = 2 if case.get("dtype") == "bf16" else 4
    if case["op"] == "tree":
        groups, d = _groups(case), case["head_dim"]
        keys = sum(p + sum(r + n for r, n in own_tokens) for p, own_tokens in groups)
        tokens = sum(n for _, own_tokens in groups for _, n in own_tokens)
        pairs = sum((p + r) * n for p, own_tokens in groups for r, n in own_tokens) + sum(bin(x).count("1") for sets in _ancestor_sets(case) for x in sets)
        mask = 0 if case["chain"] else 4 * tokens * -(-case["new_hi"] // 32)
        return {"bytes": keys * case["hkv"] * d * 2 * e + tokens * case["hq"] * (2 * d * e + 4) + mask, "flops": 4 * d * case["hq"] * pairs}
    if case["op"] == "keep":
        kept = _lens(case["seqs"], case["kept_lo"], case["kept_hi"], case["pack_seed"] + 77)
        row = 2 * case["layers"] * case["hkv"] * case["head_dim"] * e                  # keys and values of a token
        return {"bytes": 2 * sum(kept) * row + 4 * (sum(kept) + 3 * case["seqs"]), "flops": 0}
    if case["op"] == "fork":
        cached = _cached(case)
        row = 2 * case["layers"] * case["hkv"] * case["head_dim"] * e
        of_child = [cached[s % len(cached)] for s in range(case["children"])]
        tables = sum(_pages(n, case["page"]) for n in of_child) * 2 * 4
        return {"bytes": sum(n % case["page"] for n in of_child) * 2 * row + tables + 12 * case["children"], "flops": 0}
    held = sum(_pages(n + case["nodes"], case["page"]) for n in _cached(case))
    return {"bytes": 2 * 4 * (held + case["seqs"]) + 4 * (held + case["spare"]), "flops": 0}


# ---- inputs ------------------------------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device=DEVICE).manual_seed(seed)


def _randn(gen, shape, dtype):
    return torch.randn(shape, generator=gen, device=DEVICE).to(dtype)


def _int32(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def _tables(gen, lens, page, extra=3, width=None):
    """Page tables [len(lens), width] with pages in a random order, -1 behind each sequence's last; how many there are."""
    need = [_pages(n, page) for n in lens]
    order = torch.randperm(sum(need) + extra, generator=gen, device=DEVICE).to(torch.int32)
    width = width or max(1, max(need))
    at = torch.arange(width, device=DEVICE)
    count = torch.tensor(need, device=DEVICE)
    first = torch.cumsum(count, 0) - count
    inside = at[None, :] < count[:, None]
    table = torch.where(inside, order[(first[:, None] + at[None, :]).clamp(max=len(order) - 1)], -1)
    return table.to(torch.int32).contiguous(), len(order)


def _references(tables, pages):
    """How many tables hold each page."""
    held = tables[tables >= 0].long()
    return torch.zeros(pages, dtype=torch.int32, device=DEVICE).scatter_add_(0, held, torch.ones_like(held, dtype=torch.int32))


def prepare(case, seed):
    gen = _generator(seed)
    state = {"case": case}
    if case["op"] == "tree":
        dtype, groups = DTYPES[case["dtype"]], _groups(case)
        hq, hkv, d, page = case["hq"], case["hkv"], case["head_dim"], case["page"]
        prompts, own_tokens = [p for p, _ in groups], [x for _, r in groups for x in r]
        new = [n for _, n in own_tokens]
        lens = [r + n for r, n in own_tokens]
        tables, pages = _tables(gen, prompts + lens, page)
        words = -(-case["new_hi"] // 32)
        sets = [x >> 32 * w & 0xffffffff for of_seq in _ancestor_sets(case) for x in of_seq for w in range(words)]
        ancestors = torch.tensor(sets, dtype=torch.int64, device=DEVICE).view(-1, words).to(torch.int32)
        state.update(
            q=_randn(gen, (sum(new), hq, d), dtype), Gs=[len(r) for _, r in groups], new_lens=new, ancestors=None if case["chain"] else ancestors,
            prompt_tables=tables[:len(prompts)].contiguous(), resp_tables=tables[len(prompts):].contiguous(),
            prompt_lens=_int32(prompts), resp_lens=_int32(lens), scale=1.0 / math.sqrt(d),
            k_cache=_randn(gen, (pages, hkv, page, d), dtype), v_cache=_randn(gen, (pages, hkv, page, d), dtype))
        # some keys stand out, as in trained models
        loud = torch.rand((pages, hkv, page, 1), generator=gen, device=DEVICE) < 0.01
        state["k_cache"].mul_(torch.where(loud, 4.0, 1.0).to(dtype))
    elif case["op"] == "keep":
        cached, nodes, page = _cached(case), case["nodes"], case["page"]
        kept = _lens(case["seqs"], case["kept_lo"], case["kept_hi"], case["pack_seed"] + 77)
        tables, pages = _tables(gen, [n + nodes for n in cached], page)
        # accepted tokens: a random path through the drafted ones
        order = torch.rand((case["seqs"], nodes), generator=gen, device=DEVICE).argsort(dim=1)
        n_kept = _int32(kept)
        inside = torch.arange(nodes, device=DEVICE)[None, :] < n_kept[:, None]
        path = torch.where(inside, order, nodes).sort(dim=1).values.to(torch.int32)
        _caches(state, gen, case, pages)
        state.update(tables=tables, lens=_int32(cached), kept=path, n_kept=n_kept)
    elif case["op"] == "fork":
        cached, page, children = _cached(case), case["page"], case["children"]
        tables, pages = _tables(gen, cached, page, children + 3)
        _caches(state, gen, case, pages)
        state.update(src_tables=tables, src_lens=_int32(cached), refs=_references(tables, pages),
                     parents=_int32([s % len(cached) for s in range(children)]),
                     tables=torch.full((children, tables.shape[1] + 2), -1, dtype=torch.int32, device=DEVICE),
                     nothing=torch.zeros(children, dtype=torch.int32, device=DEVICE))
    else:
        cached, page, n = _cached(case), case["page"], case["seqs"]
        most = [c + case["nodes"] for c in cached]
        # one sequence in eight has ended; another takes its place
        ended = (torch.rand(n, generator=gen, device=DEVICE) < 0.125).to(torch.int32)
        accepted = torch.randint(1, case["nodes"] + 1, (n,), generator=gen, device=DEVICE).to(torch.int32)
        fresh = torch.randint(case["cached_lo"], case["cached_hi"] + 1, (n,), generator=gen, device=DEVICE).to(torch.int32)
        lens = _int32(cached) + accepted
        width = _pages(case["cached_hi"] + 2 * case["nodes"], page)
        tables, pages = _tables(gen, most, page, case["spare"], width)
        state.update(tables=tables, refs=_references(tables, pages), after=lens * (1 - ended),
                     next=torch.where(ended > 0, fresh, lens) + case["nodes"])
    if own and "k_cache" in state:
        from paper_2511_18871_amd import binding as B
        state["cache"] = (B.KvCache if state["k_cache"].dim() == 4 else B.KvLayers)(state["k_cache"], state["v_cache"])
    return state


def _caches(state, gen, case, pages):
    """The caches of all layers."""
    shape = (case["layers"], pages, case["hkv"], case["page"], case["head_dim"])
    for name in ("k_cache", "v_cache"):
        cache = torch.empty(shape, dtype=DTYPES[case["dtype"]], device=DEVICE)
        for layer in cache:
            layer.copy_(torch.randn(shape[1:], generator=gen, device=DEVICE))
        state[name] = cache


# ---- one pass ----------------------------------------------------------------------------------------------

def run(state):
    op = state["case"]["op"]
    if own:
        return {"tree": _own_tree, "keep": _own_keep, "fork": _own_fork, "fit": _own_fit}[op](state)
    return {"tree": _plain_tree, "keep": _plain_keep, "fork": _plain_fork, "fit": _plain_fit}[op](state)


def _own_tree(s):
    from paper_2511_18871_amd import binding as B
    return B.sp_attn_tree_decode(s["cache"], s["q"], s["Gs"], s["new_lens"], s["ancestors"], s["prompt_tables"], s["prompt_lens"],
                                 s["resp_tables"], s["resp_lens"], s["scale"])


def _own_keep(s):
    from paper_2511_18871_amd import binding as B
    lens = B.sp_attn_cache_keep(s["cache"], s["tables"], s["lens"], s["kept"], s["n_kept"])
    return s["k_cache"], s["v_cache"], lens


def _own_fork(s):
    from paper_2511_18871_amd import binding as B
    # what the last fork took goes back first
    B.sp_attn_pages_fit(s["refs"], s["case"]["page"], s["tables"], s["nothing"])
    lens = B.sp_attn_cache_fork(s["cache"], s["refs"], s["parents"], s["src_tables"], s["src_lens"], s["tables"])
    return s["k_cache"], s["v_cache"], s["tables"], lens, s["refs"]


def _own_fit(s):
    from paper_2511_18871_amd import binding as B
    B.sp_attn_pages_fit(s["refs"], s["case"]["page"], s["tables"], s["after"])
    missing = B.sp_attn_pages_fit(s["refs"], s["case"]["page"], s["tables"], s["next"])
    return s["tables"], s["refs"], missing


def _plain_tree(s):
    page, hkv = s["case"]["page"], s["case"]["hkv"]
    new = torch.tensor(s["new_lens"], device=DEVICE)
    most, total = max(s["new_lens"]), s["q"].shape[0]
    first = torch.cumsum(new, 0) - new
    node = torch.arange(most, device=DEVICE)
    there = node[None, :] < new[:, None]                                        # [sequences, drafted]
    token = (first[:, None] + node[None, :]).clamp(max=total - 1)
    group = torch.repeat_interleave(torch.arange(len(s["Gs"]), device=DEVICE), torch.tensor(s["Gs"], device=DEVICE))
    j_prompt = torch.arange(s["prompt_tables"].shape[1] * page, device=DEVICE)
    j_resp = torch.arange(s["resp_tables"].shape[1] * page, device=DEVICE)
    in_prompt, in_resp = j_prompt[None, :] < s["prompt_lens"][group][:, None], j_resp[None, :] < s["resp_lens"][:, None]
    m = j_resp[None, :] - (s["resp_lens"][:, None] - new[:, None])              # drafted token of each key; negative: one ahead of them
    if s["ancestors"] is None:
        sees = m[:, None, :] <= node[None, :, None]
    else:
        word = (m // 32).clamp(0, s["ancestors"].shape[1] - 1)
        rows = s["ancestors"][token]                                            # [sequences, drafted, words]
        bits = torch.gather(rows, 2, word[:, None, :].expand(-1, most, -1))
        sees = (m < 0)[:, None, :] | ((bits >> (m % 32)[:, None, :]) & 1 == 1)
    sees = torch.cat((in_prompt[:, None, :].expand(-1, most, -1), sees & in_resp[:, None, :]), dim=2)
    pages = torch.cat((s["prompt_tables"][group][:, j_prompt // page], s["resp_tables"][:, j_resp // page]), dim=1)
    at, row = pages.clamp(min=0).long(), torch.cat((j_prompt, j_resp)) % page
    hidden = ~torch.cat((in_prompt, in_resp), dim=1)[:, None, :, None]
    k = s["k_cache"][at, :, row[None, :]].permute(0, 2, 1, 3).float()           # [sequences, kv heads, keys, d]
    q = s["q"][token].float().unflatten(2, (hkv, -1)).permute(0, 2, 1, 3, 4)    # [sequences, kv heads, drafted, heads of each, d]
    rep = q.shape[3]
    score = torch.matmul(q.flatten(2, 3), k.transpose(2, 3)) * s["scale"]
    del k
    score = score.unflatten(2, (most, rep)).masked_fill(~sees[:, None, :, None, :], -math.inf)
    top = score.amax(dim=4, keepdim=True)
    p = torch.exp(score - torch.where(torch.isinf(top), 0.0, top))
    del score
    sum_p = p.sum(dim=4, keepdim=True)
    v = s["v_cache"][at, :, row[None, :]].permute(0, 2, 1, 3).float().masked_fill(hidden, 0.0)
    o = torch.matmul(p.flatten(2, 3), v).unflatten(2, (most, rep)) / torch.where(sum_p > 0, sum_p, 1.0)
    lse = (top + torch.log(sum_p))[..., 0].permute(0, 2, 1, 3).flatten(2, 3)    # [sequences, drafted, heads]
    o = o.permute(0, 2, 1, 3, 4).flatten(2, 3).to(s["q"].dtype)
    # back to tokens; what has no place goes to a row behind the last
    to = torch.where(there, token, total).flatten()
    out, out_lse = torch.empty((total + 1, *o.shape[2:]), dtype=o.dtype, device=DEVICE), torch.empty((total + 1, lse.shape[2]), device=DEVICE)
    out[to], out_lse[to] = o.flatten(0, 1), lse.flatten(0, 1)
    return out[:total], out_lse[:total].t().contiguous()


def _plain_keep(s):
    page = s["case"]["page"]
    i = torch.arange(s["kept"].shape[1], device=DEVICE)
    inside = i[None, :] < s["n_kept"][:, None]
    start = s["lens"][:, None].long()
    # tokens that do not move stand for those that have none: they are written over with what they hold
    j_from, j_to = start + torch.where(inside, s["kept"], 0), start + torch.where(inside, i[None, :], 0)
    first = s["kept"][:, :1]
    j_from = torch.where(inside, j_from, start + torch.where(s["n_kept"][:, None] > 0, first, 0))
    at_from, at_to = torch.gather(s["tables"], 1, j_from // page).long(), torch.gather(s["tables"], 1, j_to // page).long()
    for cache in (s["k_cache"], s["v_cache"]):
        cache[:, at_to, :, j_to % page] = cache[:, at_from, :, j_from % page]
    return s["k_cache"], s["v_cache"], s["lens"] + s["n_kept"]


def _count(refs, pages, by):
    refs.scatter_add_(0, pages.long(), torch.full_like(pages, by))


def _fit_plainly(refs, page, tables, lens):
    need = ((lens + page - 1) // page)[:, None]
    col = torch.arange(tables.shape[1], device=DEVICE)[None, :]
    behind = (col >= need) & (tables >= 0)
    _count(refs, tables[behind], -1)
    tables.masked_fill_(behind, -1)
    wants = ((col < need) & (tables < 0)).flatten()
    nth, free = torch.cumsum(wants, 0) - 1, refs == 0
    place = torch.where(free, torch.cumsum(free, 0) - 1, refs.shape[0])         # of each free page among them
    pages = torch.full((refs.shape[0] + 1,), -1, dtype=torch.int32, device=DEVICE)
    pages.scatter_(0, place, torch.arange(refs.shape[0], dtype=torch.int32, device=DEVICE))
    pages[-1] = -1
    got = torch.where(wants & (nth < refs.shape[0]), pages[nth.clamp(0, refs.shape[0])], -1)
    tables.copy_(torch.where(wants, got, tables.flatten()).view_as(tables))
    _count(refs, got[got >= 0], 1)
    return (wants & (got < 0)).sum().to(torch.int32).view(1)


def _plain_fork(s):
    page, tables, refs = s["case"]["page"], s["tables"], s["refs"]
    _fit_plainly(refs, page, tables, s["nothing"])
    parents = s["parents"].long()
    lens = s["src_lens"][parents]
    src = s["src_tables"][parents]
    full = (lens // page)[:, None]
    col = torch.arange(src.shape[1], device=DEVICE)[None, :]
    shared = col < full
    tables[:, :src.shape[1]] = torch.where(shared, src, -1)
    _count(refs, src[shared], 1)
    _fit_plainly(refs, page, tables, lens)                                      # the pages that are begun
    begun = (lens % page > 0).nonzero()[:, 0]
    rest = (torch.arange(page, device=DEVICE)[None, :] < (lens % page)[begun, None])[:, None, :, None]
    at_from, at_to = (torch.gather(x, 1, full.long())[begun, 0].long() for x in (torch.cat((src, src[:, :1]), dim=1), tables))
    for cache in (s["k_cache"], s["v_cache"]):
        cache[:, at_to] = torch.where(rest, cache[:, at_from], cache[:, at_to])
    return s["k_cache"], s["v_cache"], tables, lens, refs


def _plain_fit(s):
    _fit_plainly(s["refs"], s["case"]["page"], s["tables"], s["after"])
    missing = _fit_plainly(s["refs"], s["case"]["page"], s["tables"], s["next"])
    return s["tables"], s["refs"], missing


# ---- the definitions in 64 bits ----------------------------------------------------------------------------

def exact(case, seed):
    if case["op"] == "fit":
        return None                 # whole numbers only
    with torch.no_grad():
        return {"tree": _exact_tree, "keep": _exact_keep, "fork": _exact_fork}[case["op"]](prepare(case, seed))


def _exact_tree(s):
    hq, hkv = s["case"]["hq"], s["case"]["hkv"]
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    lse = torch.full((hq, s["q"].shape[0]), -math.inf, dtype=torch.float64, device=DEVICE)

    def read(cache, table, length):
        x = cache[table[table >= 0].long()].double()                            # [pages, kv heads, page, d]
        return x.transpose(0, 1).flatten(1, 2)[:, :length]

    sets = _ancestor_sets(s["case"])
    prompt_lens, resp_lens, b, t = s["prompt_lens"].tolist(), s["resp_lens"].tolist(), 0, 0
    for g, members in enumerate(s["Gs"]):
        shared = [read(c, s["prompt_tables"][g], prompt_lens[g]) for c in (s["k_cache"], s["v_cache"])]
        for n in range(b, b + members):
            count = s["new_lens"][n]
            k, v = (torch.cat((p, read(c, s["resp_tables"][n], resp_lens[n])), dim=1) for p, c in zip(shared, (s["k_cache"], s["v_cache"])))
            unseen = torch.tensor([[not x >> m & 1 for m in range(count)] for x in sets[n]], device=DEVICE)
            ahead = torch.zeros((count, k.shape[1] - count), dtype=torch.bool, device=DEVICE)
            unseen = torch.cat((ahead, unseen), dim=1).repeat_interleave(hq // hkv, dim=0)
            q = s["q"][t:t + count].double().unflatten(1, (hkv, -1)).transpose(0, 1).flatten(1, 2)      # [kv heads, drafted * heads of each, d]
            score = torch.bmm(q, k.transpose(1, 2).contiguous()) * s["scale"]
            score[:, unseen] = -math.inf
            lse[:, t:t + count] = torch.logsumexp(score, dim=2).unflatten(1, (count, -1)).transpose(1, 2).flatten(0, 1)
            o[t:t + count] = torch.bmm(torch.softmax(score, dim=2), v.contiguous()).unflatten(1, (count, -1)).transpose(0, 1).flatten(1, 2)
            t += count
        b += members
    return o, lse


def _exact_keep(s):
    page = s["case"]["page"]
    caches = [s["k_cache"].double(), s["v_cache"].double()]
    lens, n_kept, kept = s["lens"].tolist(), s["n_kept"].tolist(), s["kept"].tolist()
    for n, table in enumerate(s["tables"].tolist()):
        here = [lens[n] + x for x in kept[n][:n_kept[n]]]
        there = range(lens[n], lens[n] + n_kept[n])
        for cache in caches:
            rows = [cache[:, table[j // page], :, j % page].clone() for j in here]
            for j, row in zip(there, rows):
                cache[:, table[j // page], :, j % page] = row
    return caches[0], caches[1], None


def _exact_fork(s):
    page = s["case"]["page"]
    caches = [s["k_cache"].double(), s["v_cache"].double()]
    lens, free = s["src_lens"].tolist(), [i for i, r in enumerate(s["refs"].tolist()) if r == 0]
    sources = s["src_tables"].tolist()
    for parent in s["parents"].tolist():
        whole, rows = divmod(lens[parent], page)
        if rows:
            to = free.pop(0)
            for cache in caches:
                cache[:, to, :, :rows] = cache[:, sources[parent][whole], :, :rows]
    return caches[0], caches[1], None, None, None

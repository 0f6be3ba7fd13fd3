"""CPU fp64 oracle of the rollout step: a paged cache, the attention of one new token per sequence over it or of several drafted
ones, the pages of sequences that branch, and logits adjusted ahead of a draw with their log-probabilities and gradient.  Written from the formulas, token by token and
row by row; imports nothing from the package."""
import numpy as np

COUNT_MAX = 32767


def rotate(x, position, base):
    """Half-split rotary embedding of x [heads, d] at one position."""
    x = np.asarray(x, dtype=np.float64)
    d = x.shape[-1]
    angle = position * np.power(float(base), -2.0 * np.arange(d // 2) / d)
    a, b = x[..., : d // 2], x[..., d // 2:]
    return np.concatenate((a * np.cos(angle) - b * np.sin(angle), a * np.sin(angle) + b * np.cos(angle)), axis=-1)


def cache_append(k_cache, v_cache, q, k, v, new_lens, tables, lens, pos_base, base):
    """Returns (k_cache, v_cache, q_out, k_out, lens_out); rows of sequences that take no part are NaN in q_out and k_out."""
    kc, vc = np.array(k_cache, dtype=np.float64), np.array(v_cache, dtype=np.float64)
    n_pages, _, page, _ = kc.shape
    q_out, k_out, lens_out = np.full(q.shape, np.nan), np.full(k.shape, np.nan), np.array(lens)
    t = 0
    for s, count in enumerate(new_lens):
        if lens[s] >= 0:
            capacity = len(tables[s]) * page
            lens_out[s] = max(lens[s], min(lens[s] + count, capacity))
            for i in range(count):
                j = lens[s] + i
                position = j + (pos_base[s] if pos_base is not None else 0)
                q_out[t + i], k_out[t + i] = rotate(q[t + i], position, base), rotate(k[t + i], position, base)
                if j < capacity and 0 <= tables[s][j // page] < n_pages:
                    kc[tables[s][j // page], :, j % page] = k_out[t + i]
                    vc[tables[s][j // page], :, j % page] = v[t + i]
        t += count
    return kc, vc, q_out, k_out, lens_out


def sequence_keys(cache, table, length):
    """Rows [n, kv heads, d] of a sequence's first `length` tokens, without those on pages outside the cache."""
    n_pages, _, page, _ = cache.shape
    rows = [cache[table[j // page], :, j % page] for j in range(min(max(length, 0), len(table) * page)) if 0 <= table[j // page] < n_pages]
    return np.array(rows, dtype=np.float64).reshape(len(rows), cache.shape[1], cache.shape[3])


def decode(k_cache, v_cache, q, Gs, prompt_tables, prompt_lens, resp_tables, resp_lens, scale):
    """Returns (o, lse, weight, reach, count): weight[s, h] = sum_j p_j |v_j| per element, reach[h, s] = the largest
    scale * sum_i |q_i k_ji|, and the keys of each row, for error bounds."""
    n, hq, d = q.shape
    hkv = k_cache.shape[1]
    o, weight = np.zeros((n, hq, d)), np.zeros((n, hq, d))
    lse, reach, count = np.full((hq, n), -np.inf), np.zeros((hq, n)), np.zeros(n, dtype=int)
    s = 0
    for g, members in enumerate(Gs):
        for _ in range(members):
            if resp_lens[s] >= 0:
                parts = [(prompt_tables[g], prompt_lens[g])] if prompt_tables is not None else []
                parts.append((resp_tables[s] if resp_tables is not None else [], resp_lens[s]))
                k, v = (np.concatenate([sequence_keys(c, *p) for p in parts]) for c in (k_cache, v_cache))
                count[s] = len(k)
                for h in range(hq if len(k) else 0):
                    kh, vh, qh = k[:, h * hkv // hq], v[:, h * hkv // hq], q[s, h].astype(np.float64)
                    score = scale * (kh @ qh)
                    top = score.max()
                    p = np.exp(score - top)
                    lse[h, s] = top + np.log(p.sum())
                    o[s, h], weight[s, h] = (p @ vh) / p.sum(), (p @ np.abs(vh)) / p.sum()
                    reach[h, s] = scale * (np.abs(kh) @ np.abs(qh)).max()
            s += 1
    return o, lse, weight, reach, count


def tree_decode(k_cache, v_cache, q, Gs, new_lens, ancestors, prompt_tables, prompt_lens, resp_tables, resp_lens, scale):
    """Attention of drafted tokens; ancestors: per row a list of the drafted tokens of its sequence that it attends to, or None (those up to
    itself).  Returns what decode() returns, a row per token."""
    T, hq, d = q.shape
    hkv = k_cache.shape[1]
    o, weight = np.zeros((T, hq, d)), np.zeros((T, hq, d))
    lse, reach, count = np.full((hq, T), -np.inf), np.zeros((hq, T)), np.zeros(T, dtype=int)
    s, t = 0, 0
    n_pages, _, page, _ = k_cache.shape
    for g, members in enumerate(Gs):
        for _ in range(members):
            n, length = new_lens[s], resp_lens[s]
            table = list(resp_tables[s]) if resp_tables is not None else []
            for i in range(n):
                places = []
                if length >= 0:
                    if prompt_tables is not None:
                        places += [(prompt_tables[g][j // page], j % page) for j in range(min(max(prompt_lens[g], 0), len(prompt_tables[g]) * page))]
                    sees = range(i + 1) if ancestors is None else ancestors[t]
                    own = [j for j in range(min(length, len(table) * page)) if j < length - n or j - (length - n) in sees]
                    places += [(table[j // page], j % page) for j in own]
                places = [(p, r) for p, r in places if 0 <= p < n_pages]
                count[t] = len(places)
                if places:
                    at, row = (np.array(x) for x in zip(*places))
                    k, v = k_cache[at, :, row].astype(np.float64), v_cache[at, :, row].astype(np.float64)
                    for h in range(hq):
                        kh, vh, qh = k[:, h * hkv // hq], v[:, h * hkv // hq], q[t, h].astype(np.float64)
                        score = scale * (kh @ qh)
                        top = score.max()
                        p = np.exp(score - top)
                        lse[h, t] = top + np.log(p.sum())
                        o[t, h], weight[t, h] = (p @ vh) / p.sum(), (p @ np.abs(vh)) / p.sum()
                        reach[h, t] = scale * (np.abs(kh) @ np.abs(qh)).max()
                t += 1
            s += 1
    return o, lse, weight, reach, count


def cache_keep(caches, tables, lens, kept, n_kept):
    """Kept tokens moved together in caches [layers, pages, heads, page, d]; returns (caches, lens_out)."""
    caches, lens_out = [np.array(c) for c in caches], list(lens)
    _, n_pages, _, page, _ = caches[0].shape
    for s, table in enumerate(tables):
        if lens[s] < 0:
            continue
        before = -1
        for i in range(min(max(n_kept[s], 0), len(kept[s]))):
            x = kept[s][i]
            if x <= before or lens[s] + x >= len(table) * page:
                break
            before = x
            lens_out[s] += 1
            src, dst = lens[s] + x, lens[s] + i
            a, b = table[src // page], table[dst // page]
            if 0 <= a < n_pages and 0 <= b < n_pages:
                for c in caches:
                    c[:, b, :, dst % page] = c[:, a, :, src % page]
    return caches, lens_out


def pages_fit(refs, page, tables, lens):
    """Returns (refs, tables, missing)."""
    refs, tables, missing = list(refs), [list(t) for t in tables], 0
    n = len(refs)
    for table, length in zip(tables, lens):
        if length >= 0:
            for c in range(min(-(-length // page), len(table)), len(table)):
                if 0 <= table[c] < n:
                    refs[table[c]] -= 1
                table[c] = -1
    free = [p for p in range(n) if refs[p] == 0]
    for table, length in zip(tables, lens):
        for c in range(min(-(-max(length, 0) // page), len(table))):
            if not 0 <= table[c] < n:
                table[c] = free.pop(0) if free else -1
                if table[c] < 0:
                    missing += 1
                else:
                    refs[table[c]] = 1
    return refs, tables, missing


def cache_fork(caches, refs, parents, src_tables, src_lens, tables, lens_out):
    """Returns (caches, refs, tables, lens_out)."""
    caches, refs, tables, lens_out = [np.array(c) for c in caches], list(refs), [list(t) for t in tables], list(lens_out)
    _, n_pages, _, page, _ = caches[0].shape
    free = [p for p in range(n_pages) if refs[p] == 0]
    for s, parent in enumerate(parents):
        if not 0 <= parent < len(src_tables):
            continue
        src, width = src_tables[parent], len(tables[s])
        length = min(src_lens[parent], min(len(src), width) * page)
        row = [-1] * width
        if length >= 0:
            whole, rest = divmod(length, page)
            row[:whole] = src[:whole]
            if rest:
                row[whole] = src[whole]
                if 0 <= src[whole] < n_pages:
                    if not free:
                        tables[s], lens_out[s] = [-1] * width, -1
                        continue
                    row[whole] = free.pop(0)
                    refs[row[whole]] = 1
                    for c in caches:
                        c[:, row[whole], :, :rest] = c[:, src[whole], :, :rest]
            for p in src[:whole]:
                if 0 <= p < n_pages:
                    refs[p] += 1
        tables[s], lens_out[s] = row, length
    return caches, refs, tables, lens_out


def adjust_row(z, prompt, generated, rules, bias=None, allowed=None):
    """Adjusted row, its derivative by the raw row, and a bound on the magnitudes that went into each element.
    rules = (repetition, presence, frequency, temperature)."""
    repetition, presence, frequency, temperature = rules
    z = np.asarray(z, dtype=np.float64)
    a = z if bias is None else z + np.asarray(bias, dtype=np.float64)
    out, slope, size = np.empty_like(a), np.empty_like(a), np.empty_like(a)
    counts = {}
    for token in generated:
        counts[token] = counts.get(token, 0) + 1
    seen = set(counts) | set(prompt)
    for v in range(len(a)):
        factor = 1.0
        if v in seen:
            factor = 1.0 / repetition if a[v] > 0 else repetition
        c = min(counts.get(v, 0), COUNT_MAX)
        out[v] = (a[v] * factor - frequency * c - (presence if c > 0 else 0.0)) / temperature
        slope[v] = factor / temperature
        size[v] = ((abs(z[v]) + abs(a[v])) * factor + abs(frequency * c) + abs(presence)) / temperature
    if allowed is not None:
        out[~allowed], slope[~allowed], size[~allowed] = -np.inf, 0.0, 0.0
    return out, slope, size


def unpack_mask(words, vocab):
    """Boolean rows of a mask of uint32 words."""
    words = np.asarray(words).astype(np.int64) & 0xffffffff
    v = np.arange(vocab)
    return (words[:, v // 32] >> (v % 32)) & 1 == 1


def adjusted_logprob(logits, labels, tokens, g, rules, prompt_lens, Gs, resp_lens, bias=None, allowed=None, own_token=False):
    """Returns (rows, logp, lse, dlogits, size): the response rows, and for each its log-probability, normaliser, gradient and the largest
    magnitude of adjust_row among its allowed elements (for error bounds)."""
    rows, logp, lse, grads, sizes = [], [], [], [], []
    at, r = 0, 0
    for group, members in enumerate(Gs):
        prompt = tokens[at: at + prompt_lens[group]]
        at += prompt_lens[group]
        for length in resp_lens[r: r + members]:
            for t in range(at, at + length):
                z, slope, size = adjust_row(logits[t], prompt, tokens[at: t + int(own_token)], rules, bias, None if allowed is None else allowed[t])
                top = z.max()
                empty = top == -np.inf
                e = np.zeros_like(z) if empty else np.exp(z - top)
                L = -np.inf if empty else top + np.log(e.sum())
                y = labels[t]
                rows.append(t)
                lse.append(L)
                logp.append(z[y] - L if 0 <= y < len(z) and not empty else -np.inf)
                pick = np.zeros_like(z)
                if 0 <= y < len(z):
                    pick[y] = 1.0
                grads.append(np.zeros_like(z) if empty else g[t] * (pick - e / e.sum()) * slope)
                sizes.append(size[np.isfinite(z)].max() if not empty else 0.0)
            at += length
        r += members
    return np.array(rows, dtype=int), np.array(logp), np.array(lse), np.array(grads), np.array(sizes)

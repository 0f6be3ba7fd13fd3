"""Seeded inputs of the tests of sequences that branch."""
import torch


def dev32(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def random_trees(gen, new_lens):
    """Per drafted token the drafted tokens that it sees: itself and those on the way to the root; parents are drawn among all ahead of it."""
    rows = []
    for n in new_lens:
        mine = []
        for i in range(n):
            parent = int(torch.randint(-1, i, (1,), generator=gen)) if i else -1
            mine.append((mine[parent] if parent >= 0 else []) + [i])
        rows += mine
    return rows


def mask_words(rows, words):
    """int32 [rows, words] with bit m of a row set for each m of its list."""
    out = torch.zeros(len(rows), words, dtype=torch.int64)
    for t, row in enumerate(rows):
        for m in row:
            out[t, m // 32] |= 1 << m % 32
    return out.to(torch.int32)

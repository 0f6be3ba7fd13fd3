"""Seeded inputs and error bounds of the rollout tests."""
import numpy as np
import torch

U24 = 2.0 ** -24
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: U24}     # relative rounding error of one store at most


def make_tables(gen, lens, page, spare=3):
    """Page tables of the given lengths (pages in random order, -1 behind the last) and how many pages there are."""
    need = [-(-max(n, 0) // page) for n in lens]
    order = torch.randperm(sum(need) + spare, generator=gen).tolist()
    table, at = torch.full((len(lens), max(1, max(need))), -1, dtype=torch.int32), 0
    for i, n in enumerate(need):
        table[i, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    return table, len(order)


def numpy64(x):
    return x.detach().cpu().double().numpy()


def decode_bounds(o, lse, weight, reach, count, d, dtype):
    """(bound of o, bound of lse).  A score is a float32 sum of d products, off by (d + 4) 2^-24 of reach in any order; an exponential by
    that, by the rounding of its argument (weights that count are above e^-100) and by its own 4 units; sums of n terms by n / 16 + 64
    units (64 lanes or more share them, then their partial sums are joined).  bf16: the weights are rounded once (2^-8), and o is (2^-8)."""
    score = (d + 4) * U24 * reach
    unit = (110 + 4 + 64 + count / 16) * U24
    lse_tol = score + (unit + 4 * U24 * np.maximum(1.0, np.abs(np.where(np.isfinite(lse), lse, 0.0))))
    rel = 2 * (score + unit).T[:, :, None]
    half = HALF_STEP[dtype]
    return weight * (rel + (half if dtype == torch.bfloat16 else 0.0)) + np.abs(o) * half + 1e-37, lse_tol


def check(name, got, want, tol):
    got = numpy64(got) if isinstance(got, torch.Tensor) else got
    finite = np.isfinite(want)
    assert np.array_equal(finite, np.isfinite(got)), f"{name}: infinities or NaN differ"
    assert np.array_equal(got[~finite], want[~finite]), f"{name}: infinities differ"
    over = np.abs(got[finite] - want[finite]) - np.broadcast_to(tol, want.shape)[finite]
    assert over.size == 0 or over.max() <= 0, f"{name}: {over.max():.3e} beyond the bound"

"""NaN and infinities in what a new token does attend to: they reach its row, and no other."""
import pytest
import torch

from paper_2511_18871_amd import binding as B
from tests.rollout import make_tables

pytestmark = pytest.mark.gpu
TYPES = [(torch.bfloat16, 128), (torch.bfloat16, 64), (torch.float32, 128), (torch.float32, 64)]
# one sequence; a prompt for a wave and for several workgroups; more rows than the join gives waves of their own
LAYOUTS = {"one": (4, 1, [0], [1], [333]), "solo": (8, 2, [600], [5], [3, 70, 1, 0, 33]), "shared": (8, 2, [300], [24], [5 * i % 31 + 1 for i in range(24)]),
           "dense": (28, 4, [(i * 37) % 90 for i in range(43)], [7] * 43, [(i * 11) % 40 + 1 for i in range(301)])}


def dev32(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


def make(layout, dtype, d):
    hq, hkv, prompts, Gs, resp = LAYOUTS[layout]
    gen = torch.Generator().manual_seed(11)
    tables, pages = make_tables(gen, prompts + resp, 16)
    kc, vc = (torch.randn(pages, hkv, 16, d, generator=gen).to(dtype) for _ in range(2))
    q = torch.randn(len(resp), hq, d, generator=gen).to(dtype)
    pt, rt = tables[:len(prompts)].contiguous(), tables[len(prompts):].contiguous()
    def run(q, k):
        return B.sp_attn_decode(B.KvCache(k.cuda(), vc.cuda()), q.cuda(), Gs, pt.cuda(), dev32(prompts), rt.cuda(), dev32(resp), 0.1)
    return q, kc, pt, rt, run


def only(rows, got, clean):
    """rows [sequences, heads] are NaN; the others are what they were, but for another order of their sums."""
    (o, lse), (o0, lse0) = [[x.cpu() for x in y] for y in (got, clean)]
    assert torch.equal(o.isnan(), rows[:, :, None].expand_as(o)) and torch.equal(lse.isnan(), rows.t())
    rtol, atol = (2.0 ** -7, 2e-5) if o.dtype is torch.bfloat16 else (1e-5, 1e-5)
    assert torch.allclose(o[~rows].double(), o0[~rows].double(), rtol=rtol, atol=atol)
    assert torch.allclose(lse[~rows.t()], lse0[~rows.t()], rtol=1e-5, atol=1e-5)


@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("dtype,d", TYPES)
def test_nan_in_a_query(dtype, d, layout):
    q, kc, _, _, run = make(layout, dtype, d)
    clean = run(q, kc)
    rows = torch.zeros(q.shape[:2], dtype=torch.bool)
    for s, h in ((0, 0), (q.shape[0] - 1, q.shape[1] - 1), (q.shape[0] // 2, 1)):
        q[s, h, (7 * s + h) % d] = float("nan")
        rows[s, h] = True
    only(rows, run(q, kc), clean)


@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("dtype,d", TYPES)
def test_nan_in_a_key(dtype, d, layout):
    q, kc, pt, rt, run = make(layout, dtype, d)
    hq, hkv, prompts, Gs, resp = LAYOUTS[layout]
    rep = hq // hkv
    clean = run(q, kc)
    for s, j in ((0, 0), (len(resp) - 1, resp[-1] - 1)):                     # the first key of a response, the last of another
        k, rows = kc.clone(), torch.zeros(q.shape[:2], dtype=torch.bool)
        k[rt[s, j // 16], hkv - 1, j % 16, 5] = float("nan")
        rows[s, -rep:] = True
        only(rows, run(q, k), clean)
    if prompts[-1]:
        j = prompts[-1] - 1
        k, rows = kc.clone(), torch.zeros(q.shape[:2], dtype=torch.bool)
        k[pt[-1, j // 16], 0, j % 16] = float("nan")
        rows[len(resp) - Gs[-1]:, :rep] = True
        only(rows, run(q, k), clean)


@pytest.mark.parametrize("layout", list(LAYOUTS))
@pytest.mark.parametrize("dtype,d", TYPES)
def test_a_score_beyond_the_range(dtype, d, layout):
    q, kc, _, rt, run = make(layout, dtype, d)
    kc[rt[0, 0], 0, 0, 0] = 1e30
    q[0, :, 0] = 1.0
    clean = run(q, kc)
    rows = torch.zeros(q.shape[:2], dtype=torch.bool)
    q[0, 1, 0], rows[0, 1] = 1e30, True
    only(rows, run(q, kc), clean)


@pytest.mark.parametrize("dtype,d", TYPES)
def test_an_infinite_value_reaches_its_element(dtype, d):
    """Of every row that sees it, and nothing else: also where its key's weight is exactly 1, and whatever the number of partial sums."""
    gen = torch.Generator().manual_seed(7)
    hq, hkv, page = 8, 2, 16
    prompts, Gs, resp = [600], [5], [3, 70, 1, 0, 33]
    tables, pages = make_tables(gen, prompts + resp, page)
    kc, vc = (torch.randn(pages, hkv, page, d, generator=gen).to(dtype) for _ in range(2))
    q = torch.randn(5, hq, d, generator=gen).to(dtype)
    args = (q.cuda(), Gs, tables[:1].contiguous().cuda(), dev32(prompts), tables[1:].contiguous().cuda(), dev32(resp), 0.1)
    bad = vc.clone()
    bad[tables[0, 2], 0, 5, 3] = float("inf")                # a prompt key of kv head 0, seen by all
    bad[tables[2, 4], 1, 2, 9] = -float("inf")               # key 66 of response 1, kv head 1
    kc[tables[3, 0], 1, 0] = 0
    bad[tables[3, 0], 1, 0, 4] = float("inf")                # the only key of response 2's own, beside the prompt
    clean, clean_lse = B.sp_attn_decode(B.KvCache(kc.cuda(), vc.cuda()), *args)
    o, lse = B.sp_attn_decode(B.KvCache(kc.cuda(), bad.cuda()), *args)
    want = clean.clone()
    want[:, :4, 3] = float("inf")
    want[1, 4:, 9] = -float("inf")
    want[2, 4:, 4] = float("inf")
    assert torch.equal(o, want) and torch.equal(lse, clean_lse)
    alone = B.sp_attn_decode(B.KvCache(kc.cuda(), bad.cuda()), args[0], None, None, None, args[4], dev32([0, 0, 1, 0, 0]), 0.1)[0]      # weight 1
    assert torch.all(alone[2, 4:, 4] == float("inf")) and torch.isfinite(alone[2, :4]).all()

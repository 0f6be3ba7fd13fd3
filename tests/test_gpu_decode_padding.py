"""What a page table holds behind a list's last page does not matter, whatever it is, and a bad page among a list's own is passed over alone."""
import pytest
import torch

from oracle import rollout_oracle as ro
from paper_2511_18871_amd import binding as B
from tests.rollout import check, decode_bounds, make_tables, numpy64

pytestmark = pytest.mark.gpu


def dev32(x):
    return torch.tensor(x, dtype=torch.int32).cuda()


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.float32, 64)])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("members", [2, 40])                    # lists of a wave, shared ones
def test_padding_of_tables(dtype, d, page, members):
    gen = torch.Generator().manual_seed(page)
    prompts, Gs = [64 * page + 5, 40, 0], [members, 3, 1]
    resp = [(37 * i) % 130 for i in range(members + 4)]
    tables, pages = make_tables(gen, prompts + resp, page)
    kc, vc = (torch.randn(pages, 2, page, d, generator=gen).to(dtype) for _ in range(2))
    q = torch.randn(len(resp), 4, d, generator=gen).to(dtype)
    cache, qc, pl, rl = B.KvCache(kc.cuda(), vc.cuda()), q.cuda(), dev32(prompts), dev32(resp)
    def run(tables):
        return B.sp_attn_decode(cache, qc, Gs, tables[:3].contiguous().cuda(), pl, tables[3:].contiguous().cuda(), rl, 0.1)
    want = run(tables)
    unused = tables == -1
    for pad in (0, pages - 1, pages, 2 ** 31 - 1, -2 ** 31):
        got = run(torch.where(unused, pad, tables).to(torch.int32))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), pad
    wide = torch.cat((tables, torch.full((len(tables), 70), pages + 9, dtype=torch.int32)), 1)
    got = run(wide)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    # pages 63 and 64 of the long prompt, the last of the short one, the first of a response
    bad = tables.clone()
    bad[0, 63], bad[0, 64], bad[1, (40 - 1) // page], bad[4, 0] = -1, pages, -7, pages + 1
    o, lse = run(bad)
    ref, rlse, weight, reach, count = ro.decode(numpy64(kc), numpy64(vc), numpy64(q), Gs, bad[:3].tolist(), prompts, bad[3:].tolist(), resp, 0.1)
    tol_o, tol_lse = decode_bounds(ref, rlse, weight, reach, count, d, dtype)
    check("lse", lse, rlse, tol_lse)
    check("o", o, ref, tol_o)

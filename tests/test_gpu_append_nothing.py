"""An append of no tokens: lengths are handed on, and what is wrong is refused as with tokens."""
import pytest
import torch

from paper_2511_18871_amd import binding as B

pytestmark = pytest.mark.gpu


def test_no_tokens():
    k, v = (torch.ones(6, 2, 16, 64, device="cuda") for _ in range(2))
    cache, empty = B.KvCache(k, v), torch.empty(0, 2, 64, device="cuda")
    n = 300
    lens = (torch.arange(n, dtype=torch.int32) % 37 - 2).cuda()
    tables = torch.zeros(n, 3, dtype=torch.int32, device="cuda")
    for q in (None, torch.empty(0, 8, 64, device="cuda")):
        q_out, now = B.sp_attn_cache_append(cache, empty, empty, tables, lens, 1e4, q=q, new_lens=[0] * n)
        assert torch.equal(now, lens) and (q_out is None if q is None else q_out.shape == (0, 8, 64))
    assert torch.all(k == 1) and torch.all(v == 1)
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    assert B.sp_attn_cache_append(cache, empty, empty, tables[:0], none, 1e4)[1].shape == (0,)
    for kw in (dict(rope_base=0.5), dict(rope_base=float("nan")), dict(new_lens=[-1, 1] + [0] * (n - 2)), dict(lens_out=lens)):
        args = dict(dict(rope_base=1e4, new_lens=[0] * n), **kw)
        with pytest.raises(B.SpAttnError) as e:
            B.sp_attn_cache_append(cache, empty, empty, tables, lens, **args)
        assert e.value.status == B.SP_ERR_INVALID_ARG, kw

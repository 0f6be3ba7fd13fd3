"""What the rollout calls of the binding refuse because the library could not see it; on the host, no kernel is launched."""
import pytest
import torch

from paper_2511_18871_amd import binding as B


def message(f, *args, **kw):
    with pytest.raises(B.SpAttnError) as e:
        f(*args, **kw)
    assert e.value.status == B.SP_ERR_INVALID_ARG
    return str(e.value)


def i32(*s):
    return torch.zeros(*s, dtype=torch.int32)


# two groups, three responses; each list alone fits the pack's 7 rows
@pytest.mark.parametrize("prompts,Gs,resp", [([2, 1], [3], [1, 2, 1]), ([2, 1], [1, 1, 1], [1, 2, 1]), ([2, 1], [1, 1], [1, 2, 1]), ([2, 1], [2, 2], [1, 2, 1]),
                                             ([2, 1], [5, -2], [1, 2, 1]), ([2, 1], [], [1, 2, 1]), ([2, 1], [2, 1], [1, 3])])
def test_lists_of_a_pack_that_do_not_fit(prompts, Gs, resp):
    z, t = torch.zeros(7, 40), i32(7)
    rules = B.LogitRules()
    assert "do not fit" in message(B.sp_attn_adjusted_logprob_fwd, z, t, t, rules, prompts, Gs, resp)
    assert "do not fit" in message(B.sp_attn_adjusted_logprob_bwd, z, t, t, torch.zeros(7), torch.zeros(7), rules, prompts, Gs, resp)


@pytest.mark.parametrize("workspace", [torch.zeros(1, dtype=torch.uint8).expand(1 << 24), torch.zeros(64, 64, dtype=torch.uint8).t(), torch.zeros(64, dtype=torch.uint8)[::2]])
def test_workspaces_whose_bytes_are_not_there(workspace):
    z, t, rules = torch.zeros(7, 40), i32(7), B.LogitRules()
    pack = ([2, 1], [2, 1], [1, 2, 1])
    k = torch.zeros(4, 2, 16, 64)
    assert "workspace" in message(B.sp_attn_adjusted_logprob_fwd, z, t, t, rules, *pack, workspace=workspace)
    assert "workspace" in message(B.sp_attn_adjusted_logprob_bwd, z, t, t, torch.zeros(7), torch.zeros(7), rules, *pack, workspace=workspace)
    assert "workspace" in message(B.sp_attn_decode, B.KvCache(k, k), torch.zeros(3, 4, 64), None, None, None, i32(3, 2), i32(3), 0.1, workspace=workspace)


def test_prompt_tables_and_lengths_go_together():
    k, q = torch.zeros(4, 2, 16, 64), torch.zeros(3, 4, 64)
    for tables, lens in ((i32(3, 2), None), (None, i32(3))):
        assert "go together" in message(B.sp_attn_decode, B.KvCache(k, k), q, None, tables, lens, i32(3, 2), i32(3), 0.1)


@pytest.mark.gpu
def test_a_workspace_on_the_host():
    z, t, rules, ws = torch.zeros(7, 40).cuda(), i32(7).cuda(), B.LogitRules(), torch.empty(1 << 24, dtype=torch.uint8)
    pack = ([2, 1], [2, 1], [1, 2, 1])
    k = torch.zeros(4, 2, 16, 64).cuda()
    assert "workspace" in message(B.sp_attn_adjusted_logprob_fwd, z, t, t, rules, *pack, workspace=ws)
    assert "workspace" in message(B.sp_attn_adjusted_logprob_bwd, z, t, t, z[:, 0].contiguous(), z[:, 0].contiguous(), rules, *pack, workspace=ws)
    assert "workspace" in message(B.sp_attn_decode, B.KvCache(k, k), torch.zeros(3, 4, 64).cuda(), None, None, None, i32(3, 2).cuda(), i32(3).cuda(), 0.1, workspace=ws)

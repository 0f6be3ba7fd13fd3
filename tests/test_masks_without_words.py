"""A mask whose rows have no words is refused: its address is none, as if there were no mask."""
import pytest
import torch

from paper_2511_18871_amd import binding as B


@pytest.mark.parametrize("dtype", [torch.int32, torch.uint32])
def test_a_mask_without_words_is_refused(dtype):
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)
    cache, empty, logits = B.KvCache(torch.zeros(4, 2, 16, 64), torch.zeros(4, 2, 16, 64)), torch.zeros(3, 0, dtype=dtype), torch.zeros(3, 40)
    for call in (lambda: B.sp_attn_tree_decode(cache, torch.zeros(3, 4, 64), None, [3], empty, None, None, i32(1, 2), i32(1), 0.1),
                 lambda: B.sp_attn_adjust_logits(logits, B.LogitRules(), None, None, None, None, None, mask=empty),
                 lambda: B.sp_attn_adjusted_logprob_fwd(logits, i32(3), i32(3), B.LogitRules(), [1], [1], [2], mask=empty)):
        with pytest.raises(B.SpAttnError, match="words") as e:
            call()
        assert e.value.status == B.SP_ERR_INVALID_ARG

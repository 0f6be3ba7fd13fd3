"""Factors whose product with log2(e) float32 does not hold are refused, on the host; no kernel is launched."""
import pytest

from paper_2511_18871_amd import binding as B
from tests.test_rollout_refusals import P, decode, ints, lib, rules  # noqa: F401


@pytest.mark.parametrize("scale", [2.4e38, 3.4e38])
def test_scales(lib, scale):
    assert decode(lib, scale=scale) == B.SP_ERR_INVALID_ARG and b"softmax_scale" in lib.sp_attn_last_error()


@pytest.mark.parametrize("temperature", [3e-39, 4.2e-39])
def test_temperatures(lib, temperature):
    pack = (ints(4), ints(1), ints(3))
    args = (100, rules(temp=temperature), None, 0, 1, *pack, B.SP_F32, 0, P, 1 << 20, None)
    assert lib.sp_attn_adjusted_logprob_fwd(P, P, P, P, P, *args) == B.SP_ERR_INVALID_ARG and b"temperature" in lib.sp_attn_last_error()
    assert lib.sp_attn_adjusted_logprob_bwd(P, P, P, P, P, P, *args) == B.SP_ERR_INVALID_ARG and b"temperature" in lib.sp_attn_last_error()


def test_the_largest_that_pass(lib):
    """They are not refused: what is, comes behind them."""
    assert decode(lib, scale=2.35e38, Gs=ints(4, -1)) == B.SP_ERR_INVALID_ARG and b"negative" in lib.sp_attn_last_error()
    args = (100, rules(temp=4.3e-39), None, 0, 1, ints(4), ints(1), ints(-1), B.SP_F32, 0, P, 1 << 20, None)
    assert lib.sp_attn_adjusted_logprob_fwd(P, P, P, P, P, *args) == B.SP_ERR_INVALID_ARG and b"temperature" not in lib.sp_attn_last_error()

"""An append writes the new lengths while it reads its other arrays: memory that they share is refused, on the host (no kernel is launched)."""
import pytest

from paper_2511_18871_amd import binding as B
from tests.test_rollout_refusals import append, lib  # noqa: F401

LENS, BASE, TABLES = 0x10000, 0x20000, 0x30000        # two sequences: 8, 8 and 24 bytes


@pytest.mark.parametrize("out", [LENS, LENS + 4, LENS - 4, BASE, BASE + 4, BASE - 4, TABLES, TABLES + 20, TABLES - 4])
def test_lengths_that_overlap(lib, out):
    assert append(lib, lens=LENS, base=BASE, tables=TABLES, lens_out=out) == B.SP_ERR_INVALID_ARG
    assert b"overlap" in lib.sp_attn_last_error()


@pytest.mark.parametrize("out", [LENS + 8, LENS - 8, BASE + 8, TABLES + 24, TABLES - 8, None])
def test_neighbours_are_not_refused(lib, out):
    """Seen by the next check: a rotation's base that is refused."""
    assert append(lib, lens=LENS, base=BASE, tables=TABLES, lens_out=out, rope=0.5) == B.SP_ERR_INVALID_ARG
    assert b"rope_base" in lib.sp_attn_last_error()

"""Sizes of hs_kv_attend that 31 bits do not hold with a step of tokens added
(no GPU needed)."""
import pytest

from paper_2607_22578_gb300 import _lib
from test_kv_abi import attend, cache, message


@pytest.mark.parametrize("bt", [16, 32, 64, 128])
def test_rows_of_a_table_end_before_31_bits_do(bt):
    most = ((1 << 31) - 512) // bt
    for width in (most + 1, most + 256 // bt, (1 << 31) // bt):
        assert attend(c=cache(bt=bt), width=width) == _lib.HS_ERR_INVALID_ARG
        assert "table_width" in message()
    # the most there may be is not what is refused
    assert attend(c=cache(bt=bt), width=most, q=None) == _lib.HS_ERR_INVALID_ARG
    assert "NULL" in message()

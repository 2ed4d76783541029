"""Limits of the block-sparse calls at the ends of their integer ranges, without a device."""

import pytest

from paper_2410_05076_b200 import binding
from tests.test_blocks_abi import ATTN, call


@pytest.mark.parametrize("m", [2 ** 30 + 1, 2 ** 31 - 1])
def test_lists_whose_rounds_would_pass_32_bits_are_refused(m):
    assert call("tidal_block_attn", ATTN, dict(m=m)) == binding.ERR_UNSUPPORTED

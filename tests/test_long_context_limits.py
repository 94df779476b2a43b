"""Sizes at both sides of the long-context operators' limits, checked on the host."""
import os

import pytest

from paper_2305_19370_amd import bpt

pytestmark = pytest.mark.skipif(not os.path.exists(bpt.LIB_PATH), reason="libbpt.so not built")


@pytest.mark.parametrize("rows,code", [(2 ** 26 - 1, 0), (2 ** 26, 0), (2 ** 26 + 5, 0), (2 ** 31 - 1, 0), (2 ** 31, 2)])
def test_rope_rows(rows, code):
    """Rows are counted in 32 bits; what is accepted is launched in parts of 2^25."""
    assert bpt.rope_validate(bpt.make_rope_config(rows, rows, 1, 8)) == code

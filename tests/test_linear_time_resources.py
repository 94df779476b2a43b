"""Registers of the recurrence's and the distillation's kernels as the compiler reports them: what a thread holds between its two passes
over the elements is not in scratch memory."""
import os

import pytest

from test_kernel_resources import _report


@pytest.mark.skipif(not os.path.exists("/opt/rocm/bin/hipcc"), reason="no hipcc")
@pytest.mark.parametrize("src,least", [("recur.hip", 10), ("distill.hip", 11)])
def test_no_scratch(src, least):
    got = _report(src)
    assert len(got) >= least and not any(got.values()), got

"""Sizes at the border of what the training step's entry points take (no GPU)."""
import os
import re

import pytest

from paper_2506_12417_amd import binding as B
from paper_2506_12417_amd import build as b
from test_train_abi import combine, permute



@pytest.mark.parametrize("T", [2 ** 26 - 3, 2 ** 26 - 2, 2 ** 26 - 1])
def test_a_launch_has_less_than_2_32_threads(T):
    """Four wavefronts a work-group: (T + 3) / 4 work-groups of 256 threads."""
    assert -(-T // 4) * 256 == 2 ** 32
    assert combine(T=T, k=1) == B.MOE_ERR_UNSUPPORTED and permute(T=T, k=1) == B.MOE_ERR_UNSUPPORTED
    assert permute(T=T // 4 + 1, d=4 * 512, k=1) == B.MOE_ERR_UNSUPPORTED


@pytest.mark.parametrize("source,kernel,names", [("sort_backward.hip", "permute_backward_kernel", ("dx_add", "dx")), ("route_backward.hip", "dx_kernel", ("add", "dx"))])
def test_arguments_that_may_be_one_tensor_are_not_declared_apart(source, kernel, names):
    """dx may be dx_add: neither may carry __restrict__, or the compiler may load behind the store."""
    text = open(os.path.join(b.CSRC, source)).read()
    arguments = re.search(r"void %s\((.*?)\)\s*\{" % kernel, text, flags=re.S).group(1)
    for name in names:
        declared = re.search(r"([^,]*[\s*])%s(?:,|$)" % name, re.sub(r"\s+", " ", arguments)).group(1)
        assert "*" in declared and "__restrict__" not in declared, declared

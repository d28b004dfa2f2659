"""Sizes at the border of what the training step's entry points take (no GPU)."""
import pytest

from paper_2506_12417_amd import binding as B
from test_train_abi import combine, permute



@pytest.mark.parametrize("T", [2 ** 26 - 3, 2 ** 26 - 2, 2 ** 26 - 1])
def test_a_launch_has_less_than_2_32_threads(T):
    """Four wavefronts a work-group: (T + 3) / 4 work-groups of 256 threads."""
    assert -(-T // 4) * 256 == 2 ** 32
    assert combine(T=T, k=1) == B.MOE_ERR_UNSUPPORTED and permute(T=T, k=1) == B.MOE_ERR_UNSUPPORTED
    assert permute(T=T // 4 + 1, d=4 * 512, k=1) == B.MOE_ERR_UNSUPPORTED

"""The 4-bit head on batches of any number of rows."""
import pytest

from .test_gpu_head import BF16, F32, check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("hidden", [BF16, F32])
def test_very_many_rows(hidden):
    """350000 states: 8334 blocks of 42 fp32 ones."""
    check(*make(350000, 60, 64, 32, True, hidden, seed=3), F32)

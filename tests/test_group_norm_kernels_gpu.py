"""Every kernel of the group norm, forward and backward, against the definition in 64 bits."""
import pytest

from kernel_sizes import GROUP_NORM
from test_group_norm_gpu import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shape", GROUP_NORM, ids=str)
@pytest.mark.parametrize("dtype", ("bfloat16", "float32"))
@pytest.mark.parametrize("act", ("silu", "relu"))
def test_kernel(shape, dtype, act):
    check(shape, dtype, act)

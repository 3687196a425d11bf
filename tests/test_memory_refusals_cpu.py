"""Numbers that the operators of policies with a memory do not take."""
import ctypes as C

import pytest

from tests.test_memory_ops_cpu import EINVAL, norm_args
from tests.test_wide_ops_cpu import aligned


@pytest.fixture(scope="module")
def A():
    import paper_2211_15023_amd as A
    A.load_library()
    return A


@pytest.mark.parametrize("name", ["block_norm", "block_norm_grad"])
@pytest.mark.parametrize("eps", [1e-50, 1e-46, 1e-39])
def test_an_eps_that_fp32_does_not_hold(A, name, eps):
    """It would be 0 to the kernels, and a row of zeros NaN."""
    p, own = aligned(1 << 17)
    a = norm_args(p, eps=eps, after=p + 16384, before=p + 17408, workspace=p + 32768, workspace_bytes=1 << 16)
    assert getattr(A.load_library(), "accerl_" + name)(C.byref(a), None) == EINVAL and "eps" in A.accerl_last_error()

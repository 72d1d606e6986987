"""Group norm over fields whose few values unlike the rest lie where a kernel may look first: the first, the middle or the last
point.  Bounds: those of test_gpu_norm.py, derived there from the arithmetic; none of them grows with what such a value is."""
import numpy as np
import pytest
import torch

from test_gpu_norm import Norm


def rounded(a):
    """float32 values that bf16 holds too, as Norm's fields are."""
    return torch.from_numpy(np.asarray(a, np.float32)).bfloat16().float().numpy()


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["first", "last"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("where", [0, 1, 2])
@pytest.mark.parametrize("far,rest", [(1e6, 0.02), (1e4, 3e-4), (1e8, 1.0), (-3e4, 5.0)])
@pytest.mark.parametrize("c,groups,p", [(1, 1, 16384), (1, 1, 16000), (2, 2, 2048), (4, 2, 1023), (4, 1, 20000), (6, 2, 90001)])
def test_one_value_far_from_all_others(c, groups, p, far, rest, where, dtype, layout):
    n = Norm(1, c, groups, p, layout, dtype, "identity")
    n.x[:] = rounded(rest)
    n.x[0, :: c // groups, (0, p // 2, p - 1)[where]] = rounded(far)         # in the first channel of every group
    y, mean, rstd = n.forward()
    n.check_forward(y, mean, rstd)
    n.check_backward(mean, rstd, *n.backward(mean, rstd))

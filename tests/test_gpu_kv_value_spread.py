"""Values of very different magnitudes in one sequence, as far apart as the header states: tokens whose values are too small to
show in the output still weigh in the softmax."""
import numpy as np
import pytest

from test_gpu_kv_value_range import KERNELS, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("small,large", [(1e-18, 1e6), (1e-6, 1e18), (1e-3, 1e3), (1e6, 1e30)])
@pytest.mark.parametrize("order", ["small first", "large first", "in turn", "by sixteen"])
@pytest.mark.parametrize("dtype,which", KERNELS)
def test_spread(small, large, order, dtype, which):
    rng = np.random.default_rng(int(np.log10(large / small)))
    n, t = 700, np.arange(700)
    at = {"small first": t < 350, "large first": t >= 350, "in turn": t % 2 == 0, "by sixteen": t // 16 % 3 != 1}[order]
    v = rng.standard_normal((n, 1, 64)) * np.where(at, small, large)[:, None, None]
    check(rng, v, dtype, which)

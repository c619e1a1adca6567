"""AdamW at the ends of its range (GPU)."""
import numpy as np
import pytest
import torch

from paper_2607_10611_amd import binding as B
from test_gpu_adamw import HP, Case, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("beta2,eps,step", [(1 - 2.0 ** -39, 4e-12, 1), (0.999999, 4e-12, 50),
                                            (0.999, 4e-12, 1), (0.999, 1e-10, 1),
                                            (0.999999, 1e-8, 1), (0.999, 1e-8, 1)])
@pytest.mark.parametrize("bits", [False, True])
def test_every_operation_is_rounded_also_where_v_is_denormal(bits, beta2, eps, step):
    """v below 2^-126 beside an eps that its root reaches, and beside one that it does
    not: the same bits as the operations one by one."""
    case = Case([4000, 129], "fp32", "fp32", bits, seed=3)
    rng = np.random.default_rng(4)
    for d, h, n in zip(case.d, case.h, case.sizes):
        size = np.sqrt(2.0 ** rng.uniform(-149, -127, n) / (1 - beta2))  # v of 2^-149 to 2^-127
        h[1] = (rng.normal(0, 1, n) * size).astype(np.float32)
        h[3] = np.zeros(n, np.float32)
        d[1].copy_(torch.from_numpy(h[1]))
        d[3].zero_()
    hp = dict(HP, step=step, rounding="rne", beta2=beta2, eps=eps)
    B.madd_adamw_step(case.list, hp)
    check(case, hp, np.float32(1.0))
    v = case.h[0][3]
    assert bits or ((v > 0) & (v < 2.0 ** -126)).any()

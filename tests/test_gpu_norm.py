"""The gradient norm to one rounding: its squares are added in 64 bits (GPU)."""
import math

import numpy as np
import pytest
import torch

from paper_2607_10611_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_norm_keeps_small_squares_beside_large_ones(dtype):
    """Each of a thread's sums gets one square of 2^24 and then seven of 1, which fp32
    would lose.  In 64 bits the norm has one rounding (to fp32, 2^-24 of it) and the
    coefficient one more; 2^-40 for the sums and the root themselves."""
    n = 4096 * 2048 * 8
    g = torch.ones(4096, 16384, dtype=dtype, device="cuda")
    g[:, :2048] = 4096.0
    want = math.sqrt(4096 * 2048 * (2.0 ** 24 + 7))
    out = torch.zeros(2, device="cuda")
    B.madd_grad_norm(B.GradList([g.view(-1)]), 1.0, out)
    norm, coef = out.double().tolist()
    assert g.numel() == n and abs(norm - want) <= (2.0 ** -24 + 2.0 ** -40) * want
    assert abs(coef - 1 / want) <= (2.0 ** -23 + 2.0 ** -40) / want


@pytest.mark.parametrize("sizes", [[1], [7, 0, 129], [100000], [3] * 400, [1 << 20, 5, 333333]])
def test_norm_is_right_to_one_rounding(sizes):
    rng = np.random.default_rng(len(sizes))
    gs, total = [], 0.0
    for i, n in enumerate(sizes):
        x = torch.from_numpy(rng.normal(0, 10.0 ** rng.uniform(-6, 0), n).astype(np.float32))
        x = x.bfloat16() if i % 2 else x
        gs.append(x.cuda())
        total += float(x.double().square().sum())
    want, out = math.sqrt(total), torch.zeros(2, device="cuda")
    for limit in (float(np.float32(want / 3)), float(np.float32(want * 3))):
        B.madd_grad_norm(B.GradList(gs), limit, out)
        norm, coef = out.double().tolist()
        assert abs(norm - want) <= (2.0 ** -24 + 2.0 ** -40) * want
        assert abs(coef - min(1.0, limit / want)) <= (2.0 ** -23 + 2.0 ** -40) * min(1.0, limit / want)

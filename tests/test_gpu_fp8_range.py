"""FP8 products at the ends of the scales' and results' ranges (GPU).  Operands are
small integers times powers of two whose sums fp32 holds exactly, so bits are
compared."""
import numpy as np
import pytest
import torch

import fp8_reference as R
from paper_2607_10611_amd import fp8
from test_gpu_fp8_matmul import integers

pytestmark = pytest.mark.gpu

# rows of 16, 32 and 64, tiles of 64, of 128 (few and many) and the largest; parts along k
SHAPES = [(1, 40, 256), (5, 300, 4096), (30, 200, 384), (60, 100, 512), (61, 9000, 384),
          (300, 260, 1280), (1300, 900, 512), (50, 7000, 768), (48, 500, 5632), (2050, 2060, 512)]


def scaled(m, v, e):
    """A BlockMatrix with E8M0 scales and its values, times 2^e."""
    codes = m.scales.cpu().numpy().astype(int) + e
    assert codes.min() >= 0 and codes.max() <= 254
    m.scales.copy_(torch.from_numpy(codes.astype(np.uint8)))
    return m, v * 2.0 ** e


def same(got, want):
    """got, fp32 or bf16, holds want's values, which fp32 holds, rounded once."""
    f = want.astype(np.float32)
    assert np.isinf(f).any() or np.array_equal(f.astype(np.float64), want)
    assert torch.equal(got.cpu(), torch.from_numpy(f).to(got.dtype))


@pytest.mark.parametrize("e", [-125, -60, 60, 125])
@pytest.mark.parametrize("shape", SHAPES)
def test_scales_that_cancel(shape, e):
    """Scales of 2^-127 to 2^127 whose products are of ordinary size."""
    m, n, k = shape
    rng = np.random.default_rng(m)
    (a, av), (b, bv) = integers(rng, m, k), integers(rng, n, k)
    (a, av), (b, bv) = scaled(a, av, e), scaled(b, bv, -e)
    for dtype in (torch.float32, torch.bfloat16):
        same(fp8.matmul(a, b, dtype), av @ bv.T)


@pytest.mark.parametrize("ea,eb", [(-72, -70), (-125, -15), (-10, -125), (50, 58), (125, -17)])
@pytest.mark.parametrize("shape", SHAPES)
def test_results_near_the_ends_of_fp32(shape, ea, eb):
    """Denormal results (multiples of 2^-146 and larger), and ones up to 2^127."""
    m, n, k = shape
    rng = np.random.default_rng(n)
    (a, av), (b, bv) = integers(rng, m, k), integers(rng, n, k)
    (a, av), (b, bv) = scaled(a, av, ea), scaled(b, bv, eb)
    same(fp8.matmul(a, b, torch.float32), av @ bv.T)


@pytest.mark.parametrize("shape", SHAPES)
def test_results_past_the_ends_of_fp32(shape):
    """One product a result: infinities of its sign past the largest value, zeros below
    half the smallest one."""
    m, n, k = shape
    rng = np.random.default_rng(k)
    for e, big in ((75, True), (-90, False)):
        (a, av), (b, bv) = integers(rng, m, k), integers(rng, n, k)
        a.codes[:, 1:] = 0
        a.codes[:, 0] = torch.from_numpy(np.where(rng.random(m) < 0.5, 0x38, 0xB8).astype(np.uint8))
        (a, _), (b, _) = scaled(a, av, e), scaled(b, bv, e)
        sign = (1.0 - 2.0 * (a.codes[:, :1].cpu() > 127)) * torch.from_numpy(bv[:, 0]).sign()
        want = torch.where(sign == 0, 0.0, sign * float("inf")) if big else 0.0 * sign
        got = fp8.matmul(a, b, torch.float32).cpu().double()
        assert torch.equal(got, want)


@pytest.mark.parametrize("e", [-120, -60, 60, 122])
@pytest.mark.parametrize("shape", SHAPES)
def test_fp16_scales_beside_large_and_small_rows(shape, e):
    """A block's sum times the row's scale alone may pass fp32's largest value where the
    result, small scales applied, does not."""
    m, n, k = shape
    rng = np.random.default_rng(m + k)
    (a, av), (b, bv) = integers(rng, m, k), integers(rng, n, k, "fp16")
    a, av = scaled(a, av, e)
    if e > 0:
        b.scales.mul_(2.0 ** -11)
        bv = bv * 2.0 ** -11
    for dtype in (torch.float32, torch.bfloat16):
        same(fp8.matmul(a, b, dtype), av @ bv.T)
    x = torch.from_numpy(av.astype(np.float32)).cuda()
    assert np.array_equal(R.values(av, "e4m3"), av)  # the quantizer keeps such blocks
    same(fp8.linear(x, b, torch.float32), av @ bv.T)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("m", [1, 20, 40, 300])
def test_linear_of_the_type_s_largest_values(m, fmt):
    """Rows of values near the largest of fp32 and bf16, by the format's largest codes
    and the smallest scale.  All terms are equal, 49 times a power of two, so that sums of
    256 of them are exact."""
    k, n = 256, 70
    top = R.FMAX[fmt]
    code = int(np.nonzero(R.decode(np.arange(128), fmt) == top)[0][0])
    w = fp8.BlockMatrix(torch.full((n, k), code, dtype=torch.uint8, device="cuda"),
                        torch.full((n, k // 128), 2.0 ** -24, dtype=torch.float16, device="cuda"),
                        fmt)
    x = torch.full((m, k), -448.0 * 2.0 ** 119, device="cuda")  # 2^127.8
    want = torch.full((m, n), -448.0 * 2.0 ** 119 * k * top * 2.0 ** -24, dtype=torch.float64)
    assert float(want.abs().max()) < 2.0 ** 128
    assert torch.equal(fp8.linear(x, w, torch.float32).cpu().double(), want)
    assert torch.equal(fp8.linear(x.bfloat16(), w).cpu().double(), want.bfloat16().double())

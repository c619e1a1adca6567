"""What the FP8 and AdamW entry points refuse, before any device work (CPU)."""
import ctypes

import pytest
import torch

import test_abi
from paper_2607_10611_amd import binding as B
from paper_2607_10611_amd import fp8

fake_addresses = test_abi.fake_addresses  # made-up device addresses: CPU only
X_, B_, SB_, Y_, WS_ = (0x1000000 * (k + 1) for k in range(5))
EINVAL, EUNSUPPORTED, EDEVICE = -1, -3, -4


def linear(m=50, n=70, k=256, x=X_, b=B_, sb=SB_, y=Y_, ws=WS_, wsb=None, ldx=None):
    """madd_linear_fp8 of bf16 values and E4M3 weights with FP16 scales, bf16 results."""
    lib = B.lib()
    wsb = lib.madd_linear_fp8_workspace(m, n, k) if wsb is None else wsb
    return lib.madd_linear_fp8(x, 1, k if ldx is None else ldx, b, 1, sb, 1, y, 1, n, m, n, k, ws,
                               wsb, None)


@fake_addresses
def test_linear_refuses_weights_in_its_workspace():
    """x's codes are written into the workspace, so no other operand may lie there."""
    need = B.lib().madd_linear_fp8_workspace(50, 70, 256)
    for bad in (dict(b=WS_), dict(b=WS_ + 16), dict(b=WS_ - 16), dict(b=WS_ + need - 16),
                dict(sb=WS_), dict(sb=WS_ + 64), dict(sb=WS_ - 2), dict(sb=WS_ + need - 2)):
        assert linear(**bad) == EINVAL, bad


def _adamw(sizes):
    """madd_adamw_step of bf16 weights, bf16 gradients and 8-bit states at made-up
    addresses, 2^42 bytes apart."""
    k = len(sizes)
    at = lambda j: ctypes.cast((ctypes.c_void_p * k)(  # noqa: E731
        *[((6 * i + j + 1) << 42) for i in range(k)]), ctypes.POINTER(ctypes.c_void_p))
    h = B._adamw_hp(dict(lr=1e-3, step=1))
    return B.lib().madd_adamw_step(k, at(0), 0, None, at(1), 1, at(2), at(3), at(4), 1,
                                   (ctypes.c_int64 * k)(*sizes), 0, ctypes.byref(h), None, None)


@fake_addresses
def test_adamw_refuses_a_tensor_that_no_launch_holds_before_the_first():
    """A tensor of more workgroups than a launch holds is refused before any other
    tensor of the list is stepped.  (Without a device a launch ends in MADD_EDEVICE.)"""
    most = (2 ** 24 - 1) * 2048
    assert _adamw([1000] * 60 + [most + 1]) == EUNSUPPORTED
    assert _adamw([most + 1]) == EUNSUPPORTED
    assert _adamw([most]) == EDEVICE and _adamw([1000]) == EDEVICE


@fake_addresses
def test_adamw_splits_lists_that_no_launch_holds():
    """Tensors that fit a launch each but not together take several launches."""
    half = 2 ** 23 * 2048
    assert _adamw([half, half, half]) == EDEVICE  # a launch was tried, none was refused


@fake_addresses
def test_linear_refuses_what_no_launch_holds_before_the_first():
    """Sizes that the product cannot take are refused before x is quantized.
    (Without a device a launch ends in MADD_EDEVICE.)"""
    far = {name: (j + 1) << 45 for j, name in enumerate(("x", "b", "sb", "y", "ws"))}
    assert linear(m=50, n=70, k=128 * 65536, **far) == EUNSUPPORTED
    assert linear(m=50, n=70, k=128 * 65535, **far) == EDEVICE
    for m in (17, 3000):
        assert linear(m=m, n=2 ** 31, k=128, **far) == EUNSUPPORTED, m
    assert linear(m=40, n=2 ** 31, k=128, **far) == EDEVICE  # 2^23 tiles of 64x256
    for m in (17, 40, 3000):
        assert linear(m=m, n=2 ** 20, k=128, **far) == EDEVICE, m


@fake_addresses
def test_matrices_past_the_end_of_memory_are_refused():
    """Row strides that 64-bit offsets cannot follow: the ranges of such matrices would
    wrap round in the checks for overlap."""
    lib, far = B.lib(), [(j + 1) << 45 for j in range(5)]
    rows, ld = 2 ** 31, 2 ** 40

    def matmul(ldc):
        return lib.madd_matmul_fp8(far[0], 1, far[1], far[2], 1, far[3], 0, far[4], 0, ldc, 0,
                                   rows, 70, 128, None, 0, None)

    def quantize(ldx):
        return lib.madd_quantize_fp8(far[0], 1, rows, 128, ldx, 1, far[1], far[2], None, None,
                                     None)

    assert matmul(ld) == EINVAL and quantize(ld) == EINVAL
    assert linear(m=3, n=70, k=128, ldx=2 ** 41) == EINVAL
    ws = lib.madd_linear_fp8_workspace(rows, 70, 128)
    assert linear(m=rows, n=70, k=128, x=far[0], b=far[1], sb=far[2], y=far[3], ws=far[4] << 4,
                  wsb=ws, ldx=ld) == EINVAL
    assert quantize(128) == EDEVICE


def _blocks(rows, cols, **kw):
    k = -(-cols // 128) * 128
    return fp8.BlockMatrix(torch.zeros(rows, k, dtype=torch.uint8),
                           torch.zeros(rows, k // 128, dtype=torch.uint8), "e4m3", cols=cols, **kw)


def test_lengths_that_differ_within_a_block_are_refused(monkeypatch):
    """Operands whose padded rows are as long but which count different numbers of
    columns: the product would silently take the padding of one for zeros of the other."""
    monkeypatch.setattr(B, "madd_matmul_fp8", lambda *a: pytest.fail("reached the kernel"))
    monkeypatch.setattr(B, "madd_linear_fp8", lambda *a: pytest.fail("reached the kernel"))
    monkeypatch.setattr(B, "madd_quantize_fp8", lambda *a: None)
    x = lambda *s: torch.zeros(*s)  # noqa: E731
    with pytest.raises(ValueError, match="columns"):
        fp8.matmul(_blocks(3, 100), _blocks(4, 128))
    with pytest.raises(ValueError, match="columns"):
        fp8.linear(x(3, 128), _blocks(4, 100))
    with pytest.raises(ValueError, match="columns"):
        fp8.linear_forward(x(3, 100), _blocks(4, 128))
    xt, copy = _blocks(256, 40), x(70, 256)  # 40 rows of 256 values; 70 outputs
    for dy in (x(40, 71), x(40, 128), x(39, 70), x(128, 70)):
        with pytest.raises(ValueError, match="columns"):
            fp8.linear_backward(dy, xt, copy, need_dx=dy.shape[1] != 70)


def test_columns_that_a_block_matrix_does_not_have():
    for cols in (0, -1, 128, 257):
        with pytest.raises(ValueError, match="cols"):
            fp8.BlockMatrix(torch.zeros(3, 256, dtype=torch.uint8),
                            torch.zeros(3, 2, dtype=torch.uint8), "e4m3", cols=cols)
    assert _blocks(3, 129).shape == (3, 129) and _blocks(3, 256).shape == (3, 256)
    assert _blocks(3, 0).shape == (3, 0)


def test_scales_and_codes_of_other_formats_are_refused():
    """Types of one or two bytes that hold other values: their bits would be read as
    E8M0, FP16 or the named FP8 format."""
    codes, u8 = torch.zeros(3, 256, dtype=torch.uint8), torch.uint8
    zeros = lambda dtype: torch.zeros(3, 2, dtype=dtype)  # noqa: E731
    for good in (u8, torch.float8_e8m0fnu, torch.float16, torch.int16, torch.uint16):
        fp8.BlockMatrix(codes, zeros(good), "e4m3")
    for bad in (torch.bfloat16, torch.float8_e4m3fn, torch.float8_e5m2, torch.bool, torch.float32,
                torch.int32):
        with pytest.raises(TypeError):
            fp8.BlockMatrix(codes, zeros(bad), "e4m3")
    for bad in (torch.float8_e4m3fnuz, torch.float8_e5m2fnuz, torch.float8_e8m0fnu, torch.bool,
                torch.int16):
        with pytest.raises(TypeError):
            fp8.BlockMatrix(codes.to(bad), zeros(u8), "e4m3")
    assert fp8.BlockMatrix(codes.view(torch.int8), zeros(u8), "e5m2").fmt == "e5m2"


def test_the_binding_refuses_codes_of_other_formats(monkeypatch):
    monkeypatch.setattr(B, "_need", lambda *a: None)
    monkeypatch.setattr(B, "_need_rows", lambda what, t, rows, cols: cols)
    monkeypatch.setattr(B, "lib", lambda: pytest.fail("reached the library"))
    u8 = lambda *s: torch.zeros(*s, dtype=torch.uint8)  # noqa: E731
    c, x, s = torch.zeros(3, 4), torch.zeros(3, 128), u8(4, 1)
    for bad in (torch.zeros(4, 128), u8(4, 128).view(torch.float8_e5m2), u8(4, 128).bool()):
        with pytest.raises(TypeError):
            B.madd_matmul_fp8(u8(3, 128), "e4m3", u8(3, 1), bad, "e4m3", s, c)
        with pytest.raises(TypeError):
            B.madd_matmul_fp8(bad[:3], "e4m3", u8(3, 1), u8(4, 128), "e4m3", s, c)
        with pytest.raises(TypeError):
            B.madd_linear_fp8(x, bad, "e4m3", s, c)
    for bad in (s.view(torch.float8_e4m3fn), s.to(torch.bfloat16)):
        with pytest.raises(TypeError):
            B.madd_matmul_fp8(u8(3, 128), "e4m3", u8(3, 1), u8(4, 128), "e4m3", bad, c)
        with pytest.raises(TypeError):
            B.madd_linear_fp8(x, u8(4, 128), "e4m3", bad, c)


def test_scales_of_another_shape_are_refused():
    """As many scales in another order, such as the transposed ones."""
    codes = torch.zeros(4, 256, dtype=torch.uint8)
    make = lambda *s: fp8.BlockMatrix(codes, torch.zeros(*s, dtype=torch.uint8), "e4m3")  # noqa: E731
    for bad in ((2, 4), (1, 8), (8, 1), (4, 2, 1), (2, 2, 2)):
        with pytest.raises(ValueError, match="scales"):
            make(*bad)
    assert make(4, 2).scales.shape == make(8).scales.shape == (4, 2)

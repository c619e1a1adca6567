"""What the FP8 and AdamW entry points refuse, before any device work (CPU)."""
import test_abi
from paper_2607_10611_amd import binding as B

fake_addresses = test_abi.fake_addresses  # made-up device addresses: CPU only
X_, B_, SB_, Y_, WS_ = (0x1000000 * (k + 1) for k in range(5))
EINVAL, EUNSUPPORTED = -1, -3


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

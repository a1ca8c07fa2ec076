"""Sizes next to 2^31 at the entry points on 4-bit floating point and on experts: what cannot be rounded up to whole blocks in 32 bits is
refused, not wrapped round (no GPU: a call that is not refused gets as far as a launch, which fails here)."""
import pytest

import test_f4_abi as abi

TOP = 0x7FFFFFFF
SHAPE = 2


@pytest.fixture(scope="module")
def B():
    from paper_1706_09453_b200 import build, binding
    build.build()
    return binding


@pytest.mark.parametrize("n", [TOP, TOP - 1, TOP - 7, TOP - 1023, TOP - 2047, TOP - 4095])
def test_lengths_that_do_not_round_up(B, n):
    much = 1 << 62
    for name, good, bad in (
            ("bnn_f4_quantize", abi.QUANTIZE, dict(rows=n, src_rows=n, K=32, scale_bytes=much)),
            ("bnn_f4_dequantize", abi.DEQUANTIZE, dict(rows=n, K=32, scale_bytes=much)),
            ("bnn_f4_gemm", abi.GEMM, dict(N=n, ldy=n, w_bytes=much)),
            ("bnn_f4_gemm_grouped", abi.GROUPED, dict(M=n, N=1, K=32, ldy=1, groups=1024, a_bytes=much, w_bytes=much)),
            ("bnn_route_experts", abi.ROUTE, dict(T=n, E=1, k=1, bytes=much)),
            ("bnn_combine_experts", abi.COMBINE, dict(N=n, ldz=n, ldy=n)),
            ("bnn_combine_experts", abi.COMBINE, dict(N=n, ldz=n, ldy=n, z_dtype=2, y_dtype=2))):
        if name == "bnn_f4_gemm" and n < TOP - 256:
            continue                        # (rounded up to 256 units)
        abi.refused(B, name, good, SHAPE, **bad)
    assert B.bnn_route_workspace_bytes(n, 1) == 0

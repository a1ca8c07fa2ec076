"""Packed bits asked for together with an activation that does not write them are refused, not handed back as they were (no GPU)."""
import ctypes as C

import pytest

import test_f4_abi as abi

UNSUPPORTED = 4


@pytest.fixture(scope="module")
def B():
    from paper_1706_09453_b200 import build, binding
    build.build()
    return binding


@pytest.mark.parametrize("act", ["ACT_NONE", "ACT_HARDTANH", "ACT_SIGMOID"])
def test_bits_without_the_sign_activation(B, act):
    e = B.Epilogue()
    e.act, e.out_bits, e.ldob = getattr(B, act), abi.FAKE, 8
    abi.refused(B, "bnn_f4_gemm", abi.GEMM, UNSUPPORTED, epi=C.byref(e))
    abi.refused(B, "bnn_f4_gemm_grouped", abi.GROUPED, UNSUPPORTED, epi=C.byref(e))

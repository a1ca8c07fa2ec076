"""Refusals of the operators on 4-bit floating point and on experts: every bad argument is answered before a launch (no GPU)."""
import ctypes as C

import numpy as np
import pytest

import f4_reference as ref

FAKE = 0x100000   # aligned "pointer", never dereferenced on the host


@pytest.fixture(scope="module")
def B():
    from paper_1706_09453_b200 import build, binding
    build.build()
    return binding


QUANTIZE = dict(X=FAKE, dtype=0, src_rows=300, K=100, ldx=100, source=None, offsets=None, groups=1, rows=300, fmt=0, exponent=0,
                codes=FAKE, ldc=64, scales=FAKE, scale_bytes=3 * 512, stream=None)
DEQUANTIZE = dict(codes=FAKE, ldc=64, scales=FAKE, scale_bytes=3 * 512, offsets=None, groups=1, rows=300, K=100, fmt=0, exponent=0,
                  Y=FAKE, dtype=0, ldy=100, stream=None)
GEMM = dict(A=FAKE, lda=64, a_scales=FAKE, a_bytes=3 * 512, W=FAKE, ldw=64, w_scales=FAKE, w_bytes=2 * 512, M=300, N=200, K=100, fmt=0,
            exponent=0, Y=FAKE, dtype=0, ldy=200, epi=None, stream=None)
GROUPED = dict(A=FAKE, lda=64, a_scales=FAKE, a_bytes=6 * 512, offsets=FAKE, groups=4, W=FAKE, ldw=64, w_scales=FAKE, w_bytes=10 * 512,
               M=300, N=200, K=100, fmt=0, exponent=0, Y=FAKE, dtype=0, ldy=200, epi=None, stream=None)
ROUTE = dict(logits=FAKE, dtype=0, T=10, E=64, ld=64, k=8, mode=0, index=FAKE, weight=FAKE, offsets=FAKE, slot=FAKE, source=FAKE,
             workspace=FAKE, bytes=4, stream=None)
COMBINE = dict(Z=FAKE, z_dtype=0, rows=80, ldz=64, slot=FAKE, weight=FAKE, T=10, k=8, N=64, Y=FAKE, y_dtype=0, ldy=64, stream=None)

NULL, SHAPE, ALIGN, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4, 5
BIG = (1 << 24) + 1


def refused(B, name, good, status, **bad):
    assert B.raw_call(name, *{**good, **bad}.values()) == status, (name, bad)


QUANTIZE_BAD = [
    (dict(X=None), NULL), (dict(codes=None), NULL), (dict(scales=None), NULL), (dict(fmt=2), UNSUPPORTED), (dict(fmt=-1), UNSUPPORTED),
    (dict(dtype=3), UNSUPPORTED), (dict(rows=0), SHAPE), (dict(K=0), SHAPE), (dict(K=BIG, ldx=BIG), SHAPE), (dict(ldx=99), SHAPE),
    (dict(src_rows=0), SHAPE), (dict(src_rows=299), SHAPE), (dict(groups=0), SHAPE), (dict(groups=2), SHAPE), (dict(offsets=FAKE, groups=1025), SHAPE),
    (dict(exponent=65), SHAPE), (dict(exponent=-65), SHAPE), (dict(ldc=48), SHAPE), (dict(ldc=72), ALIGN), (dict(codes=FAKE + 8), ALIGN),
    (dict(scales=FAKE + 4), ALIGN), (dict(X=FAKE + 2), ALIGN), (dict(source=FAKE + 1), ALIGN), (dict(offsets=FAKE + 2, groups=1), ALIGN),
    (dict(scale_bytes=3 * 512 - 1), WORKSPACE), (dict(fmt=1), WORKSPACE), (dict(offsets=FAKE, groups=2), WORKSPACE)]


@pytest.mark.parametrize("bad,status", QUANTIZE_BAD)
def test_quantize(B, bad, status):
    refused(B, "bnn_f4_quantize", QUANTIZE, status, **bad)


DEQUANTIZE_BAD = [
    (dict(Y=None), NULL), (dict(codes=None), NULL), (dict(scales=None), NULL), (dict(fmt=7), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED),
    (dict(rows=0), SHAPE), (dict(K=0), SHAPE), (dict(ldy=99), SHAPE), (dict(ldc=48), SHAPE), (dict(ldc=65), ALIGN), (dict(Y=FAKE + 2), ALIGN),
    (dict(exponent=100), SHAPE), (dict(groups=3), SHAPE), (dict(scale_bytes=0), WORKSPACE)]


@pytest.mark.parametrize("bad,status", DEQUANTIZE_BAD)
def test_dequantize(B, bad, status):
    refused(B, "bnn_f4_dequantize", DEQUANTIZE, status, **bad)


PRODUCT = [
    (dict(A=None), NULL), (dict(W=None), NULL), (dict(a_scales=None), NULL), (dict(w_scales=None), NULL), (dict(Y=None), NULL),
    (dict(fmt=2), UNSUPPORTED), (dict(dtype=3), UNSUPPORTED), (dict(M=0), SHAPE), (dict(N=0), SHAPE), (dict(K=0), SHAPE), (dict(K=BIG), SHAPE),
    (dict(lda=48), SHAPE), (dict(ldw=48), SHAPE), (dict(lda=65), ALIGN), (dict(ldw=72), ALIGN), (dict(A=FAKE + 1), ALIGN), (dict(W=FAKE + 8), ALIGN),
    (dict(a_scales=FAKE + 8), ALIGN), (dict(w_scales=FAKE + 8), ALIGN), (dict(ldy=199), SHAPE), (dict(Y=FAKE + 2), ALIGN), (dict(exponent=65), SHAPE),
    (dict(a_bytes=512), WORKSPACE), (dict(w_bytes=512), WORKSPACE), (dict(fmt=1), WORKSPACE)]


@pytest.mark.parametrize("bad,status", PRODUCT)
def test_product(B, bad, status):
    refused(B, "bnn_f4_gemm", GEMM, status, **bad)


GROUPED_BAD = PRODUCT + [(dict(offsets=None), NULL), (dict(offsets=FAKE + 1), ALIGN), (dict(groups=0), SHAPE),
                                                  (dict(groups=1025), SHAPE), (dict(groups=1024, N=1 << 21), SHAPE)]


@pytest.mark.parametrize("bad,status", GROUPED_BAD)
def test_grouped_product(B, bad, status):
    refused(B, "bnn_f4_gemm_grouped", GROUPED, status, **bad)


@pytest.mark.parametrize("fields,bad,status", [
    (dict(act=7), {}, UNSUPPORTED), (dict(scale=FAKE + 1), {}, ALIGN), (dict(shift=FAKE + 2), {}, ALIGN),
    (dict(act=1, out_bits=FAKE, ldob=8), {}, UNSUPPORTED),                       # bits and Y
    (dict(act=1), dict(Y=None), NULL), (dict(act=1, out_bits=FAKE, ldob=6), dict(Y=None), SHAPE),
    (dict(act=1, out_bits=FAKE, ldob=9), dict(Y=None), ALIGN), (dict(act=1, out_bits=FAKE + 4, ldob=8), dict(Y=None), ALIGN),
    (dict(act=1, out_bits=FAKE, ldob=8, sign_mode=2), dict(Y=None), UNSUPPORTED), (dict(act=2), dict(Y=None), NULL)])
def test_epilogues(B, fields, bad, status):
    e = B.Epilogue()
    for n, v in fields.items():
        setattr(e, n, v)
    refused(B, "bnn_f4_gemm", GEMM, status, epi=C.byref(e), **bad)
    refused(B, "bnn_f4_gemm_grouped", GROUPED, status, epi=C.byref(e), **bad)


ROUTE_BAD = [
    *[({n: None}, NULL) for n in ("logits", "index", "weight", "offsets", "slot", "source")], (dict(workspace=None), WORKSPACE),
    (dict(bytes=3), WORKSPACE), (dict(T=1000), WORKSPACE), (dict(dtype=3), UNSUPPORTED), (dict(mode=2), UNSUPPORTED), (dict(T=0), SHAPE),
    (dict(E=0), SHAPE), (dict(E=1025, ld=1025), SHAPE), (dict(ld=63), SHAPE), (dict(k=0), SHAPE), (dict(k=33), SHAPE), (dict(k=5, E=4), SHAPE),
    (dict(T=1 << 28, k=8), SHAPE), (dict(logits=FAKE + 2), ALIGN), (dict(weight=FAKE + 2), ALIGN), (dict(slot=FAKE + 1), ALIGN)]


@pytest.mark.parametrize("bad,status", ROUTE_BAD)
def test_router(B, bad, status):
    refused(B, "bnn_route_experts", ROUTE, status, **bad)


COMBINE_BAD = [
    *[({n: None}, NULL) for n in ("Z", "slot", "weight", "Y")], (dict(z_dtype=3), UNSUPPORTED), (dict(y_dtype=-1), UNSUPPORTED), (dict(rows=0), SHAPE),
    (dict(T=0), SHAPE), (dict(k=0), SHAPE), (dict(k=33), SHAPE), (dict(N=0), SHAPE), (dict(ldz=63), SHAPE), (dict(ldy=63), SHAPE),
    (dict(Z=FAKE + 2), ALIGN), (dict(y_dtype=2, Y=FAKE + 1), ALIGN), (dict(slot=FAKE + 2), ALIGN), (dict(weight=FAKE + 2), ALIGN)]


@pytest.mark.parametrize("bad,status", COMBINE_BAD)
def test_weighted_sum(B, bad, status):
    refused(B, "bnn_combine_experts", COMBINE, status, **bad)


def test_sizes(B):
    assert [B.bnn_f4_pitch(k) for k in (0, 1, 32, 33, 100, BIG)] == [0, 16, 16, 32, 64, 0]
    for fmt in (0, 1):
        for rows, groups, K in ((1, 1, 1), (300, 1, 100), (300, 4, 1000), (1 << 20, 1024, 4096)):
            assert B.bnn_f4_scale_bytes(fmt, rows, K, groups) == (rows // 128 + groups) * ref.scale_tiles(fmt, K) * 512
    assert B.bnn_f4_scale_bytes(2, 1, 1) == B.bnn_f4_scale_bytes(0, 0, 1) == B.bnn_f4_scale_bytes(0, 1, 0) == B.bnn_f4_scale_bytes(0, 1, 1, 1025) == 0
    assert B.bnn_route_workspace_bytes(0, 4) == B.bnn_route_workspace_bytes(4, 1025) == 0
    assert 0 < B.bnn_route_workspace_bytes(1, 1) <= B.bnn_route_workspace_bytes(1 << 20, 1024)


def test_row_tiles_of_groups_do_not_meet():
    """Tile offsets[g] / 128 + g: behind the tiles of the groups before, and inside rows / 128 + groups tiles."""
    rng = np.random.default_rng(0)
    for _ in range(2000):
        G = int(rng.integers(1, 20))
        n = rng.choice([0, 1, 5, 127, 128, 129, 256, 300], G)
        off = np.concatenate([[rng.integers(0, 3)], n]).cumsum()
        start = off[:-1] // 128 + np.arange(G)
        end = start + -(-n // 128)
        assert (start[1:] >= end[:-1]).all() and end[-1] <= off[-1] // 128 + G


def test_the_reference_rounds_to_the_nearest():
    """Against a search over all codes in exact fractions."""
    from fractions import Fraction as F
    rng = np.random.default_rng(1)
    for fmt in (ref.MX, ref.NV):
        x = (rng.normal(0, 1, (4, 64)) * 2.0 ** rng.integers(-3, 4, (4, 64))).astype(np.float16).astype(np.float64)
        code, byte = ref.quantize(x, fmt)
        v, n = ref.values(code, byte, fmt, 64), ref.BLOCK[fmt]
        for r in range(4):
            for k in range(64):
                s = F(2.0 ** (float(byte[r, k // n]) - 127)) if fmt == ref.MX else F(float(ref.E4M3[byte[r, k // n]]))
                best = min(abs(min(abs(F(float(x[r, k]))), 6 * s) - F(float(g)) * s) for g in ref.E2M1)
                assert abs(min(abs(F(float(x[r, k]))), 6 * s) - abs(F(float(v[r, k])))) == best


@pytest.mark.parametrize("number,name,good,bads", [
    (0, "bnn_f4_quantize", QUANTIZE, QUANTIZE_BAD), (1, "bnn_f4_dequantize", DEQUANTIZE, DEQUANTIZE_BAD), (2, "bnn_f4_gemm", GEMM, PRODUCT),
    (3, "bnn_f4_gemm_grouped", GROUPED, GROUPED_BAD), (4, "bnn_route_experts", ROUTE, ROUTE_BAD), (5, "bnn_combine_experts", COMBINE, COMBINE_BAD)])
def test_arguments_as_words(B, number, name, good, bads):
    """bnn_call_words: the refusals of the calls, and its own."""
    import struct

    def words(call, values):
        values = [v or 0 for v in values]
        return B.lib()["bnn_call_words"](call, struct.pack("%dq" % len(values), *values), len(values))
    for bad, status in bads:
        assert words(number, {**good, **bad}.values()) == status, bad
    values = list(good.values())
    assert words(number, values[:-1]) == words(number, values + [0]) == SHAPE
    ints = [i for i, t in enumerate(getattr(B.lib(), name).argtypes) if t is C.c_int]
    assert len(ints) >= 6
    for at in ints:
        for v in (1 << 31, -(1 << 31) - 1, (1 << 32) + values[at]):      # would be another int if it were cut
            assert words(number, values[:at] + [v] + values[at + 1:]) == SHAPE, (at, v)
    assert words(6, values) == words(-1, values) == UNSUPPORTED
    assert B.lib()["bnn_call_words"](number, None, len(values)) == NULL


def test_the_bindings_hand_over_as_many_words_as_the_calls_have_arguments(B):
    for c in (B._f4_quantize, B._f4_dequantize, B._f4_gemm, B._f4_gemm_grouped, B._route_experts, B._combine_experts):
        assert c.n == len(getattr(B.lib(), c.name).argtypes), c.name

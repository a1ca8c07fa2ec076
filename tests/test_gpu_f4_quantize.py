"""Quantisation to 4-bit floating point and back: codes and scales bit for bit against the definition in 64 bits, over types,
odd widths, gathered rows, rows in groups, and values on and next to the borders between codes."""
import numpy as np
import pytest

import f4_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available()
    from paper_1706_09453_b200 import build, binding
    build.build()
    return torch, binding


def dtype_of(torch, name):
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def run_quantize(torch, B, x, fmt, rows=None, source=None, offsets=None, exponent=0, pad=0):
    """Codes and scales as numpy, around which nothing may have been written."""
    K, rows = x.shape[1], x.shape[0] if rows is None else rows
    groups = 1 if offsets is None else len(offsets) - 1
    ld = B.bnn_f4_pitch(K) + 16 * pad
    codes = torch.full((rows + 1, ld), 0xA5, dtype=torch.uint8, device=DEV)
    n = B.bnn_f4_scale_bytes(fmt, rows, K, groups)
    scales = torch.full((n + 64,), 0xA5, dtype=torch.uint8, device=DEV)
    dev = lambda a: None if a is None else torch.as_tensor(np.asarray(a, dtype=np.int32), device=DEV)
    B.bnn_f4_quantize(x, codes[:rows], scales[:n], fmt, source=dev(source), offsets=dev(offsets), exponent=exponent)
    c, s = codes.cpu().numpy(), scales.cpu().numpy()
    assert (c[rows] == 0xA5).all() and (c[:, B.bnn_f4_pitch(K):] == 0xA5).all() and (s[n:] == 0xA5).all()
    return c[:rows, :B.bnn_f4_pitch(K)], s[:n]


def check(torch, B, x, fmt, **kw):
    got_c, got_s = run_quantize(torch, B, x, fmt, **kw)
    xs = x.float().cpu().numpy().astype(np.float64)
    source, offsets = kw.get("source"), kw.get("offsets")
    if source is not None:
        src = np.asarray(source)
        ok = (src >= 0) & (src < xs.shape[0])
        xs = np.where(ok[:, None], xs[np.where(ok, src, 0)], 0.0)
    code, byte = ref.quantize(xs, fmt, kw.get("exponent", 0))
    want_c = ref.pack(code)
    groups = 1 if offsets is None else len(offsets) - 1
    want_s = ref.store_scales(byte, offsets, groups, 0xA5)
    if offsets is not None:
        want_c[ref.places(len(want_c), offsets) < 0] = 0xA5
    np.testing.assert_array_equal(got_s, want_s)
    np.testing.assert_array_equal(got_c, want_c)


def test_sizes_of_the_stored_form(env):
    _, B = env
    for K in (1, 31, 32, 33, 64, 127, 1000, 4096):
        assert B.bnn_f4_pitch(K) == ref.pitch(K)
        for fmt in (ref.MX, ref.NV):
            for rows, groups in ((1, 1), (127, 1), (128, 3), (1000, 64)):
                assert B.bnn_f4_scale_bytes(fmt, rows, K, groups) == (rows // 128 + groups) * ref.scale_tiles(fmt, K) * 512


@pytest.mark.parametrize("fmt", [ref.MX, ref.NV])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,K", [(1, 1), (1, 2048), (3, 31), (10, 440), (130, 33), (257, 64), (5, 1000), (2, 4097), (129, 2304), (900, 1024)])
def test_shapes(env, fmt, dtype, rows, K):
    torch, B = env
    g = torch.Generator(device=DEV)
    g.manual_seed(rows * 7 + K)
    x = (torch.randn((rows, K), generator=g, device=DEV) * torch.exp2(torch.randint(-6, 7, (rows, K), generator=g, device=DEV).float())).to(dtype_of(torch, dtype))
    check(torch, B, x, fmt, pad=rows % 2)
    # rows that start anywhere
    wide = torch.zeros((rows, K + 3), dtype=x.dtype, device=DEV)
    wide[:, 1:K + 1] = x
    check(torch, B, wide[:, 1:K + 1], fmt, exponent=3)


@pytest.mark.parametrize("fmt", [ref.MX, ref.NV])
def test_gathered_rows_in_groups(env, fmt):
    torch, B = env
    rng = np.random.default_rng(5)
    x = torch.as_tensor(rng.normal(0, 1, (37, 200)).astype(np.float32), device=DEV)
    for offsets in ([0, 0, 5, 5, 140, 269, 300], [0, 300], [4, 10, 10, 297], [0] * 40 + [300], [0] * 6, sorted(rng.integers(0, 301, 1025))):
        source = rng.integers(0, 37, 300)
        source[[3, 77]] = -1, 37            # outside X: rows of zeros
        check(torch, B, x, fmt, rows=300, source=source, offsets=offsets)


@pytest.mark.parametrize("fmt", [ref.MX, ref.NV])
def test_offsets_that_make_no_sense_stay_inside(env, fmt):
    torch, B = env
    x = torch.ones((50, 64), device=DEV)
    for offsets in ([50, 20, 0], [-5, 10, 1 << 30], [7, -1, 3, 50], [1 << 30, 1 << 30]):
        run_quantize(torch, B, x, fmt, offsets=offsets)


@pytest.mark.parametrize("fmt", [ref.MX, ref.NV])
def test_borders_between_codes(env, fmt):
    """Largest element of a block fixed, the others on the borders between two codes, one fp32 step off, and on the codes."""
    torch, B = env
    border = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0])
    rows = []
    scales = 2.0 ** np.arange(-100, 100, 7) if fmt == ref.MX else ref.E4M3[[1, 2, 3, 5, 7, 8, 9, 13, 20, 33, 56, 57, 63, 80, 101, 126]]
    n = ref.BLOCK[fmt]
    for s in scales:
        for top in ((6.0, 4.0, 7.99) if fmt == ref.MX else (6.0,)):
            for step in (0, 1, -1):
                v = (border * s).astype(np.float32)
                v = np.nextafter(v, np.float32(np.inf if step > 0 else -np.inf)) if step else v
                v = np.where(np.abs(v) > top * s, 0.0, v)
                row = np.zeros(n, dtype=np.float32)
                row[0] = top * s
                row[1:1 + len(v)] = np.where(np.arange(len(v)) % 2, -v, v)
                rows.append(row)
    check(torch, B, torch.as_tensor(np.array(rows, dtype=np.float32), device=DEV), fmt)
    # maxima on and next to the borders between two e4m3 scales, and to powers of two
    m = ref.E4M3[:-1] + np.diff(ref.E4M3) / 2 if fmt == ref.NV else 2.0 ** np.arange(-126, 127) / 6
    top = (m * 6).astype(np.float32)
    rows = []
    for v in (top, np.nextafter(top, np.float32(np.inf)), np.nextafter(top, np.float32(0))):
        r = np.zeros((len(v), n), dtype=np.float32)
        r[:, 3], r[:, 4] = v, -v / 3
        rows.append(r)
    check(torch, B, torch.as_tensor(np.concatenate(rows), device=DEV), fmt)


@pytest.mark.parametrize("fmt", [ref.MX, ref.NV])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
def test_values_without_a_place(env, fmt, dtype):
    """Zeros of both signs, subnormal and huge numbers, infinities and NaNs, in whole and in cut blocks."""
    torch, B = env
    dt = dtype_of(torch, dtype)
    fi = torch.finfo(dt)
    x = torch.randn((12, 75), device=DEV)
    x[0] = 0.0
    x[1] = -0.0
    x = x.to(dt)
    x[2] = fi.smallest_normal / 4
    x[3] = fi.max
    x[4, 40], x[5, 70], x[6, 3], x[7, 74] = float("inf"), float("-inf"), float("nan"), float("nan")
    x[8] = -fi.max
    x[9, ::2] = 0.0
    x[10] = fi.tiny
    check(torch, B, x, fmt)
    if dtype == "f32":
        check(torch, B, x, fmt, exponent=64)
        check(torch, B, x, fmt, exponent=-64)


@pytest.mark.parametrize("fmt", [ref.MX, ref.NV])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,K", [(1, 1), (3, 440), (130, 33), (300, 1000), (1, 4097), (600, 2048)])
def test_values_back(env, fmt, dtype, rows, K):
    torch, B = env
    rng = np.random.default_rng(rows + K)
    dt = dtype_of(torch, dtype)
    code, byte = ref.random_stored(rng, rows, K, fmt)
    offsets = None if rows < 5 else np.array([0, 0, 3, rows // 2, rows - 1])
    groups = 1 if offsets is None else 4
    if rows >= 5:   # a scale that is NaN
        byte[1, 0] = 255 if fmt == ref.MX else 127
    codes = torch.as_tensor(ref.pack(code), device=DEV)
    scales = torch.as_tensor(ref.store_scales(byte, offsets, groups, 0xA5), device=DEV)
    off = None if offsets is None else torch.as_tensor(offsets.astype(np.int32), device=DEV)
    for cols, exponent in ((K, 0), (K + 5, -2)):
        y = torch.full((rows, cols), 7.0, dtype=dt, device=DEV)
        B.bnn_f4_dequantize(codes, scales, y[:, :K], fmt, offsets=off, exponent=exponent)
        # a code times a scale has at most six significant bits and stays far from the types' limits: no rounding
        want = ref.values(code, byte, fmt, K) * 2.0 ** exponent
        want[ref.places(rows, offsets) < 0] = 7.0
        got = y.double().cpu().numpy()
        np.testing.assert_array_equal(got[:, :K], want)
        assert (got[:, K:] == 7.0).all()


def test_rows_further_apart_than_32_bits_hold(env):
    torch, B = env
    far, K = 1 << 30, 300
    x = torch.randn((3, K), device=DEV).to(torch.bfloat16)
    apart = torch.empty((2 * far + K,), dtype=torch.bfloat16, device=DEV).as_strided((3, K), (far, 1))
    apart.copy_(x)
    check(torch, B, apart, ref.NV)
    codes = torch.empty((2 * far + 4096,), dtype=torch.uint8, device=DEV).as_strided((3, B.bnn_f4_pitch(K)), (far, 1))
    near, scales = torch.empty((3, B.bnn_f4_pitch(K)), dtype=torch.uint8, device=DEV), torch.empty((B.bnn_f4_scale_bytes(ref.NV, 3, K),), dtype=torch.uint8, device=DEV)
    B.bnn_f4_quantize(x, codes, scales, ref.NV)
    B.bnn_f4_quantize(x, near, scales, ref.NV)
    assert torch.equal(codes, near)
    y = torch.empty((3, K), dtype=torch.bfloat16, device=DEV)
    B.bnn_f4_dequantize(codes, scales, apart, ref.NV)
    B.bnn_f4_dequantize(near, scales, y, ref.NV)
    assert torch.equal(apart, y)


@pytest.mark.parametrize("fmt", [ref.MX, ref.NV])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("exponent", [0, -64, 64])
def test_every_scale_back(env, fmt, dtype, exponent):
    """All codes with all scale bytes; what lies below the type's smallest normal number is rounded to its subnormal ones."""
    torch, B = env
    K, dt = 128, dtype_of(torch, dtype)
    code = np.tile(np.arange(16, dtype=np.uint8), (256 if fmt == ref.MX else 128, K // 16))
    rows = code.shape[0]
    byte = np.tile(np.arange(rows, dtype=np.uint8)[:, None], (1, 4 * ref.scale_tiles(fmt, K)))
    y = torch.empty((rows, K), dtype=dt, device=DEV)
    B.bnn_f4_dequantize(torch.as_tensor(ref.pack(code), device=DEV), torch.as_tensor(ref.store_scales(byte, None, 1), device=DEV), y, fmt, exponent=exponent)
    want = torch.as_tensor(ref.values(code, byte, fmt, K) * 2.0 ** exponent).to(dt).double().numpy()
    np.testing.assert_array_equal(y.double().cpu().numpy(), want)

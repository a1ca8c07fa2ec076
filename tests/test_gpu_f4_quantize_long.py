"""Quantisation and values back in the forms that many rows take, a warp to 1024 elements of a row: from 37888 segments of 256 elements on, four or
more to a row.  Rows on 32-byte boundaries are read in 32-byte pieces where a whole segment exists, others as in the small form.  Bit for bit against the
definition in 64 bits; the rows are a few hundred different ones in random order, so that this takes no longer than for those."""
import numpy as np
import pytest

import f4_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SIZES = [(8000, 1200), (4800, 2056), (9500, 1024), (2400, 4097)]


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available()
    from paper_1706_09453_b200 import build, binding
    build.build()
    return torch, binding


def dtype_of(torch, name):
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


def test_sizes_are_long():
    assert all(rows * -(-K // 256) >= 37888 and K >= 1024 for rows, K in SIZES)


def some_rows(torch, dtype, n, K, seed):
    """Ordinary rows of many magnitudes, and rows with zeros of both signs, subnormal and huge numbers, infinities and NaNs."""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    fi = torch.finfo(dtype)
    x = torch.randn((n, K), generator=g, device=DEV) * torch.exp2(torch.randint(-6, 7, (n, K), generator=g, device=DEV).float())
    x = x.to(dtype)
    x[0], x[1], x[2], x[3], x[4] = 0.0, -0.0, fi.smallest_normal / 4, fi.max, -fi.max
    x[5, ::2] = 0.0
    x[6, 1::3] = -0.0
    for r, v in enumerate((float("inf"), float("-inf"), float("nan"), -float("nan"))):
        for c in (0, 17, 511, 513, 1023, K - 1):       # either half of a word of two, of a lane's pieces and of a segment
            x[7 + 6 * r + (0, 17, 511, 513, 1023, K - 1).index(c), c] = v
    return x


def layouts(torch, x):
    """The same matrix with rows on 32-byte boundaries, on 16-byte ones, and anywhere."""
    rows, K = x.shape
    to32, to16 = 32 // x.element_size(), 16 // x.element_size()
    ld = -(-K // to32) * to32
    for first, pitch in ((0, ld), (0, ld + to16), (to16, ld + to32), (1, ld + 3)):
        wide = torch.full((rows, pitch + first), 3.0, dtype=x.dtype, device=DEV)
        wide[:, first:first + K] = x
        yield wide[:, first:first + K]


def run(torch, B, x, fmt, rows, **kw):
    """Codes and scales, around which nothing may have been written."""
    K = x.shape[1]
    wide = B.bnn_f4_pitch(K)
    groups = 1 if kw.get("offsets") is None else len(kw["offsets"]) - 1
    n = B.bnn_f4_scale_bytes(fmt, rows, K, groups)
    codes = torch.full((rows + 1, wide + 32), 0xA5, dtype=torch.uint8, device=DEV)
    scales = torch.full((n + 64,), 0xA5, dtype=torch.uint8, device=DEV)
    B.bnn_f4_quantize(x, codes[:rows], scales[:n], fmt, **kw)
    assert (codes[rows] == 0xA5).all() and (codes[:, wide:] == 0xA5).all() and (scales[n:] == 0xA5).all()
    return codes[:rows, :wide].cpu().numpy(), scales[:n].cpu().numpy()


@pytest.mark.parametrize("fmt", [ref.MX, ref.NV])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,K", SIZES)
def test_quantize(env, fmt, dtype, rows, K):
    torch, B = env
    few = some_rows(torch, dtype_of(torch, dtype), 200, K, rows + K)
    rng = np.random.default_rng(K)
    at = rng.integers(0, 200, rows)
    at[:200] = np.arange(200)
    x = few[torch.as_tensor(at, device=DEV)]
    plain = few.float().cpu().numpy().astype(np.float64)
    for exponent in (0, 5, -64) if dtype == "f32" else (0, -3):
        code, byte = ref.quantize(plain, fmt, exponent)
        want_c, want_s = ref.pack(code)[at], ref.store_scales(byte[at], None, 1, 0xA5)
        for view in layouts(torch, x):
            c, s = run(torch, B, view, fmt, rows, exponent=exponent)
            np.testing.assert_array_equal(s, want_s)
            np.testing.assert_array_equal(c, want_c)


@pytest.mark.parametrize("fmt", [ref.MX, ref.NV])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,K", [(8000, 1200), (2400, 4097)])
def test_gathered_rows_in_groups(env, fmt, dtype, rows, K):
    torch, B = env
    few = some_rows(torch, dtype_of(torch, dtype), 150, K, 7)
    rng = np.random.default_rng(rows)
    source = rng.integers(0, 150, rows)
    code, byte = ref.quantize(few.float().cpu().numpy().astype(np.float64), fmt)
    zero_c, zero_s = ref.quantize(np.zeros((1, K)), fmt)
    outside = rng.permutation(rows)[:40]
    source[outside] = rng.choice([-1, -7, 150, 1 << 30], 40)        # rows of zeros
    ok = (source >= 0) & (source < 150)
    pick = np.where(ok, source, 0)
    for offsets in (None, [0, 0, 5, rows // 2, rows // 2 + 129, rows], [11, 140, rows - 9], sorted(rng.integers(0, rows + 1, 301))):
        groups = 1 if offsets is None else len(offsets) - 1
        want_c = np.where(ok[:, None], ref.pack(code)[pick], ref.pack(zero_c))
        want_s = ref.store_scales(np.where(ok[:, None], byte[pick], zero_s), offsets, groups, 0xA5)
        if offsets is not None:
            want_c[ref.places(rows, offsets) < 0] = 0xA5
        dev = lambda a: None if a is None else torch.as_tensor(np.asarray(a, dtype=np.int32), device=DEV)
        for view in layouts(torch, few):
            c, s = run(torch, B, view, fmt, rows, source=dev(source), offsets=dev(offsets))
            np.testing.assert_array_equal(s, want_s)
            np.testing.assert_array_equal(c, want_c)


@pytest.mark.parametrize("fmt", [ref.MX, ref.NV])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,K", SIZES)
def test_values_back(env, fmt, dtype, rows, K):
    torch, B = env
    rng = np.random.default_rng(rows + K)
    dt = dtype_of(torch, dtype)
    code, byte = ref.random_stored(rng, 120, K, fmt)
    byte[3, 0] = byte[5, (K - 1) // ref.BLOCK[fmt]] = 255 if fmt == ref.MX else 127         # NaN
    at = rng.integers(0, 120, rows)
    values = ref.values(code, byte, fmt, K)
    codes = torch.as_tensor(ref.pack(code)[at], device=DEV)
    for offsets in (None, np.array([0, 0, 3, rows // 2, rows // 2 + 130, rows - 1])):
        groups = 1 if offsets is None else len(offsets) - 1
        scales = torch.as_tensor(ref.store_scales(byte[at], offsets, groups, 0xA5), device=DEV)
        off = None if offsets is None else torch.as_tensor(offsets.astype(np.int32), device=DEV)
        for exponent in (0, -2):
            # a code times a scale has at most six significant bits and stays far from the types' limits: no rounding
            want = torch.as_tensor(values * 2.0 ** exponent, device=DEV)[torch.as_tensor(at, device=DEV)].to(dt)
            want[torch.as_tensor(ref.places(rows, offsets) < 0, device=DEV)] = 7.0
            for cols in ((K + 7) // 8 * 8 + 8, K + 1 + K % 2):
                y = torch.full((rows, cols), 7.0, dtype=dt, device=DEV)
                B.bnn_f4_dequantize(codes, scales, y[:, :K], fmt, offsets=off, exponent=exponent)
                torch.testing.assert_close(y[:, :K], want, rtol=0, atol=0, equal_nan=True)
                assert (y[:, K:] == 7.0).all()

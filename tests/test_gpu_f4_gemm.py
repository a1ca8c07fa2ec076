"""Products of quantised matrices, dense and by groups, against 64 bits: every width of a tile, cut blocks, stages and
tiles, empty groups, rows in no group, the epilogues, and scales that are NaN."""
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


def stored(torch, code, byte, offsets=None, groups=1, pad=0):
    """Device tensors of a quantised matrix; bytes that belong to no row are garbage."""
    c = ref.pack(code)
    wide = np.full((c.shape[0], c.shape[1] + 16 * pad), 0xA5, dtype=np.uint8)
    wide[:, :c.shape[1]] = c
    return (torch.as_tensor(wide, device=DEV), torch.as_tensor(ref.store_scales(byte, offsets, groups, 0xFF), device=DEV))


def product(a, w):
    """(sums, sums of magnitudes) in 64 bits"""
    return a @ w.T, np.abs(a) @ np.abs(w).T


def bound(total, mag, K, eps):
    """K additions in fp32 that may cut instead of round, each off by at most a step of a partial sum (2^-23 of the sum of
    magnitudes), and the rounding to the result's type, half a step of it."""
    return K * 2.0 ** -23 * mag * (1 + eps) + eps / 2 * np.abs(total) + 1e-30


EPS = {"f32": 2.0 ** -23, "f16": 2.0 ** -10, "bf16": 2.0 ** -7}


def dtype_of(torch, name):
    return {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}[name]


@pytest.mark.parametrize("fmt", [ref.MX, ref.NV])
@pytest.mark.parametrize("M,N,K", [
    (1, 1, 1), (1, 128, 32), (1, 130, 64), (2, 5, 33), (1, 2048, 2048), (7, 300, 440), (16, 127, 96), (17, 129, 128), (31, 64, 160), (32, 256, 256),
    (33, 140, 288), (64, 100, 513), (100, 257, 1000), (128, 128, 384), (129, 384, 224), (200, 77, 640), (255, 200, 31), (256, 128, 512),
    (257, 300, 100), (300, 129, 1100), (511, 640, 300), (513, 260, 2048), (1100, 900, 700),
    # enough tiles for pairs of CTAs
    (1100, 2304, 300), (2050, 1300, 513), (1537, 2561, 64), (2300, 1290, 1100), (1290, 2056, 32),
    (1100, 2304, 2600), (1290, 2304, 2048), (2300, 1290, 4200),
    # pairs whose tiles have 192 rows
    (731, 3307, 300), (576, 4700, 2050), (700, 3300, 1000)])
def test_product(env, fmt, M, N, K):
    torch, B = env
    rng = np.random.default_rng(M * 31 + N * 7 + K)
    a, w = ref.random_stored(rng, M, K, fmt), ref.random_stored(rng, N, K, fmt)
    (ad, asc), (wd, wsc) = stored(torch, *a, pad=M % 2), stored(torch, *w, pad=N % 2)
    total, mag = product(ref.values(*a, fmt, K), ref.values(*w, fmt, K))
    for name in ("f32", "f16", "bf16"):
        y = torch.full((M + 1, N + 3), 9.0, dtype=dtype_of(torch, name), device=DEV)
        B.bnn_f4_gemm(ad, asc, wd, wsc, K, y[:M, :N], fmt, exponent=-3)
        got = y.double().cpu().numpy()
        assert (got[M] == 9.0).all() and (got[:, N:] == 9.0).all()
        err = np.abs(got[:M, :N] - total / 8)
        assert (err <= bound(total / 8, mag / 8, K, EPS[name])).all(), (err / bound(total / 8, mag / 8, K, EPS[name])).max()
    assert B.bnn_device_status() == 0


@pytest.mark.parametrize("fmt", [ref.MX, ref.NV])
@pytest.mark.parametrize("M,N,K", [(1, 200, 4096), (40, 128, 1000), (300, 300, 2050), (700, 513, 352)])
def test_sums_that_fp32_holds_are_exact(env, fmt, M, N, K):
    """Scales of 1: products are multiples of 1/4 and sums stay below 2^22."""
    torch, B = env
    rng = np.random.default_rng(K)
    a, w = ref.random_stored(rng, M, K, fmt, 0), ref.random_stored(rng, N, K, fmt, 0)
    (ad, asc), (wd, wsc) = stored(torch, *a), stored(torch, *w)
    y = torch.empty((M, N), device=DEV)
    B.bnn_f4_gemm(ad, asc, wd, wsc, K, y, fmt)
    np.testing.assert_array_equal(y.double().cpu().numpy(), product(ref.values(*a, fmt, K), ref.values(*w, fmt, K))[0])


@pytest.mark.parametrize("fmt", [ref.MX, ref.NV])
def test_every_scale_meets_its_block(env, fmt):
    """One element of A in each row, of another block; W's scales all differ from their neighbours."""
    torch, B = env
    rng = np.random.default_rng(3)
    K, N, n = 1200, 300, ref.BLOCK[fmt]
    M = -(-K // n)
    code, byte = np.zeros((M, 2 * ref.pitch(K)), dtype=np.uint8), ref.random_stored(rng, M, K, fmt, 3)[1]
    code[np.arange(M), np.minimum(np.arange(M) * n + n // 3, K - 1)] = 7
    w = ref.random_stored(rng, N, K, fmt, 3)
    (ad, asc), (wd, wsc) = stored(torch, code, byte), stored(torch, *w)
    y = torch.empty((M, N), device=DEV)
    B.bnn_f4_gemm(ad, asc, wd, wsc, K, y, fmt)
    np.testing.assert_array_equal(y.double().cpu().numpy(), product(ref.values(code, byte, fmt, K), ref.values(*w, fmt, K))[0])


@pytest.mark.parametrize("fmt", [ref.MX, ref.NV])
@pytest.mark.parametrize("M", [5, 150, 400])
def test_epilogues(env, fmt, M):
    torch, B = env
    rng = np.random.default_rng(M)
    N, K = 203, 500
    a, w = ref.random_stored(rng, M, K, fmt), ref.random_stored(rng, N, K, fmt)
    (ad, asc), (wd, wsc) = stored(torch, *a), stored(torch, *w)
    total, mag = product(ref.values(*a, fmt, K), ref.values(*w, fmt, K))
    scale, shift = rng.normal(0, 0.02, N).astype(np.float32), rng.normal(0, 1, N).astype(np.float32)
    sc, sh = torch.as_tensor(scale, device=DEV), torch.as_tensor(shift, device=DEV)
    for use in ("both", "scale", "shift", "none"):
        s, h = (scale if use in ("both", "scale") else np.ones(N)), (shift if use in ("both", "shift") else np.zeros(N))
        pre, off = total * s + h, K * 2.0 ** -23 * mag * np.abs(s)
        kw = dict(scale=sc if use in ("both", "scale") else None, shift=sh if use in ("both", "shift") else None)
        off = off + 2.0 ** -23 * np.abs(pre) + 1e-30           # the sums, and the rounding of the fused multiply-add
        y = torch.empty((M, N), device=DEV)
        B.bnn_f4_gemm(ad, asc, wd, wsc, K, y, fmt, **kw)
        assert (np.abs(y.double().cpu().numpy() - pre) <= off).all(), use
        B.bnn_f4_gemm(ad, asc, wd, wsc, K, y, fmt, act=B.ACT_HARDTANH, **kw)
        assert (np.abs(y.double().cpu().numpy() - np.clip(pre, -1, 1)) <= off).all(), use
        B.bnn_f4_gemm(ad, asc, wd, wsc, K, y, fmt, act=B.ACT_SIGMOID, **kw)
        # expf is within 2 steps of 2^-23, the sum and the quotient half a step each; the slope is at most 1/4
        with np.errstate(over="ignore"):
            want = 1 / (1 + np.exp(-pre))
        assert (np.abs(y.double().cpu().numpy() - want) <= off / 4 + 4 * 2.0 ** -23 * want + 1e-30).all(), use
        for mode in (B.SIGN_ZERO_POS, B.SIGN_ZERO_NEG):
            bits = torch.full((M + 1, B.packed_pitch(N) + 4), -1, dtype=torch.int32, device=DEV)
            B.bnn_f4_gemm(ad, asc, wd, wsc, K, None, fmt, act=B.ACT_SIGN_PACK, sign_mode=mode, out_bits=bits[:M], **kw)
            words = bits.cpu().numpy().view(np.uint32)
            nw = (N + 31) // 32
            assert (words[M] == 0xFFFFFFFF).all() and (words[:, nw:] == 0xFFFFFFFF).all()
            got = (words[:M, :nw, None] >> np.arange(32, dtype=np.uint32) & 1).reshape(M, -1).astype(bool)
            assert not got[:, N:].any()
            sure = np.abs(pre) > off
            assert (got[:, :N] == (pre > 0))[sure].all() and sure.mean() > 0.9
    assert B.bnn_device_status() == 0


def test_sign_of_zero_sums(env):
    torch, B = env
    K, M, N = 64, 3, 40
    code, byte = np.zeros((M, 2 * ref.pitch(K)), dtype=np.uint8), np.full((M, 4), 127, dtype=np.uint8)
    byte[:, 2:] = 0
    w = ref.random_stored(np.random.default_rng(0), N, K, ref.MX)
    (ad, asc), (wd, wsc) = stored(torch, code, byte), stored(torch, *w)
    for mode, word in ((B.SIGN_ZERO_POS, (0xFFFFFFFF, 0xFF)), (B.SIGN_ZERO_NEG, (0, 0))):
        bits = torch.zeros((M, 4), dtype=torch.int32, device=DEV)
        B.bnn_f4_gemm(ad, asc, wd, wsc, K, None, ref.MX, act=B.ACT_SIGN_PACK, sign_mode=mode, out_bits=bits)
        assert (bits.cpu().numpy().view(np.uint32)[:, :2] == word).all()


@pytest.mark.parametrize("fmt", [ref.MX, ref.NV])
def test_a_scale_that_is_nan_stays_in_its_row(env, fmt):
    torch, B = env
    rng = np.random.default_rng(8)
    for M, N, K in ((3, 130, 96), (150, 200, 300), (400, 140, 512)):
        a, w = ref.random_stored(rng, M, K, fmt), ref.random_stored(rng, N, K, fmt)
        nan = 255 if fmt == ref.MX else 127
        a[1][M // 2, 1], w[1][N - 1, 0] = nan, nan
        (ad, asc), (wd, wsc) = stored(torch, *a), stored(torch, *w)
        y = torch.empty((M, N), device=DEV)
        B.bnn_f4_gemm(ad, asc, wd, wsc, K, y, fmt)
        want = np.zeros((M, N), dtype=bool)
        want[M // 2], want[:, N - 1] = True, True
        np.testing.assert_array_equal(np.isnan(y.cpu().numpy()), want)


GROUPS = {
    "one_row_each": lambda rng: np.arange(41),
    "mostly_empty": lambda rng: np.array([0] * 9 + [1, 1, 1, 3, 3, 40, 40]),
    "ragged": lambda rng: np.concatenate([[0], np.cumsum(rng.integers(0, 300, 12))]),
    "one_large": lambda rng: np.array([0, 2, 1000, 1000, 1001]),
    "with_rows_outside": lambda rng: np.array([5, 70, 70, 333, 600]),
    "none": lambda rng: np.zeros(8, dtype=np.int64),
    "pairs": lambda rng: np.array([3, 300, 1301, 1301, 1302, 2799]),
    "many_pairs": lambda rng: np.concatenate([[0], np.cumsum(rng.integers(1, 700, 13))]),
    "many": lambda rng: np.concatenate([[0], np.sort(rng.integers(0, 1500, 1023)), [1500]]),
}


@pytest.mark.parametrize("fmt", [ref.MX, ref.NV])
@pytest.mark.parametrize("kind", sorted(GROUPS))
def test_groups(env, fmt, kind):
    torch, B = env
    rng = np.random.default_rng(len(kind))
    off = GROUPS[kind](rng)
    G, M = len(off) - 1, max(int(off[-1]), 1) + 7
    N, K = (33, 70) if G > 100 else (1300, 200) if "pairs" in kind else (300, 420)
    a, w = ref.random_stored(rng, M, K, fmt), ref.random_stored(rng, G * N, K, fmt)
    (ad, asc), (wd, wsc) = stored(torch, *a, offsets=off, groups=G), stored(torch, *w, offsets=np.arange(G + 1) * N, groups=G)
    av, wv = ref.values(*a, fmt, K), ref.values(*w, fmt, K).reshape(G, N, K)
    shift = rng.normal(0, 1, (G, N)).astype(np.float32)
    offd = torch.as_tensor(off.astype(np.int32), device=DEV)
    for name, sh in (("f32", None), ("bf16", torch.as_tensor(shift, device=DEV))):
        y = torch.full((M, N), 9.0, dtype=dtype_of(torch, name), device=DEV)
        B.bnn_f4_gemm_grouped(ad, asc, offd, wd.view(G, N, -1), wsc, K, y, fmt, shift=sh)
        got = y.double().cpu().numpy()
        seen = np.zeros(M, dtype=bool)
        for g in range(G):
            lo, hi = int(off[g]), int(off[g + 1])
            seen[lo:hi] = True
            if hi > lo:
                total, mag = product(av[lo:hi], wv[g])
                total = total + (0 if sh is None else shift[g])
                err, most = np.abs(got[lo:hi] - total), bound(total, mag + np.abs(total), K + 1, EPS[name])
                assert (err <= most).all(), (g, (err / most).max())
        assert (got[~seen] == 9.0).all()
    assert B.bnn_device_status() == 0


@pytest.mark.parametrize("fmt", [ref.MX, ref.NV])
@pytest.mark.parametrize("rows", [12, 500, 3000])
def test_groups_to_bits_and_other_pitches(env, fmt, rows):
    """A binary layer behind each expert's layer: few rows, single CTAs and pairs; weights whose rows are further apart."""
    torch, B = env
    rng = np.random.default_rng(rows)
    G, N, K = 4, 1290, 530
    off = np.concatenate([[0], np.sort(rng.integers(0, rows, G - 1)), [rows]])
    a, w = ref.random_stored(rng, rows, K, fmt), ref.random_stored(rng, G * N, K, fmt)
    (ad, asc), (wd, wsc) = stored(torch, *a, offsets=off, groups=G), stored(torch, *w, offsets=np.arange(G + 1) * N, groups=G, pad=2)
    scale, shift = rng.normal(0, 1, (G, N)).astype(np.float32), rng.normal(0, 20, (G, N)).astype(np.float32)
    dev = lambda x: torch.as_tensor(x, device=DEV)
    bits = torch.full((rows, B.packed_pitch(N)), -1, dtype=torch.int32, device=DEV)
    B.bnn_f4_gemm_grouped(ad, asc, dev(off.astype(np.int32)), wd.view(G, N, -1), wsc, K, None, fmt, act=B.ACT_SIGN_PACK, scale=dev(scale), shift=dev(shift), out_bits=bits)
    nw = (N + 31) // 32
    got = (bits.cpu().numpy().view(np.uint32)[:, :nw, None] >> np.arange(32, dtype=np.uint32) & 1).reshape(rows, -1).astype(bool)
    av, wv = ref.values(*a, fmt, K), ref.values(*w, fmt, K).reshape(G, N, K)
    for g in range(G):
        lo, hi = off[g], off[g + 1]
        total, mag = product(av[lo:hi], wv[g])
        pre = total * scale[g] + shift[g]
        sure = np.abs(pre) > K * 2.0 ** -23 * mag * np.abs(scale[g]) + 2.0 ** -23 * np.abs(pre)
        assert (got[lo:hi, :N] == (pre > 0))[sure].all()
    assert not got[:, N:].any() and B.bnn_device_status() == 0


def test_a_thousand_groups_on_pairs(env):
    torch, B = env
    rng = np.random.default_rng(6)
    G, N, K = 1024, 600, 64
    off = np.concatenate([[0], np.cumsum(rng.integers(0, 300, G))])
    M = int(off[-1])
    a, w = ref.random_stored(rng, M, K, ref.MX, 0), ref.random_stored(rng, G * N, K, ref.MX, 0)
    (ad, asc), (wd, wsc) = stored(torch, *a, offsets=off, groups=G), stored(torch, *w, offsets=np.arange(G + 1) * N, groups=G)
    y = torch.empty((M, N), device=DEV)
    B.bnn_f4_gemm_grouped(ad, asc, torch.as_tensor(off.astype(np.int32), device=DEV), wd.view(G, N, -1), wsc, K, y, ref.MX)
    got, av, wv = y.cpu().numpy(), ref.values(*a, ref.MX, K), ref.values(*w, ref.MX, K).reshape(G, N, K)
    for g in range(G):      # multiples of 1/4 that fp32 holds
        np.testing.assert_array_equal(got[off[g]:off[g + 1]], (av[off[g]:off[g + 1]] @ wv[g].T).astype(np.float32))
    assert B.bnn_device_status() == 0


def test_offsets_that_make_no_sense_stay_inside(env):
    torch, B = env
    rng = np.random.default_rng(1)
    M, N, K = 100, 130, 64
    for off in ([90, 20, 0], [-5, 10, 1 << 30], [7, -1, 3, 50], [1 << 30, 1 << 30], [0, 100, 0, 100]):
        G = len(off) - 1
        a, w = ref.random_stored(rng, M, K, ref.MX), ref.random_stored(rng, G * N, K, ref.MX)
        ad, asc = stored(torch, *a, groups=G)
        wd, wsc = stored(torch, *w, offsets=np.arange(G + 1) * N, groups=G)
        y = torch.full((M + 1, N), 9.0, device=DEV)
        B.bnn_f4_gemm_grouped(ad, asc, torch.as_tensor(np.array(off, dtype=np.int32), device=DEV), wd.view(G, N, -1), wsc, K, y[:M], ref.MX)
        assert (y[M] == 9.0).all()
    assert B.bnn_device_status() == 0


@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_rows_further_apart_than_32_bits_hold(env, name):
    torch, B = env
    rng = np.random.default_rng(4)
    M, N, K, far = 3, 200, 96, 1 << 30
    a, w = ref.random_stored(rng, M, K, ref.MX, 0), ref.random_stored(rng, N, K, ref.MX, 0)
    (ad, asc), (wd, wsc) = stored(torch, *a), stored(torch, *w)
    room = torch.empty((2 * far + N,), dtype=dtype_of(torch, name), device=DEV)
    y = room.as_strided((M, N), (far, 1))
    B.bnn_f4_gemm(ad, asc, wd, wsc, K, y, ref.MX)
    apart = torch.empty((2 * far + 4096,), dtype=torch.uint8, device=DEV).as_strided((M, ad.shape[1]), (far, 1))
    apart.copy_(ad)
    z = torch.empty((M, N), dtype=y.dtype, device=DEV)
    B.bnn_f4_gemm(apart, asc, wd, wsc, K, z, ref.MX)
    want = product(ref.values(*a, ref.MX, K), ref.values(*w, ref.MX, K))[0]       # multiples of 1/4, held exactly by fp32
    got = y.double().cpu().numpy()
    assert (np.abs(got - want) <= (0 if name == "f32" else 2.0 ** -8) * np.abs(want)).all()
    assert torch.equal(z, y)


@pytest.mark.parametrize("M,N,K", [(1, 700, 2048), (20, 300, 1100), (90, 900, 700), (1100, 2304, 600)])
def test_captured_products_on_two_streams(env, M, N, K):
    """Two products of each form captured into graphs and replayed side by side, on new values each time."""
    torch, B = env
    rng = np.random.default_rng(M)
    runs = []
    for fmt in (ref.MX, ref.NV):
        a, w = ref.random_stored(rng, M, K, fmt, 0), ref.random_stored(rng, N, K, fmt, 0)
        (ad, asc), (wd, wsc) = stored(torch, *a), stored(torch, *w)
        y, g = torch.empty((M, N), device=DEV), torch.cuda.CUDAGraph()
        B.bnn_f4_gemm(ad, asc, wd, wsc, K, y, fmt)
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            for _ in range(3):
                B.bnn_f4_gemm(ad, asc, wd, wsc, K, y, fmt)
        runs.append((fmt, ad, asc, w, y, g, torch.cuda.Stream(), (wd, wsc)))     # (a graph keeps no tensor alive)
    for turn in range(3):
        news = []
        for fmt, ad, asc, w, y, g, st, _ in runs:
            a = ref.random_stored(rng, M, K, fmt, 0)
            ad.copy_(torch.as_tensor(ref.pack(a[0]), device=DEV))
            asc.copy_(torch.as_tensor(ref.store_scales(a[1], None, 1, 0xFF), device=DEV))
            news.append(a)
        torch.cuda.synchronize()
        for fmt, ad, asc, w, y, g, st, _ in runs:
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for a, (fmt, ad, asc, w, y, g, st, _) in zip(news, runs):
            # scales of 1: the sums are multiples of 1/4 that fp32 holds
            np.testing.assert_array_equal(y.double().cpu().numpy(), product(ref.values(*a, fmt, K), ref.values(*w, fmt, K))[0])
    assert B.bnn_device_status() == 0


def test_the_binding_refuses_what_does_not_fit(env):
    torch, B = env
    u8 = dict(dtype=torch.uint8, device=DEV)
    M, N, K = 5, 40, 96
    a, w, y = torch.zeros((M, 48), **u8), torch.zeros((N, 48), **u8), torch.zeros((M, N), device=DEV)
    sa, sw = torch.zeros((512,), **u8), torch.zeros((512,), **u8)
    B.bnn_f4_gemm(a, sa, w, sw, K, y)
    for bad in (dict(A=a.cpu()), dict(w_scales=sw.cpu()), dict(Y=y[:4]), dict(Y=y.t().contiguous()), dict(Y=y[:, :39]), dict(A=a.float()),
                dict(W=w.t()), dict(a_scales=sa.int()), dict(shift=torch.zeros(N + 1, device=DEV)), dict(scale=torch.zeros(N, device=DEV).half())):
        with pytest.raises((ValueError, TypeError)):
            B.bnn_f4_gemm(**{**dict(A=a, a_scales=sa, W=w, w_scales=sw, K=K, Y=y), **bad})
    for bad, status in ((dict(K=97), 2), (dict(a_scales=sa[:256]), 5), (dict(exponent=65), 2), (dict(fmt=7), 4), (dict(Y=None), 1)):
        with pytest.raises(B.BnnError) as e:
            B.bnn_f4_gemm(**{**dict(A=a, a_scales=sa, W=w, w_scales=sw, K=K, Y=y), **bad})
        assert e.value.status == status and "bnn_f4_gemm" in str(e.value)
    off = torch.zeros((3,), dtype=torch.int32, device=DEV)
    for bad in (w, w.view(4, 10, 48), torch.zeros((2, 2 * 20, 48), **u8)[:, :20]):
        with pytest.raises(ValueError):
            B.bnn_f4_gemm_grouped(a, torch.zeros((1024,), **u8), off, bad, torch.zeros((2048,), **u8), K, y[:, :20])
    with pytest.raises(ValueError):
        B.bnn_f4_quantize(torch.zeros((9, K), device=DEV), a, sa, source=torch.zeros((4,), dtype=torch.int32, device=DEV))
    with pytest.raises(TypeError):
        B.bnn_f4_quantize(torch.zeros((M, K), device=DEV, dtype=torch.float64), a, sa)
    with pytest.raises(ValueError):
        B.bnn_f4_dequantize(a, sa, torch.zeros((4, K), device=DEV))
    i32 = dict(dtype=torch.int32, device=DEV)
    route = dict(logits=torch.zeros((6, 8), device=DEV), index=torch.zeros((6, 2), **i32), weight=torch.zeros((6, 2), device=DEV), offsets=torch.zeros((9,), **i32),
                 slot=torch.zeros((6, 2), **i32), source=torch.zeros((12,), **i32), workspace=torch.zeros((64,), **u8))
    B.bnn_route_experts(**route)
    for bad in (dict(index=torch.zeros((5, 2), **i32)), dict(offsets=torch.zeros((8,), **i32)), dict(source=torch.zeros((11,), **i32)), dict(weight=route["weight"].half()),
                dict(slot=torch.zeros((6, 3), **i32)), dict(logits=route["logits"].t())):
        with pytest.raises(ValueError):
            B.bnn_route_experts(**{**route, **bad})
    z, yy = torch.zeros((12, 40), device=DEV), torch.zeros((6, 40), device=DEV)
    for bad in ((z, route["slot"], route["weight"], yy[:5]), (z, route["slot"], route["weight"][:, :1], yy), (z[:, :39], route["slot"], route["weight"], yy)):
        with pytest.raises(ValueError):
            B.bnn_combine_experts(*bad)
    assert B.bnn_device_status() == 0

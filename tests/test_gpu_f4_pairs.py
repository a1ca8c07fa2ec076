"""Products of quantised matrices in the forms that large sizes take: pairs of CTAs with 192 and 256 rows, several tiles a pair of several
steps of K each, every type of result, pitch and epilogue, dense and by groups.  Each test states the form that its sizes
choose.

Scales are powers of two between 1/2 and 2: products are multiples of 1/16, and as long as the magnitudes of a sum add up to less than 2^20
(checked) every partial sum is held exactly by fp32, whatever the order.  So the sums are compared for equality."""
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


def matrix(torch, rng, rows, K, fmt, offsets=None, groups=1, pad=0):
    """(codes, scales, values): scales 1/2, 1, 2; bytes that belong to no row are garbage, a scale of NaN among them"""
    code, byte = ref.random_stored(rng, rows, K, fmt, 0)
    live = -(-K // ref.BLOCK[fmt])
    one, step = (127, 1) if fmt == ref.MX else (0x38, 8)
    byte[:, :live] = one + step * rng.integers(-1, 2, (rows, live))
    packed = ref.pack(code)
    wide = np.full((rows, packed.shape[1] + 16 * pad), 0xA5, dtype=np.uint8)
    wide[:, :packed.shape[1]] = packed
    dev = lambda x: torch.as_tensor(x, device=DEV)
    return dev(wide), dev(ref.store_scales(byte, offsets, groups, 0xFF)), dev(ref.values(code, byte, fmt, K))


def exact_sums(av, wv):
    assert (av.abs() @ wv.abs().T).max() < 1 << 20
    return av @ wv.T


def types(torch):
    return torch.float32, torch.float16, torch.bfloat16


def turns(form, M, N):
    return -(-M // form[1]) * -(-N // (128 * form[0])) / (148 // form[0])


DENSE = [
    # several turns, several steps; N and K end inside a tile, a stage and a block
    (4096, 2304, 2100, (2, 256, 1)), (8200, 1290, 1999, (2, 256, 1)), (5000, 3336, 2056, (2, 256, 1)), (3000, 9001, 513, (2, 256, 1)),
    (4100, 2310, 2100, (2, 192, 1)), (1800, 7000, 1300, (2, 192, 1)), (1500, 3336, 2100, (2, 192, 1)),
    (300, 520, 2304, (1, 128, 1)), (90, 21000, 700, (1, 128, 1))]


@pytest.mark.parametrize("fmt", [ref.MX, ref.NV])
@pytest.mark.parametrize("M,N,K,form", DENSE)
def test_dense(env, fmt, M, N, K, form):
    torch, B = env
    assert B.bnn_f4_gemm_form(M, N, K) == form and (form[0] == 1 or turns(form, M, N) > 1)
    rng = np.random.default_rng(M + N + K)
    a, asc, av = matrix(torch, rng, M, K, fmt, pad=1)
    w, wsc, wv = matrix(torch, rng, N, K, fmt)
    want = exact_sums(av, wv) / 8
    for dtype in types(torch):
        for cols in ((N + 15) // 8 * 8, N + 1 + N % 2):        # rows of 16-byte pieces, and rows that start anywhere
            y = torch.full((M + 1, cols), 9.0, dtype=dtype, device=DEV)
            B.bnn_f4_gemm(a, asc, w, wsc, K, y[:M, :N], fmt, exponent=-3)
            assert torch.equal(y[:M, :N], want.to(dtype)), (dtype, cols)
            assert (y[M] == 9.0).all() and (y[:, N:] == 9.0).all()
    assert B.bnn_device_status() == 0


def check_epilogues(torch, B, call, want, scale, shift, M, N):
    """All activations and types of result; `call(Y, **epilogue)`, `want`: the exact sums, `scale`, `shift`: as they meet them."""
    pre = want * scale.double() + shift.double()
    # The sum is exact, the fused multiply-add off by half a step of fp32, a 16-bit result by half a step of its own (of fp16's subnormal
    # numbers 2^-25).  expf is within two steps, the sum and the quotient of a sigmoid half a step each; its slope is at most 1/4.
    fma = 2.0 ** -24 * pre.abs() + 1e-40
    for act, exact, off in ((B.ACT_NONE, pre, fma), (B.ACT_HARDTANH, pre.clamp(-1, 1), fma), (B.ACT_SIGMOID, torch.sigmoid(pre), fma / 4 + 4 * 2.0 ** -23 * torch.sigmoid(pre))):
        for dtype in types(torch):
            for cols in ((N + 7) // 8 * 8, N + 1 + N % 2):
                y = torch.full((M, cols), 9.0, dtype=dtype, device=DEV)
                call(y[:, :N], act=act)
                most = off if dtype == torch.float32 else off + torch.finfo(dtype).eps / 2 * (exact.abs() + off) + (2.0 ** -25 if dtype == torch.float16 else 0)
                assert ((y[:, :N].double() - exact).abs() <= most).all(), (act, dtype, cols)
                assert (y[:, N:] == 9.0).all()
    clear = pre.abs() > 2.0 ** -50 * ((want * scale.double()).abs() + shift.double().abs())      # (pre itself is rounded to 53 bits)
    nw = (N + 31) // 32
    for mode in (B.SIGN_ZERO_POS, B.SIGN_ZERO_NEG):
        bits = torch.full((M, B.packed_pitch(N) + 4), -1, dtype=torch.int32, device=DEV)
        call(None, act=B.ACT_SIGN_PACK, sign_mode=mode, out_bits=bits)
        assert (bits[:, nw:] == -1).all()
        got = (bits[:, :nw, None] >> torch.arange(32, device=DEV) & 1).reshape(M, -1).bool()
        assert not got[:, N:].any() and (got[:, :N] == (pre > 0))[clear].all() and clear.double().mean() > 0.99
    assert B.bnn_device_status() == 0


@pytest.mark.parametrize("fmt", [ref.MX, ref.NV])
@pytest.mark.parametrize("M,N,K,form", [(4096, 2301, 2100, (2, 256, 1)), (4100, 2310, 700, (2, 192, 1)), (300, 523, 2304, (1, 128, 1)), (20, 1003, 2100, (1, 32, 4)),
                                        (9, 12003, 700, (1, 32, 1))])
def test_dense_epilogues(env, fmt, M, N, K, form):
    torch, B = env
    assert B.bnn_f4_gemm_form(M, N, K) == form
    rng = np.random.default_rng(M + N)
    a, asc, av = matrix(torch, rng, M, K, fmt)
    w, wsc, wv = matrix(torch, rng, N, K, fmt)
    dev = lambda x: torch.as_tensor(x.astype(np.float32), device=DEV)
    scale, shift = dev(rng.normal(0, 0.01, N)), dev(rng.normal(0, 1, N))
    check_epilogues(torch, B, lambda y, **kw: B.bnn_f4_gemm(a, asc, w, wsc, K, y, fmt, scale=scale, shift=shift, **kw), exact_sums(av, wv), scale, shift, M, N)


def spread(rng, rows, G, outside=0):
    """Offsets of G groups of unequal size, some empty, `outside` rows before the first and behind the last."""
    share = rng.dirichlet(np.full(G, 1.5))
    share[rng.permutation(G)[:G // 4]] = 0
    ends = np.round(np.cumsum(share / share.sum()) * (rows - 2 * outside)).astype(np.int64)
    return np.concatenate([[0], ends]) + outside


def group_of_rows(off, M):
    g = np.full(M, -1)
    for i in range(len(off) - 1):
        g[off[i]:off[i + 1]] = i
    return g


def make_groups(torch, rng, M, N, K, off, fmt, pad=0):
    G = len(off) - 1
    a, asc, av = matrix(torch, rng, M, K, fmt, off, G)
    w, wsc, wv = matrix(torch, rng, G * N, K, fmt, np.arange(G + 1) * N, G, pad)
    offd = torch.as_tensor(off.astype(np.int32), device=DEV)
    want = torch.zeros((M, N), dtype=torch.float64, device=DEV)
    for g in range(G):
        if off[g + 1] > off[g]:
            want[off[g]:off[g + 1]] = exact_sums(av[off[g]:off[g + 1]], wv[g * N:(g + 1) * N])
    return a, asc, offd, w.view(G, N, -1), wsc, want


GROUPED = [(6000, 1290, 2100, 9, (2, 256, 1)), (9000, 2568, 1100, 12, (2, 256, 1)), (4000, 5000, 700, 5, (2, 256, 1)), (8000, 2048, 2304, 8, (2, 256, 1)),
           (2000, 1003, 1100, 64, (1, 128, 1)), (1500, 2056, 300, 3, (1, 128, 1))]


@pytest.mark.parametrize("fmt", [ref.MX, ref.NV])
@pytest.mark.parametrize("M,N,K,G,form", GROUPED)
def test_groups(env, fmt, M, N, K, G, form):
    torch, B = env
    assert B.bnn_f4_gemm_form(M, N, K, G) == form
    rng = np.random.default_rng(M + G)
    outside = 3 * (G % 2)
    off = spread(rng, M, G, outside)
    a, asc, offd, w, wsc, want = make_groups(torch, rng, M, N, K, off, fmt, pad=G % 3)
    live = torch.as_tensor(group_of_rows(off, M) >= 0, device=DEV)
    for dtype in types(torch):
        for cols in ((N + 7) // 8 * 8, N + 1 + N % 2):
            y = torch.full((M, cols), 9.0, dtype=dtype, device=DEV)
            B.bnn_f4_gemm_grouped(a, asc, offd, w, wsc, K, y[:, :N], fmt, exponent=-3)
            assert torch.equal(y[live][:, :N], (want / 8).to(dtype)[live]), (dtype, cols)
            assert (y[~live] == 9.0).all() and (y[:, N:] == 9.0).all()
    assert B.bnn_device_status() == 0


@pytest.mark.parametrize("fmt", [ref.MX, ref.NV])
@pytest.mark.parametrize("M,N,K,G,form", [(6000, 1290, 2100, 9, (2, 256, 1)), (9000, 2570, 530, 6, (2, 256, 1)), (2000, 523, 700, 40, (1, 128, 1)), (30, 700, 2100, 6, (1, 32, 4))])
def test_epilogues_of_groups(env, fmt, M, N, K, G, form):
    torch, B = env
    assert B.bnn_f4_gemm_form(M, N, K, G) == form
    rng = np.random.default_rng(M + N + G)
    off = spread(rng, M, G)
    a, asc, offd, w, wsc, want = make_groups(torch, rng, M, N, K, off, fmt)
    dev = lambda x: torch.as_tensor(x.astype(np.float32), device=DEV)
    scale, shift = dev(rng.normal(0, 0.01, (G, N))), dev(rng.normal(0, 1, (G, N)))
    g = torch.as_tensor(group_of_rows(off, M), device=DEV)
    call = lambda y, **kw: B.bnn_f4_gemm_grouped(a, asc, offd, w, wsc, K, y, fmt, scale=scale, shift=shift, **kw)
    check_epilogues(torch, B, call, want, scale[g], shift[g], M, N)


@pytest.mark.parametrize("fmt", [ref.MX, ref.NV])
def test_one_group_with_nearly_all_rows(env, fmt):
    """Copies are sized for the average group: the large one takes several to a stage."""
    torch, B = env
    M, N, K, G = 2000, 700, 600, 64
    assert B.bnn_f4_gemm_form(M, N, K, G) == (1, 128, 1)
    rng = np.random.default_rng(2)
    for large, rest in ((0, 8), (40, 8), (63, 8), (20, 0)):
        n = np.full(G, rest)
        n[large] = M - rest * (G - 1)
        off = np.concatenate([[0], np.cumsum(n)])
        a, asc, offd, w, wsc, want = make_groups(torch, rng, M, N, K, off, fmt)
        y = torch.empty((M, N), device=DEV)
        B.bnn_f4_gemm_grouped(a, asc, offd, w, wsc, K, y, fmt)
        assert torch.equal(y.double(), want)
    assert B.bnn_device_status() == 0


def test_a_thousand_groups(env):
    torch, B = env
    M, N, K, G = 600000, 600, 64, 1024
    assert B.bnn_f4_gemm_form(M, N, K, G) == (2, 256, 1)
    rng = np.random.default_rng(6)
    off = spread(rng, M, G)
    a, asc, offd, w, wsc, want = make_groups(torch, rng, M, N, K, off, ref.MX)
    for dtype in (torch.float32, torch.bfloat16):
        y = torch.empty((M, N), dtype=dtype, device=DEV)
        B.bnn_f4_gemm_grouped(a, asc, offd, w, wsc, K, y, ref.MX)
        assert torch.equal(y, want.to(dtype))
    assert B.bnn_device_status() == 0


@pytest.mark.parametrize("fmt", [ref.MX, ref.NV])
@pytest.mark.parametrize("M,N,K", [(4096, 2304, 600), (1500, 3336, 600)])
def test_captured_on_pairs_beside_another_stream(env, fmt, M, N, K):
    """Several turns a pair, replayed on two streams at once, on new activations each time."""
    torch, B = env
    assert B.bnn_f4_gemm_form(M, N, K)[0] == 2
    rng = np.random.default_rng(K)
    w, wsc, wv = matrix(torch, rng, N, K, fmt)
    runs = []
    for i in range(2):
        a, asc, _ = matrix(torch, rng, M, K, fmt)
        y, g = torch.empty((M, N), dtype=torch.bfloat16, device=DEV), torch.cuda.CUDAGraph()
        B.bnn_f4_gemm(a, asc, w, wsc, K, y, fmt)
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            for _ in range(3):
                B.bnn_f4_gemm(a, asc, w, wsc, K, y, fmt)
        runs.append((a, asc, y, g, torch.cuda.Stream()))
    for turn in range(2):
        values = []
        for a, asc, y, g, st in runs:
            new = matrix(torch, rng, M, K, fmt)
            a.copy_(new[0])
            asc.copy_(new[1])
            values.append(new[2])
        torch.cuda.synchronize()
        for a, asc, y, g, st in runs:
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for av, (a, asc, y, g, st) in zip(values, runs):
            assert torch.equal(y, exact_sums(av, wv).to(torch.bfloat16))
    assert B.bnn_device_status() == 0


@pytest.mark.parametrize("M,N,K,form", [(20, 700, 2100, (1, 32, 4)), (9000, 2570, 1100, (2, 256, 1))])
def test_offsets_that_make_no_sense_stay_inside(env, M, N, K, form):
    torch, B = env
    rng = np.random.default_rng(M)
    for off in ([M, M // 2, 0, M], [-5, 10, 1 << 30, 3], [7, -1, 3, M + 40], [1 << 30] * 4, [0, M, 0, M]):
        G = len(off) - 1
        assert B.bnn_f4_gemm_form(M, N, K, G) == form
        a, asc, _ = matrix(torch, rng, M, K, ref.MX, groups=G)
        w, wsc, _ = matrix(torch, rng, G * N, K, ref.MX, np.arange(G + 1) * N, G)
        y = torch.full((M + 1, N), 9.0, device=DEV)
        B.bnn_f4_gemm_grouped(a, asc, torch.as_tensor(np.array(off, dtype=np.int64).astype(np.int32), device=DEV), w.view(G, N, -1), wsc, K, y[:M], ref.MX)
        assert (y[M] == 9.0).all()
    assert B.bnn_device_status() == 0

"""Products of quantised matrices whose waits run out: each form reports it in the status word, returns, and leaves the context as it
was.  A tile takes some hundred microseconds, the limit is one; on its way out a kernel waits for its copies and MMAs by a bound of its own."""
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


def ones(torch, B, fmt, rows, K, seed):
    """(codes, scales of 1, values): whole numbers of halves"""
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    codes = torch.randint(0, 256, (rows, K // 2), generator=g, device=DEV, dtype=torch.uint8)
    scales = torch.full((B.bnn_f4_scale_bytes(fmt, rows, K),), 127 if fmt == ref.MX else 0x38, dtype=torch.uint8, device=DEV)
    return codes, scales, B.bnn_f4_dequantize(codes, scales, torch.empty((rows, K), device=DEV), fmt)


# few rows with a shared K and without, single CTAs, pairs of 192 and of 256 rows
@pytest.mark.parametrize("M,N,K", [(1, 128, 1 << 18), (5, 9700, 1 << 16), (100, 128, 1 << 17), (192, 256, 1 << 17), (4096, 1024, 1 << 17)])
@pytest.mark.parametrize("fmt", [ref.MX, ref.NV])
def test_a_product_that_gives_up(env, fmt, M, N, K):
    torch, B = env
    a, a_scales, av = ones(torch, B, fmt, M, K, 1)
    w, w_scales, wv = ones(torch, B, fmt, N, K, 2)
    y = torch.full((M + 1, N), 9.0, device=DEV)
    assert B.bnn_device_status() == 0
    prev = B.bnn_set_option(B.OPT_WAIT_LIMIT_US, 1)
    try:
        B.bnn_f4_gemm(a, a_scales, w, w_scales, K, y[:M], fmt)
        B.bnn_f4_gemm(a, a_scales, w, w_scales, K, y[:M], fmt)
        assert B.bnn_device_status() == 1
        B.bnn_reset_status()
        assert B.bnn_device_status() == 0
    finally:
        B.bnn_set_option(B.OPT_WAIT_LIMIT_US, prev)
    assert (y[M] == 9.0).all()
    B.bnn_f4_gemm(a, a_scales, w, w_scales, K, y[:M], fmt)
    want = sum(av[:, k:k + 8192].double() @ wv[:, k:k + 8192].double().T for k in range(0, K, 8192))
    # multiples of 1/4; a sum beyond 2^22 would be rounded, and of 2^18 terms of at most 36 with random signs none comes near
    assert want.abs().max() < 1 << 20 and torch.equal(y[:M].double(), want)
    assert (y[M] == 9.0).all() and B.bnn_device_status() == 0

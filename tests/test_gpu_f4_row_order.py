"""The order of a product's sums depends on its sizes and not on the row: equal rows of activations give equal rows of results, bit for
bit, wherever they stand in the batch."""
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


# K shared by four and by two CTAs, K in one, single CTAs, pairs
@pytest.mark.parametrize("M,N,K", [(2, 300, 4096), (31, 2048, 8192), (32, 1000, 2000), (17, 300, 513), (7, 12000, 2048), (100, 700, 4096), (731, 3307, 1000)])
@pytest.mark.parametrize("fmt", [ref.MX, ref.NV])
def test_equal_rows(env, fmt, M, N, K):
    torch, B = env
    rng = np.random.default_rng(M)
    dev = lambda x: torch.as_tensor(x, device=DEV)

    def stored(rows, spread):
        """scales far apart, so that sums are rounded at many places"""
        code, byte = ref.random_stored(rng, rows, K, fmt)
        live = -(-K // ref.BLOCK[fmt])
        byte[:, :live] = rng.integers(127 - spread, 128 + spread, (rows, live)) if fmt == ref.MX else rng.integers(0x20, 0x60, (rows, live))
        return code, byte
    code, byte = stored(1, 12)
    code, byte = np.repeat(code, M, 0), np.repeat(byte, M, 0)
    w = stored(N, 12)
    y = torch.empty((M, N), device=DEV)
    B.bnn_f4_gemm(dev(ref.pack(code)), dev(ref.store_scales(byte, None, 1)), dev(ref.pack(w[0])), dev(ref.store_scales(w[1], None, 1)), K, y, fmt)
    assert torch.equal(y, y[:1].expand(M, N)) and B.bnn_device_status() == 0

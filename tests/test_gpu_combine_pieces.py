"""The weighted sum of the experts' results in the form that many tokens take, 16 columns a lane in two pieces of 8: rows of more than
1024 columns, and 1184 blocks of 2048 columns or more."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def env():
    import torch
    assert torch.cuda.is_available()
    from paper_1706_09453_b200 import build, binding
    build.build()
    return torch, binding


# a second piece of one lane, of nearly all, of half a block behind a whole one, whole ones; numbers of choices that end inside four
@pytest.mark.parametrize("T,k,N", [(1300, 2, 1032), (1300, 5, 2040), (700, 3, 3080), (600, 8, 4096), (1200, 1, 1536), (640, 7, 2056)])
@pytest.mark.parametrize("zt", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("yt", ["f32", "f16", "bf16"])
def test_two_pieces(env, zt, yt, T, k, N):
    torch, B = env
    types = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
    assert N > 1024 and N % 8 == 0 and T * -(-N // 2048) >= 1184
    rng = np.random.default_rng(T + k + N)
    g = torch.Generator(device=DEV)
    g.manual_seed(N)
    rows = T * k
    z = torch.randn((rows + 2, N + 8), generator=g, device=DEV).to(types[zt])
    z[:, N:] = float("nan")                         # columns that are not the matrix'
    slot = rng.permutation(rows).reshape(T, k).astype(np.int32)
    gone = rng.random((T, k)) < 0.1
    slot[gone] = rng.choice([-1, -5, rows + 2, 1 << 30], gone.sum())
    slot[5] = -1                                    # a token without any row
    weight = torch.rand((T, k), generator=g, device=DEV)
    s = torch.as_tensor(slot, device=DEV)
    there = (s >= 0) & (s < rows + 2)
    weight[~there] = float("nan")                   # a weight without a row adds nothing
    y = torch.full((T + 1, N + 8), 9.0, dtype=types[yt], device=DEV)
    B.bnn_combine_experts(z[:, :N], s, weight, y[:T, :N])
    want, mag = torch.zeros((T, N), dtype=torch.float64, device=DEV), torch.zeros((T, N), dtype=torch.float64, device=DEV)
    for j in range(k):
        term = torch.where(there[:, j:j + 1], weight[:, j:j + 1].double() * z[torch.where(there[:, j], s[:, j], 0).long(), :N].double(), 0.0)
        want += term
        mag += term.abs()
    # k fused multiply-adds, half a step of a partial sum each, and the rounding to Y's type (of fp16's subnormal numbers 2^-25)
    sums = k * 2.0 ** -24 * mag
    off = sums + (torch.finfo(types[yt]).eps / 2 * (want.abs() + sums) if yt != "f32" else 0) + (2.0 ** -25 if yt == "f16" else 0)
    assert ((y[:T, :N].double() - want).abs() <= off).all()
    assert (y[T] == 9.0).all() and (y[:, N:] == 9.0).all()
    assert (y[5, :N] == 0).all()

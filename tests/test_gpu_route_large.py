"""The router with most experts, choices and tokens: the largest masks, and counts that are summed by a kernel of their own over all of
its blocks."""
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


@pytest.mark.parametrize("T,E,k", [(90001, 1024, 32), (82000, 1001, 9), (300000, 130, 3), (76000, 1024, 32)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_route(env, dtype, T, E, k):
    torch, B = env
    g = torch.Generator(device=DEV)
    g.manual_seed(T)
    x = torch.randn((T, E), generator=g, device=DEV).to(getattr(torch, dtype))         # (bf16: many ties)
    x[torch.rand((T,), generator=g, device=DEV) < 0.05] = -float("inf")
    x[1, k // 2:] = -float("inf")                                                      # fewer than k
    i32 = dict(dtype=torch.int32, device=DEV)
    index, weight, offsets, slot, source = torch.full((T, k), -7, **i32), torch.full((T, k), -7.0, device=DEV), torch.full((E + 1,), -7, **i32), torch.full((T, k), -7, **i32), torch.full((T * k,), -1, **i32)
    n = B.bnn_route_workspace_bytes(T, E)
    ws = torch.full((n + 64,), 0xA5, dtype=torch.uint8, device=DEV)
    B.bnn_route_experts(x, index, weight, offsets, slot, source, ws[:n], B.ROUTE_SOFTMAX)
    assert (ws[n:] == 0xA5).all()
    top, want = torch.sort(x.float(), dim=-1, descending=True, stable=True)
    top, want = top[:, :k], want[:, :k]
    real = top > -float("inf")
    assert torch.equal(index, torch.where(real, want, -1).int())
    expert = torch.where(real, want, E).flatten()
    order = torch.argsort(expert, stable=True)
    place = torch.empty_like(order)
    place[order] = torch.arange(T * k, device=DEV)
    live = int(real.sum())
    assert torch.equal(offsets, torch.nn.functional.pad(torch.bincount(expert, minlength=E + 1)[:E].cumsum(0), (1, 0)).int())
    assert torch.equal(slot, torch.where(real, place.view(T, k), -1).int())
    assert torch.equal(source[:live], (order[:live] // k).int()) and (source[live:] == -1).all()
    p = torch.where(real, torch.exp(top.double() - torch.logsumexp(x.double(), -1, keepdim=True)), 0.0)
    # a term's exponent is a rounded difference (half a step of up to 2^4: 2^-20), exponentials within a few steps of 2^-22, 1024 terms in
    # more than five levels, one quotient
    assert torch.allclose(weight.double(), p, rtol=64 * 2.0 ** -23, atol=1e-30)

"""The router and the weighted sum of the experts' results against plain statements of them, and a layer that is split
into 4-bit experts, from the logits to its outputs."""
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


def run_route(torch, B, x, k, mode):
    T, E = x.shape
    i32 = dict(dtype=torch.int32, device=DEV)
    out = dict(index=torch.full((T, k), -7, **i32), weight=torch.full((T, k), -7.0, device=DEV), offsets=torch.full((E + 1,), -7, **i32),
               slot=torch.full((T, k), -7, **i32), source=torch.full((T * k,), -1, **i32))
    ws = torch.empty((B.bnn_route_workspace_bytes(T, E),), dtype=torch.uint8, device=DEV)
    B.bnn_route_experts(x, out["index"], out["weight"], out["offsets"], out["slot"], out["source"], ws, mode)
    return {n: t.cpu().numpy() for n, t in out.items()}


def check_route(torch, B, x, k):
    for mode in (B.ROUTE_SOFTMAX, B.ROUTE_SOFTMAX_CHOSEN):
        got = run_route(torch, B, x, k, mode)
        index, weight, offsets, slot, source = ref.route(x.double().cpu().numpy(), k, mode == B.ROUTE_SOFTMAX_CHOSEN)
        np.testing.assert_array_equal(got["index"], index)
        np.testing.assert_array_equal(got["offsets"], offsets)
        np.testing.assert_array_equal(got["slot"], slot)
        np.testing.assert_array_equal(got["source"], source)
        # exponent: a rounded difference (half a step of up to 2^7 moves the power by 2^-17 at most; the terms that far down
        # weigh e^-64), expf within 2 steps, up to 1024 additions in five or more levels, one quotient
        np.testing.assert_allclose(got["weight"], weight, rtol=64 * 2.0 ** -23, atol=1e-30)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 64, 8), (8, 64, 8), (3, 7, 7), (127, 33, 2), (128, 8, 1), (129, 100, 6), (700, 256, 8), (200, 1024, 32), (5000, 16, 4)])
def test_route(env, dtype, T, E, k):
    torch, B = env
    g = torch.Generator(device=DEV)
    g.manual_seed(T + E)
    x = torch.randn((T, E + 2), generator=g, device=DEV).to(dtype_of(torch, dtype))[:, 1:E + 1]
    check_route(torch, B, x, k)


@pytest.mark.parametrize("T,E,k", [(9, 40, 5), (300, 64, 4), (6000, 24, 8)])
def test_ties_and_masked_experts(env, T, E, k):
    torch, B = env
    rng = np.random.default_rng(T)
    x = rng.integers(-2, 3, (T, E)).astype(np.float32)             # many ties
    x[rng.random((T, E)) < 0.5] = -0.0                             # +0 and -0 tie as well
    x[rng.random((T, E)) < 0.3] = -np.inf
    x[rng.random(T) < 0.2] = -np.inf                               # tokens without any expert
    x[0, 3:] = -np.inf                                             # fewer than k
    check_route(torch, B, torch.as_tensor(x, device=DEV), k)
    check_route(torch, B, torch.full((T, E), -float("inf"), device=DEV), k)
    lowest = torch.full((T, E), torch.finfo(torch.float32).min, device=DEV)   # a mask of the type's lowest value is a number
    check_route(torch, B, lowest, k)


@pytest.mark.parametrize("E", [40, 256, 900])
def test_logits_that_differ_in_their_last_bits(env, E):
    """fp32 steps apart, on both sides of zero, at and around the k-th place."""
    torch, B = env
    rng = np.random.default_rng(E)
    T, k = 300, 6
    base = rng.choice(np.array([1.0, -1.0, 3.5e-3, -7.25e4], dtype=np.float32), (T, 1))
    x = (base.view(np.int32) + rng.integers(0, 40, (T, E), dtype=np.int32)).view(np.float32)
    check_route(torch, B, torch.as_tensor(x, device=DEV), k)
    h = (rng.choice(np.array([1.0, -1.0, 0.01, -300.0, 1e-6], dtype=np.float16), (T, 1)).view(np.int16) + rng.integers(0, 60, (T, E), dtype=np.int16)).view(np.float16)
    check_route(torch, B, torch.as_tensor(h, device=DEV), k)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("E", [20, 33, 100, 200, 500, 1000])
def test_logits_of_large_size(env, dtype, E):
    """Rows of masks (finite ones: -1e4, -1e9, the type's lowest value), whole and in part, and logits far above one."""
    torch, B = env
    t = dtype_of(torch, dtype)
    top = torch.finfo(t).max
    g = torch.Generator(device=DEV)
    g.manual_seed(E)
    rows = []
    for size in (1e4, 5e4, 1048575.0, 1048577.0, 1e9, 1.2345e30, top):
        if size > top:
            continue
        for sign in (1.0, -1.0):
            flat = torch.full((4, E), sign * size, device=DEV)
            flat[1, E // 2:] = 0.0
            flat[2, ::3] = torch.randn((1, flat[2, ::3].numel()), generator=g, device=DEV)[0]
            flat[3] *= 1.0 - torch.randint(0, 32, (E,), generator=g, device=DEV) * 2.0 ** -24       # steps apart
            rows.append(flat)
    check_route(torch, B, torch.cat(rows).to(t), min(E, 6))


def test_nan_and_infinity(env):
    torch, B = env
    x = torch.randn((6, 20), device=DEV)
    x[1, 4] = float("nan")
    x[2] = float("nan")
    x[4, 0] = float("nan")
    x[4, 1:] = -float("inf")
    check_route(torch, B, x, 3)
    x[3, 7] = float("inf")
    got = run_route(torch, B, x, 3, B.ROUTE_SOFTMAX)
    assert got["index"][3, 0] == 7 and np.isnan(got["weight"][3]).all()
    assert not np.isnan(got["weight"][[0, 5]]).any()


def test_many_tokens(env):
    """Beyond 81920 tokens the counts are summed by a kernel of their own."""
    torch, B = env
    T, E, k = 100003, 48, 2
    x = torch.randn((T, E), device=DEV)
    got = run_route(torch, B, x, k, B.ROUTE_SOFTMAX)
    key = x.cpu().numpy()
    index = np.argsort(-key, axis=1, kind="stable")[:, :k]
    np.testing.assert_array_equal(got["index"], index)
    order = np.argsort(index.reshape(-1), kind="stable")
    np.testing.assert_array_equal(got["source"], order // k)
    slot = np.empty(T * k, dtype=np.int64)
    slot[order] = np.arange(T * k)
    np.testing.assert_array_equal(got["slot"].reshape(-1), slot)
    np.testing.assert_array_equal(got["offsets"], np.concatenate([[0], np.cumsum(np.bincount(index.reshape(-1), minlength=E))]))


@pytest.mark.parametrize("zt,yt", [("f32", "f32"), ("f16", "f16"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "f16")])
@pytest.mark.parametrize("T,k,N", [(1, 1, 1), (3, 8, 2048), (50, 5, 1001), (7, 32, 130), (200, 2, 4096)])
def test_combine(env, zt, yt, T, k, N):
    torch, B = env
    rng = np.random.default_rng(T * k + N)
    z = torch.as_tensor(rng.normal(0, 1, (T * k + 2, N + 8)).astype(np.float32), device=DEV).to(dtype_of(torch, zt))
    slot = rng.permutation(T * k).reshape(T, k).astype(np.int32)
    slot[rng.random((T, k)) < 0.1] = -1
    slot[0, 0] = T * k + 2 if T > 1 else 0          # behind the last row
    weight = rng.random((T, k)).astype(np.float32)
    weight[slot < 0] = np.nan                       # a weight without a row adds nothing
    for first, cols in ((0, N), (3, N)):            # rows that start anywhere
        y = torch.full((T, N + 8), 9.0, dtype=dtype_of(torch, yt), device=DEV)
        B.bnn_combine_experts(z[:, first:first + cols], torch.as_tensor(slot, device=DEV), torch.as_tensor(weight, device=DEV), y[:, :N])
        zs = z[:, first:first + cols].double().cpu().numpy()
        ok = (slot >= 0) & (slot < zs.shape[0])
        terms = np.where(ok, weight, 0.0)[..., None].astype(np.float64) * np.where(ok[..., None], zs[np.where(ok, slot, 0)], 0.0)
        want, mag = terms.sum(1), np.abs(terms).sum(1)
        got = y.double().cpu().numpy()
        # k fused multiply-adds, half a step of a partial sum each, and the rounding to Y's type
        off = k * 2.0 ** -24 * mag + torch.finfo(y.dtype).eps / 2 * (np.abs(want) + k * 2.0 ** -24 * mag) + 1e-7 * (yt == "f16")
        assert (np.abs(got[:, :N] - want) <= off).all()
        assert (got[:, N:] == 9.0).all()


def test_combine_rows_further_apart_than_32_bits_hold(env):
    torch, B = env
    far, N = 1 << 30, 264
    z = torch.randn((3, N), device=DEV).to(torch.bfloat16)
    apart = torch.empty((2 * far + N,), dtype=torch.bfloat16, device=DEV).as_strided((3, N), (far, 1))
    apart.copy_(z)
    slot = torch.tensor([[2, 0], [1, 2], [0, -1]], dtype=torch.int32, device=DEV)
    weight = torch.rand((3, 2), device=DEV)
    want = B.bnn_combine_experts(z, slot, weight, torch.empty((3, N), dtype=torch.bfloat16, device=DEV))
    assert torch.equal(B.bnn_combine_experts(apart, slot, weight, torch.empty_like(want)), want)
    out = torch.empty((2 * far + N,), dtype=torch.bfloat16, device=DEV).as_strided((3, N), (far, 1))
    assert torch.equal(B.bnn_combine_experts(z, slot, weight, out), want)


def experts_layer(torch, B, s):
    """A layer of experts as a program runs it: route, gather and quantise, two products by expert, bring the results back."""
    B.bnn_route_experts(s["logits"], s["index"], s["weight"], s["offsets"], s["slot"], s["source"], s["workspace"], B.ROUTE_SOFTMAX_CHOSEN)
    B.bnn_f4_quantize(s["x"], s["a"], s["a_scales"], s["fmt"], source=s["source"], offsets=s["offsets"])
    B.bnn_f4_gemm_grouped(s["a"], s["a_scales"], s["offsets"], s["w1"], s["w1_scales"], s["K"], s["h"], s["fmt"], act=B.ACT_HARDTANH)
    B.bnn_f4_quantize(s["h"], s["b"], s["b_scales"], s["fmt"], offsets=s["offsets"])
    B.bnn_f4_gemm_grouped(s["b"], s["b_scales"], s["offsets"], s["w2"], s["w2_scales"], s["H"], s["z"], s["fmt"])
    return B.bnn_combine_experts(s["z"], s["slot"], s["weight"], s["y"])


def make_layer(torch, B, fmt, T, E, k, K, H, N, seed=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    R, u8, i32 = T * k, dict(dtype=torch.uint8, device=DEV), dict(dtype=torch.int32, device=DEV)
    s = dict(fmt=fmt, K=K, H=H, x=torch.randn((T, K), generator=g, device=DEV).to(torch.bfloat16), logits=torch.randn((T, E), generator=g, device=DEV),
             index=torch.zeros((T, k), **i32), weight=torch.zeros((T, k), device=DEV), offsets=torch.zeros((E + 1,), **i32), slot=torch.zeros((T, k), **i32),
             source=torch.zeros((R,), **i32), workspace=torch.empty((B.bnn_route_workspace_bytes(T, E),), **u8),
             a=torch.zeros((R, B.bnn_f4_pitch(K)), **u8), a_scales=torch.zeros((B.bnn_f4_scale_bytes(fmt, R, K, E),), **u8),
             b=torch.zeros((R, B.bnn_f4_pitch(H)), **u8), b_scales=torch.zeros((B.bnn_f4_scale_bytes(fmt, R, H, E),), **u8),
             h=torch.zeros((R, H), device=DEV), z=torch.zeros((R, N), dtype=torch.bfloat16, device=DEV), y=torch.zeros((T, N), device=DEV))
    s["logits"][T // 3] = -float("inf")          # a padded position
    for name, n, width in (("w1", H, K), ("w2", N, H)):
        w = torch.randn((E * n, width), generator=g, device=DEV) / 16
        s[name + "_full"] = w.view(E, n, width)
        codes, scales = torch.zeros((E * n, B.bnn_f4_pitch(width)), **u8), torch.zeros((B.bnn_f4_scale_bytes(fmt, E * n, width, E),), **u8)
        B.bnn_f4_quantize(w, codes, scales, fmt, offsets=torch.arange(E + 1, **i32) * n)
        s[name], s[name + "_scales"] = codes.view(E, n, -1), scales
    return s


def layer_reference(s, T, E, k, fmt):
    """The same in 64 bits, from what the GPU's quantiser is held to elsewhere."""
    def q(v):
        return ref.values(*ref.quantize(v, fmt), fmt, v.shape[1])
    index, weight, _, _, _ = ref.route(s["logits"].double().cpu().numpy(), k, True)
    x, y = q(s["x"].double().cpu().numpy()), np.zeros(tuple(s["y"].shape))
    w1, w2 = (np.stack([q(w) for w in s[n].double().cpu().numpy()]) for n in ("w1_full", "w2_full"))
    for t in range(T):
        for j in range(k):
            e = index[t, j]
            if e >= 0:
                h = np.clip(x[t] @ w1[e].T, -1, 1).astype(np.float32).astype(np.float64)
                y[t] += weight[t, j] * (q(h[None])[0] @ w2[e].T)
    return y


@pytest.mark.parametrize("fmt", [ref.MX, ref.NV])
@pytest.mark.parametrize("T", [1, 6, 90])
def test_a_layer_of_experts(env, fmt, T):
    torch, B = env
    E, k, K, H, N = 12, 3, 200, 264, 136
    s = make_layer(torch, B, fmt, T, E, k, K, H, N, seed=T)
    got = experts_layer(torch, B, s).double().cpu().numpy()
    want = layer_reference(s, T, E, k, fmt)
    # A hidden value whose fp32 sum lies next to a border between two codes may take the other one, which moves an output by
    # a code's step of one of 264 terms; all else is the bf16 rounding of z.  Together well below 2 % of an output's spread.
    assert np.linalg.norm(got - want) <= 0.02 * np.linalg.norm(want) + 1e-12
    assert (got[T // 3] == 0).all()
    assert B.bnn_device_status() == 0


def test_captured_and_replayed_beside_another(env):
    """Two layers captured into graphs, replayed on new inputs on two streams, equal to what eager calls give."""
    torch, B = env
    sizes = dict(E=12, k=3, K=200, H=264, N=136)
    one, two = make_layer(torch, B, ref.MX, 40, seed=1, **sizes), make_layer(torch, B, ref.NV, 200, seed=2, **sizes)
    graphs = []
    for s in (one, two):
        experts_layer(torch, B, s)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            experts_layer(torch, B, s)
        graphs.append(g)
    for turn in range(3):
        for s in (one, two):
            s["x"].normal_()
            s["logits"].normal_()
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        torch.cuda.synchronize()
        for s in (one, two):
            replayed = s["y"].clone()
            s["y"].zero_()
            assert torch.equal(experts_layer(torch, B, s), replayed)
    assert B.bnn_device_status() == 0


def test_on_another_stream(env):
    torch, B = env
    s = make_layer(torch, B, ref.MX, 30, 12, 3, 200, 264, 136)
    want = experts_layer(torch, B, s).clone()
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    for _ in range(5):
        s["y"].zero_()
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            experts_layer(torch, B, s)
        torch.cuda.current_stream().wait_stream(st)
        assert torch.equal(s["y"], want)

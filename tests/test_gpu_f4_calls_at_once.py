"""Calls from several host threads at once, each on a stream of its own, and a first call in a process that has not used the GPU yet."""
import subprocess
import sys
import threading

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


def test_threads(env):
    torch, B = env
    sizes = [(1, 700, 2048, ref.MX), (90, 900, 700, ref.NV), (731, 3307, 512, ref.MX), (40, 300, 1100, ref.NV)]
    u8 = dict(dtype=torch.uint8, device=DEV)
    work = []
    for i, (M, N, K, fmt) in enumerate(sizes):
        g = torch.Generator(device=DEV)
        g.manual_seed(i)
        xs = [torch.randn((M, K), generator=g, device=DEV).to(torch.bfloat16) for _ in range(8)]
        w = torch.randn((N, K), generator=g, device=DEV)
        mats = [(torch.zeros((r, B.bnn_f4_pitch(K)), **u8), torch.zeros((B.bnn_f4_scale_bytes(fmt, r, K),), **u8)) for r in (M, N)]
        B.bnn_f4_quantize(w, *mats[1], fmt)

        def layer(x, y, K=K, fmt=fmt, a=mats[0], w=mats[1]):
            B.bnn_f4_quantize(x, *a, fmt)
            return B.bnn_f4_gemm(*a, *w, K, y, fmt)
        want = [layer(x, torch.empty((M, N), device=DEV)) for x in xs]
        work.append((layer, xs, want, [torch.empty((M, N), device=DEV) for _ in xs], torch.cuda.Stream()))
    torch.cuda.synchronize()
    failed = []

    def go(layer, xs, want, ys, stream):
        try:
            with torch.cuda.stream(stream):
                for _ in range(20):
                    for x, y in zip(xs, ys):
                        layer(x, y)
        except Exception as e:      # a thread's exception does not reach the test by itself
            failed.append(e)
    threads = [threading.Thread(target=go, args=w) for w in work]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed
    for layer, xs, want, ys, stream in work:
        assert all(torch.equal(y, v) for y, v in zip(ys, want))
    assert B.bnn_device_status() == 0


def test_a_first_call_without_any_use_of_the_gpu_before(env):
    code = "from paper_1706_09453_b200 import binding as B; B.bnn_reset_status(); print(B.bnn_device_status())"
    out = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=120)
    assert out.returncode == 0 and out.stdout.strip() == "0", out.stderr[-500:]

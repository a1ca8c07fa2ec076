"""Which form a product of quantised matrices takes, from its sizes and the number of SMs (no GPU)."""
import pytest

SMS = 148


@pytest.fixture(scope="module")
def B():
    from paper_1706_09453_b200 import build, binding
    build.build()
    return binding


def test_forms_of_ordinary_sizes(B):
    for M, N, K, groups, form in (
            (1, 2048, 2048, 0, (1, 32, 4)), (1, 2048, 256, 0, (1, 32, 1)), (1, 2048, 512, 0, (1, 32, 2)), (5, 19000, 8192, 0, (1, 32, 1)),
            (64, 2048, 2048, 0, (1, 128, 1)), (731, 3307, 2048, 0, (2, 192, 1)), (8192, 8192, 4096, 0, (2, 256, 1)),
            (64, 2048, 2048, 64, (1, 128, 1)), (16384, 4096, 2048, 32, (2, 256, 1)), (20, 500, 2048, 4, (1, 32, 4))):
        assert B.bnn_f4_gemm_form(M, N, K, groups, SMS) == form, (M, N, K, groups)
    assert B.bnn_f4_gemm_form(8192, 8192, 4096, 0, 1)[0] == 1           # one SM makes no pair


def test_refusals(B):
    good = dict(M=10, N=20, K=30, groups=0, sms=SMS)
    form = (B.C.c_int * 3)()
    assert B.raw_call("bnn_f4_gemm_form", *good.values(), form) == 0
    assert B.raw_call("bnn_f4_gemm_form", *good.values(), None) == 1
    for bad in (dict(M=0), dict(N=0), dict(K=0), dict(K=(1 << 24) + 1), dict(groups=-1), dict(groups=1025), dict(sms=-1), dict(M=0x7FFFFFFF), dict(N=0x7FFFFFFF)):
        assert B.raw_call("bnn_f4_gemm_form", *{**good, **bad}.values(), form) == 2, bad


@pytest.mark.parametrize("N,K", [(2048, 2048), (4096, 4096), (8192, 8192), (2048, 8192), (1000, 700)])
def test_no_step_at_thirty_two_rows(B, N, K):
    """All of 17 to 32 rows are one tile, and share its K between as many CTAs."""
    forms = {B.bnn_f4_gemm_form(M, N, K, 0, SMS) for M in range(17, 33)}
    assert len(forms) == 1, forms
    assert B.bnn_f4_gemm_form(32, N, K, 1, SMS) == B.bnn_f4_gemm_form(31, N, K, 1, SMS) in forms


def test_few_rows_share_k_wherever_it_leaves_no_tile_waiting(B):
    for N in range(128, 20000, 331):
        tiles = -(-N // 128)
        want = 4 if tiles * 4 <= SMS else 2 if tiles * 2 <= SMS else 1
        for M in (1, 16, 31, 32):
            assert B.bnn_f4_gemm_form(M, N, 4096, 0, SMS) == (1, 32, want), (M, N)

"""What the binding hands to the operators on 4-bit floating point when its tensors are views whose rows are shorter than the kernels
take: a pitch alone does not show that the last row ends inside its buffer.  No GPU: the calls' own words are checked."""
import pytest
import torch


@pytest.fixture
def B(monkeypatch):
    from paper_1706_09453_b200 import build, binding
    build.build()
    monkeypatch.setattr(binding, "_get_device", lambda: -1)      # where CPU tensors lie
    monkeypatch.setattr(binding, "_stream", lambda: 0)
    monkeypatch.setattr(binding, "_ptr", lambda t, dtype=None: None if t is None else t.data_ptr())
    return binding


class Seen(Exception):
    pass


def words_of(monkeypatch, B, name, call):
    """The words that a call would hand over (nothing runs)."""
    def seen(self, *args):
        assert self.name == name
        raise Seen(args)
    monkeypatch.setattr(B._Call, "__call__", seen)
    with pytest.raises(Seen) as e:
        call()
    return e.value.args[0]


SHAPE = 2


def u8(*shape):
    return torch.zeros(shape, dtype=torch.uint8)


def cases(B):
    """(entry point, call with codes `c` [40][..] in the place in question, the pitch's place among the words), K = 100: 64 bytes"""
    K, x, s, y = 100, torch.zeros((40, 100)), u8(4096), torch.zeros((40, 40))
    good = u8(40, 64)
    off = torch.zeros((3,), dtype=torch.int32)
    return [
        ("bnn_f4_quantize", lambda c: B.bnn_f4_quantize(x, c, s), 12),
        ("bnn_f4_dequantize", lambda c: B.bnn_f4_dequantize(c, s, x), 1),
        ("bnn_f4_gemm", lambda c: B.bnn_f4_gemm(c, s, good, s, K, y), 1),
        ("bnn_f4_gemm", lambda c: B.bnn_f4_gemm(good, s, c, s, K, y), 5),
        ("bnn_f4_gemm_grouped", lambda c: B.bnn_f4_gemm_grouped(c, s, off, good.view(2, 20, 64), s, K, y[:, :20]), 1),
        ("bnn_f4_gemm_grouped", lambda c: B.bnn_f4_gemm_grouped(good, s, off, c.unflatten(0, (2, 20)), s, K, y[:, :20]), 7),
    ]


@pytest.mark.parametrize("case", range(6))
@pytest.mark.parametrize("width", [16, 48, 63])
def test_codes_whose_rows_are_shorter_than_k(B, monkeypatch, case, width):
    name, call, at = cases(B)[case]
    whole = u8(40, 128)
    assert words_of(monkeypatch, B, name, lambda: call(whole))[at] == 128
    assert words_of(monkeypatch, B, name, lambda: call(whole[:, 64:]))[at] == 128       # long enough, further apart
    monkeypatch.undo()
    monkeypatch.setattr(B, "_get_device", lambda: -1)
    monkeypatch.setattr(B, "_stream", lambda: 0)
    with pytest.raises(B.BnnError) as e:
        call(whole[:, 128 - width:])       # 128 bytes apart, but the last row ends behind `width`
    assert e.value.status == SHAPE


@pytest.mark.parametrize("grouped", [False, True])
def test_bits_whose_rows_are_shorter_than_the_units(B, monkeypatch, grouped):
    K, s, a, n = 100, u8(4096), u8(40, 64), 40           # 40 units: two words
    bits = torch.zeros((40, 8), dtype=torch.int32)
    off = torch.zeros((2,), dtype=torch.int32)

    def call(out):
        if grouped:
            B.bnn_f4_gemm_grouped(a, s, off, a.view(1, n, 64), s, K, None, act=B.ACT_SIGN_PACK, out_bits=out)
        else:
            B.bnn_f4_gemm(a, s, a, s, K, None, act=B.ACT_SIGN_PACK, out_bits=out)
    name = "bnn_f4_gemm_grouped" if grouped else "bnn_f4_gemm"
    for out in (bits, bits[:, 4:], bits[:, 4:6]):
        words_of(monkeypatch, B, name, lambda: call(out))
    for out in (bits[:, 7:], bits[:39], bits[0]):
        with pytest.raises(ValueError):
            call(out)

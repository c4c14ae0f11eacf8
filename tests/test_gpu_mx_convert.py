"""What the mxfp4 cache's kernels take of the E2M1 conversions of gfx950 (tests/probes/mx_probe.hip):
a code's value times a power of two is exact in bf16 and fp32, only the exponent of the scale counts
and 255 gives NaN, and a bf16 value divided by a power of two rounds to the nearest code, ties to the even one, saturating at 6."""
import ctypes
import os

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
LIB = os.path.join(os.path.dirname(os.path.abspath(__file__)), "probes", "libmxprobe.so")
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
VALUES = np.concatenate([E2M1, -E2M1])


def _lib():
    assert os.path.exists(LIB), "tests/probes/libmxprobe.so is not built (run __graft_entry__.build())"
    lib = ctypes.CDLL(LIB)
    lib.vxt_from_e2m1.argtypes = [ctypes.c_void_p] * 4 + [ctypes.c_int, ctypes.c_void_p]
    lib.vxt_to_e2m1.argtypes = [ctypes.c_void_p] * 3 + [ctypes.c_int, ctypes.c_void_p]
    return lib


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _bf16(bits):
    return (bits.astype(np.uint32) << 16).view(np.float32).astype(np.float64)


def _widen(codes, scale_bits):
    c = torch.from_numpy(codes.astype(np.uint32).view(np.int32)).cuda()
    s = torch.from_numpy(scale_bits.astype(np.uint32).view(np.float32)).cuda()
    pairs = torch.zeros((len(codes), 2), dtype=torch.int32, device="cuda")
    vals = torch.zeros((len(codes), 2), dtype=torch.float32, device="cuda")
    assert _lib().vxt_from_e2m1(c.data_ptr(), s.data_ptr(), pairs.data_ptr(), vals.data_ptr(), len(codes), _stream()) == 0
    torch.cuda.synchronize()
    p = pairs.cpu().numpy().view(np.uint32)
    halves = np.stack([_bf16(p & 0xFFFF), _bf16(p >> 16)], -1)          # [n][byte 0, byte 3][low, high nibble]
    return halves, vals.cpu().numpy().astype(np.float64)


def test_every_code_at_every_scale_is_exact():
    byte, e = np.meshgrid(np.arange(256), np.arange(8, 253), indexing="ij")
    byte, e = byte.ravel(), e.ravel()
    halves, vals = _widen(byte | byte << 8 | (255 - byte) << 24, e << 23)
    scale = np.exp2(e - 127.0)[:, None]
    want = lambda b: np.stack([VALUES[b & 15], VALUES[b >> 4]], -1) * scale  # noqa: E731
    assert np.array_equal(halves[:, 0], want(byte)) and np.array_equal(halves[:, 1], want(255 - byte))
    assert np.array_equal(vals, want(byte))


@pytest.mark.parametrize("bits", [0x7F800000, 0x7FC00000, 0x7F812345, 0xFF800000, 0xFFFFFFFF])
def test_an_exponent_of_255_gives_nan(bits):
    byte = np.arange(256)
    halves, vals = _widen(byte * 0x01010101, np.full(256, bits))
    assert np.isnan(halves).all() and np.isnan(vals).all()


@pytest.mark.parametrize("bits", [0x3F800001, 0x3FC00000, 0x3FFFFFFF, 0xBF800000, 0xBFFFFFFF])
def test_only_the_exponent_of_a_scale_counts(bits):
    byte = np.arange(256)
    halves, vals = _widen(byte * 0x01010101, np.full(256, bits))
    one, one_vals = _widen(byte * 0x01010101, np.full(256, 0x3F800000))
    assert np.array_equal(halves, one) and np.array_equal(vals, one_vals)


def test_codes_round_to_nearest_even_and_saturate():
    bits = np.arange(0, 0x7F80, dtype=np.uint32)                        # every finite non-negative bf16 value
    for e in (8, 60, 120, 127, 130, 200, 252):
        x = _bf16(bits) / 2.0 ** (e - 127)
        a = np.minimum(x, 6.0)
        step = np.where(a < 2, 0.5, np.where(a < 4, 1.0, 2.0))
        want = np.searchsorted(E2M1, np.rint(a / step) * step)
        pairs = torch.from_numpy((bits | (bits | 0x8000) << 16).view(np.int32)).cuda()
        s = torch.full((len(bits),), float(2.0 ** (e - 127)), dtype=torch.float32, device="cuda")
        out = torch.zeros(len(bits), dtype=torch.int32, device="cuda")
        assert _lib().vxt_to_e2m1(pairs.data_ptr(), s.data_ptr(), out.data_ptr(), len(bits), _stream()) == 0
        torch.cuda.synchronize()
        got = out.cpu().numpy().view(np.uint32)
        assert (got & 0xFF00FFFF == 0x11001111).all()
        assert np.array_equal((got >> 16) & 15, want), e
        assert np.array_equal((got >> 20) & 15, want + 8), e

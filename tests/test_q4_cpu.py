"""The 4-bit cache without a GPU: the oracle's quantiser against exact arithmetic and closed forms, the row layout, and the
refusals that the host makes before it touches a device."""
import ctypes
from fractions import Fraction

import numpy as np
import pytest

from oracle import rap_oracle as O
from paper_2602_02599_b200 import binding, build

import q4_util


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding._lib()


def test_row_bytes_and_layout(lib):
    for W in range(1, 257):
        n = binding.rap_q4_row_bytes(W)
        assert n == 4 * q4_util.row_words(W) and (n // 4) % 2 == 1 and n >= (W + 1) // 2 + 4 and n < (W + 1) // 2 + 4 + 8 + 3
    assert [binding.rap_q4_row_bytes(W) for W in (90, 64, 128, 115, 48, 256)] == [52, 36, 68, 68, 28, 132]
    assert binding.rap_q4_row_bytes(0) == 0 and binding.rap_q4_row_bytes(-3) == 0
    assert O.kv_bytes_per_token_q4(32, 8, 90, 90) == 32 * 8 * (52 + 52)
    rng = np.random.default_rng(1)
    for W in (1, 2, 7, 90, 115, 256):
        x = rng.normal(0, 1, (5, W)).astype(np.float32)
        held = O.quantize_rows_q4(x)
        back = q4_util.unpack(q4_util.pack(*held), W)
        assert all(np.array_equal(a, b) for a, b in zip(held, back))


def _bf16(v):
    """Fraction -> nearest bf16 as a Fraction, ties to even (normal range)."""
    if v == 0:
        return Fraction(0)
    a, e = abs(v), 0
    while a >= 2:
        a, e = a / 2, e + 1
    while a < 1:
        a, e = a * 2, e - 1
    m = a * 128
    n = m.numerator // m.denominator
    r = m - n
    if r > Fraction(1, 2) or (r == Fraction(1, 2) and n % 2):
        n += 1
    return (1 if v > 0 else -1) * Fraction(n, 128) * (Fraction(2) ** e)


def test_quantiser_against_exact_arithmetic():
    """Middle, step and codes by rational arithmetic (bf16 inputs, so hi / 2 + lo / 2 and the differences are exact but for
    their fp32 rounding, which numpy does); a code next to a border may go either way, no other may."""
    rng = np.random.default_rng(2)
    for x in (O.round_bf16(rng.normal(m, 1, (40, 23))).astype(np.float32) for m in (0.0, 3.0, -40.0)):
        codes, s, z = O.quantize_rows_q4(x)
        for row, c, step, mid in zip(x, codes, s, z):
            f = [Fraction(float(v)) for v in row]
            assert Fraction(mid) == _bf16(Fraction(float(np.float32(float((max(f) + min(f)) / 2)))))
            reach = max(max(f) - Fraction(mid), Fraction(mid) - min(f))
            assert Fraction(step) == _bf16(Fraction(float(np.float32(float(reach)) / np.float32(7.5))))
            for v, k in zip(f, c):
                place = (v - Fraction(mid)) / Fraction(step) + Fraction(15, 2)
                near = abs(place - int(k))
                assert near <= Fraction(1, 2) + Fraction(1, 2 ** 18)


def test_quantiser_round_trip_and_special_rows():
    rng = np.random.default_rng(3)
    x = (rng.normal(0, 1, (200, 90)) * rng.lognormal(0, 3, (200, 1)) + rng.normal(0, 5, (200, 1))).astype(np.float32)
    codes, s, z = O.quantize_rows_q4(x)
    assert codes.max() <= 15 and codes.min() == 0
    # half a step, and the fp32 rounding of the place (its largest terms are 7.5 and (x - z) / s)
    assert np.all(np.abs(O.dequantize_rows_q4(codes, s, z) - x) <= s[:, None] * (0.5 + 2.0 ** -18))
    # a power of two moves middle and step along and leaves the codes
    c2, s2, z2 = O.quantize_rows_q4(x * np.float32(8))
    assert np.array_equal(c2, codes) and np.array_equal(s2, 8 * s) and np.array_equal(z2, 8 * z)
    # a row of one bf16 number reads back as it, a zero row as zero
    for v in (0.0, -0.5, 3.0):
        c, s1, z1 = O.quantize_rows_q4(np.full((1, 7), v))
        assert s1 == 0 and z1 == v and np.all(c == 8) and np.all(O.dequantize_rows_q4(c, s1, z1) == v)
    # steps too small to be normal numbers count as zero
    c, s1, z1 = O.quantize_rows_q4(np.array([[2.0 ** -126, -2.0 ** -126]]))
    assert s1 == 0 and z1 == 0 and np.all(c == 8)
    # rows without a form
    for bad in (np.nan, np.inf, -np.inf):
        c, s1, z1 = O.quantize_rows_q4(np.array([[1.0, bad, 2.0]]))
        assert np.isnan(s1) and np.isnan(z1) and np.all(c == 8)
    c, s1, z1 = O.quantize_rows_q4(np.array([[3e38, -3e38]]))       # the differences are still inside fp32
    assert np.isfinite(s1) and z1 == 0 and c.tolist() == [[15, 0]]
    assert np.isnan(O.quantize_rows_q4(np.array([[3.4e38, 3.4e38]]))[1])      # the middle is not a bf16 number


def test_k_rotation_as_the_append_defines_it():
    """Against complex arithmetic in fp64: three roundings to fp32 and that of the sine, each half a step of at most the pair's
    length; positions far out; and a quarter turn is exact up to the cosine of the fp64 angle."""
    rng = np.random.default_rng(3)
    y = rng.normal(0, 2, (50, 2, 18)).astype(np.float32)
    pos, freq = rng.integers(0, 10 ** 6, 50), 500000.0 ** (-rng.random((2, 9)))
    z = (y[..., 0::2] + 1j * y[..., 1::2].astype(np.complex128)) * np.exp(1j * (pos[:, None, None] * freq))
    got = O.rotate_k_q4(y, pos, freq)
    off = np.abs(got[..., 0::2] + 1j * got[..., 1::2].astype(np.complex128) - z)
    assert got.dtype == np.float32 and np.all(off <= 4 * 2.0 ** -24 * 2 * np.abs(z))
    got = O.rotate_k_q4(np.array([[[3.0, -5.0]]]), [1], [[np.pi / 2]])
    assert np.allclose(got, [5.0, 3.0], rtol=2.0 ** -22, atol=0)


def test_attention_closed_forms():
    rng = np.random.default_rng(4)
    B, Hkv, G, cap, P2, dv, D = 2, 2, 2, 8, 6, 5, 8
    K, V = rng.normal(0, 1, (B, Hkv, cap, P2)), rng.normal(1, 2, (B, Hkv, cap, dv))
    kh, vh = O.quantize_rows_q4(K), O.quantize_rows_q4(V)
    q = rng.normal(0, 1, (B, Hkv * G, P2))
    Vd = O.dequantize_rows_q4(*vh)
    out = O.decode_attn_q4(q, kh, vh, [1, 3], D)
    assert np.allclose(out[0], np.repeat(Vd[0, :, 0], G, axis=0), rtol=0, atol=1e-15)
    for a in kh:
        a[1, :, 1:3] = a[1, :, :1]                  # equal K rows: the mean of the V rows
    out = O.decode_attn_q4(q, kh, vh, [1, 3], D)
    assert np.allclose(out[1], np.repeat(Vd[1, :, :3].mean(1), G, axis=0), rtol=0, atol=1e-14)


def test_host_refusals_before_any_device_call(lib):
    """Arguments are checked on the host first: a context whose device side never came up is enough to see it."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present: the GPU tests make these calls on a whole context")
    desc = binding.rap_model_desc(1, 256, 4, 2, 64, 10000.0, 0, binding.RAP_BF16, 4, 4)
    ctx = ctypes.c_void_p()
    assert lib.rap_create(ctypes.byref(desc), ctypes.byref(ctx)) == binding.RAP_ECUDA
    try:
        a, b, odd = 4096, 8192, 4100
        for f in (lib.rap_quantize_rows_q4, lib.rap_dequantize_rows_q4):
            assert f(None, 1, 1, 90, a, b, None) == binding.RAP_EINVAL
            assert f(ctx, 1, 1, 90, None, b, None) == binding.RAP_EINVAL and f(ctx, 1, 1, 90, a, None, None) == binding.RAP_EINVAL
            assert f(ctx, 2, 1, 90, a, b, None) == binding.RAP_EINVAL and f(ctx, 1, -1, 90, a, b, None) == binding.RAP_EINVAL
            assert f(ctx, 1, 1, 0, a, b, None) == binding.RAP_EINVAL and f(ctx, 1, 1, 257, a, b, None) == binding.RAP_ESHAPE
            assert f(ctx, 1, 1, 90, odd, b, None) == binding.RAP_EALIGN and f(ctx, 1, 1, 90, a, odd, None) == binding.RAP_EALIGN
            assert f(ctx, 1, 1 << 35, 90, a, b, None) == binding.RAP_ESHAPE
        # no tables yet
        assert lib.rap_decode_attn_q4(ctx, 0, 1, a, a, a, 8, a, 8, 0, a, None) == binding.RAP_ESTATE
        assert lib.rap_read_cache_q4(ctx, 0, 1, a, a, 8, a, 8, a, a, None) == binding.RAP_ESTATE
        assert lib.rap_qkv_rope_append_q4(ctx, 0, 1, a, a, None, a, a, a, 0, a, a, a, a, 1, 8, None) == binding.RAP_ESTATE
        assert lib.rap_decode_attn_q4(ctx, 0, 1, None, a, a, 8, a, 8, 0, a, None) == binding.RAP_EINVAL
    finally:
        lib.rap_destroy(ctx)


def test_conversions_refuse_buffers_that_overlap(lib):
    import torch
    if torch.cuda.is_available():
        pytest.skip("a GPU is present: the GPU tests make these calls on a whole context")
    desc = binding.rap_model_desc(1, 256, 4, 2, 64, 10000.0, 0, binding.RAP_BF16, 4, 4)
    ctx = ctypes.c_void_p()
    assert lib.rap_create(ctypes.byref(desc), ctypes.byref(ctx)) == binding.RAP_ECUDA
    try:
        rows, a = 100, 1 << 20
        wide, narrow = rows * 90 * 2, rows * 52
        for f in (lib.rap_quantize_rows_q4, lib.rap_dequantize_rows_q4):
            first, second = (wide, narrow) if f is lib.rap_quantize_rows_q4 else (narrow, wide)
            # (no device: a call that passes the checks ends at the question for the current device)
            for b, clear in ((a, False), (a + first - first % 16 - 16, False), (a + first + 16 - first % 16, True),
                             (a - second + second % 16 + 16, False), (a - second - 16 + second % 16, True)):
                s = f(ctx, binding.RAP_BF16, rows, 90, a, b // 16 * 16, None)
                assert s == (binding.RAP_ECUDA if clear else binding.RAP_EINVAL), (b - a, s)
    finally:
        lib.rap_destroy(ctx)

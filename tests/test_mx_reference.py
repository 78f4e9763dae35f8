"""The plain 4-bit numbers of block_reference against a search over all held values, and the host-side refusals of the 4-bit calls."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2502_16927_amd import binding as B
import block_reference as R


def test_nearest_of_all_held_values():
    rng = np.random.default_rng(1)
    v = rng.standard_normal((40, 32)) * np.exp2(rng.integers(-40, 40, (40, 1)))
    codes, scales, values = R.quantise(v)
    for row, c, s, got in zip(v, codes, scales, values):
        top = np.abs(row).max()
        assert s[0] == int(np.floor(np.log2(top))) - 2 + 127
        every = np.concatenate([-R.HELD, R.HELD]) * 2.0 ** (int(s[0]) - 127)
        assert np.array_equal(np.abs(row - got), np.abs(row[:, None] - every).min(1))
        assert np.array_equal(got, np.where(c & 8, -1, 1) * R.HELD[c & 7] * 2.0 ** (int(s[0]) - 127))
    assert np.array_equal(R.quantise(values)[2], values)
    ties = np.zeros(32)
    ties[:8] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.9]
    assert list(R.quantise(ties)[0][:8]) == [0, 2, 2, 4, 4, 6, 6, 7]


def test_sizes_and_refusals():
    L = B.lib()
    fake = ctypes.c_void_p(4096)                 # never dereferenced
    assert [B.mx_scale_bytes(c) for c in (32, 256, 288, 1024)] == [8, 8, 16, 32] and B.mx_scale_bytes(0) == 0 and B.mx_scale_bytes(-5) == 0
    assert B.mx_packed_bytes(2, 320, 64) == 2 * 320 * 64 // 2 + 2 * 2 * 2 * 256
    for bad in ((0, 64, 64), (1, 32, 64), (1, 64, 96), (1, 100, 64), (1025, 64, 64), (1, 1 << 25, 64)):
        assert B.mx_packed_bytes(*bad) == 0
        code = -5 if bad[0] > 1024 or bad[1] > 1 << 24 else -1
        assert L.bigmac_mx_pack(*bad, B.BF16, fake, fake, None) == code and L.bigmac_mx_unpack(*bad, fake, B.BF16, fake, None) == code
        assert L.bigmac_mx_product(ctypes.byref(B.make_mx_dims(5, *bad)), fake, fake, fake, fake, None, fake, fake, 1 << 40, None) == code
    for rows, cols, dtype, code in ((0, 32, 1, -1), (-1, 32, 1, -1), (1, 0, 1, -1), (1, 48, 1, -1), (1, 32, 2, -1), (1 << 31, 32, 1, -5), (1, (1 << 24) + 32, 1, -5)):
        assert L.bigmac_mx_quantize(rows, cols, dtype, fake, fake, fake, None) == code
        assert L.bigmac_mx_dequantize(rows, cols, fake, fake, dtype, fake, None) == code
    odd = ctypes.c_void_p(4100)
    for args in ((None, fake, fake), (fake, None, fake), (fake, fake, None), (odd, fake, fake), (fake, odd, fake), (fake, fake, odd)):
        assert L.bigmac_mx_quantize(1, 32, 1, *args, None) == -1
        assert L.bigmac_mx_dequantize(1, 32, *args[:2], 1, args[2], None) == -1
    for args in ((None, fake), (fake, None), (odd, fake), (fake, odd)):
        assert L.bigmac_mx_pack(1, 64, 64, 1, *args, None) == -1 and L.bigmac_mx_unpack(1, 64, 64, args[0], 1, args[1], None) == -1
    assert L.bigmac_mx_pack(1, 64, 64, 2, fake, fake, None) == -1

    def product(d, codes=fake, scales=fake, offsets=fake, packed=fake, bias=None, out=fake, ws=fake, ws_bytes=1 << 40):
        return L.bigmac_mx_product(ctypes.byref(d), codes, scales, offsets, packed, bias, out, ws, ws_bytes, None)

    d = B.make_mx_dims(100, 4, 128, 64)
    assert B.mx_workspace_bytes(d) > 0 and B.mx_workspace_bytes(B.make_mx_dims(0, 4, 128, 64)) == 0 and B.mx_workspace_bytes(B.make_mx_dims(1, 4, 128, 64, 3)) == 0
    for bad in (dict(codes=None), dict(scales=None), dict(offsets=None), dict(packed=None), dict(out=None), dict(ws=None), dict(codes=odd), dict(bias=odd), dict(out=odd), dict(ws=odd)):
        assert product(d, **bad) == -1, bad
    assert product(d, ws_bytes=B.mx_workspace_bytes(d) - 1) == -2
    assert product(B.make_mx_dims((1 << 30) + 1, 1, 64, 64)) == -5 and product(B.make_mx_dims(1 << 30, 1, 64, 1 << 20)) == -5    # rows; workgroups
    assert product(B.make_mx_dims(0, 4, 128, 64)) == -1 and product(B.make_mx_dims(9, 4, 128, 64, 2)) == -1

    def ffn(d, x=fake, offsets=fake, w1=fake, w2=fake, b1=None, b2=None, out=fake, ws=fake, ws_bytes=1 << 40):
        return L.bigmac_mx_grouped_ffn(ctypes.byref(d), x, offsets, w1, w2, b1, b2, out, ws, ws_bytes, None)

    d = B.make_dims(128, 128, 64, 8, 2, 128)
    assert B.workspace_bytes(d, B.WS_MX_GROUPED_FFN) > 128 * 2 * (32 + 64)
    for bad in (dict(x=None), dict(offsets=None), dict(w1=None), dict(w2=None), dict(out=None), dict(ws=None), dict(x=odd), dict(b1=odd), dict(w2=odd), dict(out=odd)):
        assert ffn(d, **bad) == -1, bad
    assert ffn(d, ws_bytes=B.workspace_bytes(d, B.WS_MX_GROUPED_FFN) - 1) == -2
    f32 = B.make_dims(128, 128, 64, 8, 2, 128, dtype=B.F32)
    assert ffn(f32) == -3 and B.workspace_bytes(f32, B.WS_MX_GROUPED_FFN) == 0
    assert ffn(B.make_dims(0, 128, 64, 8, 2, 128)) == -1


@pytest.mark.parametrize("kind", range(8))
def test_workspace_kinds_of_bad_dims(kind):
    assert B.workspace_bytes(B.make_dims(0, 128, 64, 8, 2, 128), kind) == 0


def test_tensors_of_the_host_and_of_another_gpu_are_refused(monkeypatch):
    """Before anything reaches the library: host tensors, and tensors of a GPU that is not the current one."""
    class On1:
        device = "cuda:1"

        def get_device(self):
            return 1

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    t, d = torch.zeros(64, dtype=torch.uint8), B.make_mx_dims(1, 1, 64, 64)
    ffn, norm = B.make_dims(1, 64, 64, 1, 1, 64), B.make_norm_dims(1, 64)
    with pytest.raises(ValueError):
        B.make_norm_params(pre_w=torch.ones(64))
    p = B.make_norm_params()
    for bad in (t, On1()):
        for call in (lambda: B.bigmac_mx_quantize(1, 64, B.BF16, bad, None, None), lambda: B.bigmac_mx_dequantize(1, 64, None, bad, B.F32, None),
                     lambda: B.bigmac_mx_pack(1, 64, 64, B.BF16, None, bad), lambda: B.bigmac_mx_unpack(1, 64, 64, bad, B.BF16, None),
                     lambda: B.bigmac_mx_product(d, None, None, None, bad, None, None), lambda: B.bigmac_mx_grouped_ffn(ffn, None, None, None, None, None, None, b2=bad),
                     lambda: B.bigmac_norm_forward(norm, p, None, None, None, bad), lambda: B.bigmac_norm_backward(norm, p, *[None] * 11, bad)):
            with pytest.raises(ValueError):
                call()


def test_sizes_of_columns_that_the_calls_refuse():
    """A size query answers for what the calls take: 0 for columns that bigmac_mx_quantize refuses."""
    fake = ctypes.c_void_p(4096)
    for cols in (1, 5, 31, 33, 48, 255, (1 << 24) + 32, -32, 1 << 40):
        assert B.mx_scale_bytes(cols) == 0, cols
        assert B.lib().bigmac_mx_quantize(1, cols, B.BF16, fake, fake, fake, None) < 0
    assert [B.mx_scale_bytes(c) for c in (32, 224, 8224, 1 << 24)] == [8, 8, 33 * 8, 1 << 19]


def test_workspace_of_experts_that_the_call_refuses():
    fake = ctypes.c_void_p(4096)
    for d in (B.make_dims((1 << 28) + 1, 128, 64, 8, 4, 128), B.make_dims(4, 128, 64, 8, 4, (1 << 24) + 64), B.make_dims(4, (1 << 24) + 64, 64, 8, 4, 64, order=B.ORDER_CDAC),
              B.make_dims(1 << 28, 256, 256, 8, 4, 128), B.make_dims(4, 128, 128, 1024, 4, 1 << 24)):
        assert B.lib().bigmac_mx_grouped_ffn(ctypes.byref(d), fake, fake, fake, fake, None, None, fake, fake, 1 << 62, None) == -5
        assert B.workspace_bytes(d, B.WS_MX_GROUPED_FFN) == 0
    d = B.make_dims(1 << 22, 128, 64, 8, 4, 128)
    rows, up = 1 << 24, lambda n: -(-n // 256) * 256                                       # noqa: E731
    at_least = up(rows * 32) + up(rows * 8) + up(rows * 64) + up(rows * 8)
    assert at_least < B.workspace_bytes(d, B.WS_MX_GROUPED_FFN) < at_least * 1.1


def test_workspace_of_products_that_the_call_refuses():
    fake = ctypes.c_void_p(4096)
    for d in (B.make_mx_dims(1 << 30, 1, 64, 1 << 20), B.make_mx_dims(1 << 24, 1024, 64, 1 << 16), B.make_mx_dims((1 << 30) + 1, 4, 64, 64)):
        assert B.lib().bigmac_mx_product(ctypes.byref(d), fake, fake, fake, fake, None, fake, fake, 1 << 62, None) == -5
        assert B.mx_workspace_bytes(d) == 0
    assert B.mx_workspace_bytes(B.make_mx_dims(1 << 30, 1024, 64, 64)) >= 16 * (1 << 30) // 128

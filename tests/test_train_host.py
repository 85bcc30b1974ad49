"""Refusals of the microscaled and distillation calls, through the C ABI and the binding, before anything is launched (CPU)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2506_12038_b200 as lcd
from paper_2506_12038_b200 import binding

lib = binding.lib
A = ctypes.c_void_p(1 << 20)          # an aligned address that nothing reads
ODD = ctypes.c_void_p((1 << 20) + 8)


def quantize(x=A, type=0, M=2, K=64, ldx=64, inv=None, codes=A, ldc=32, scales=A, lds=16):
    return lib.lcd_mx_quantize(x, type, M, K, ldx, inv, codes, ldc, scales, lds, None)


def dequantize(codes=A, ldc=32, scales=A, lds=16, M=2, K=64, out=A, type=0, ldo=64):
    return lib.lcd_mx_dequantize(codes, ldc, scales, lds, M, K, out, type, ldo, None)


def linear(wc=A, ldwc=32, ws=A, ldws=16, N=5, K=64, xc=A, ldxc=32, xs=A, ldxs=16, M=2, y=A, type=0, ldy=5, word=None):
    return lib.lcd_mx_linear(wc, ldwc, ws, ldws, N, K, xc, ldxc, xs, ldxs, M, y, type, ldy, word, None)


def fused(wc=A, ldwc=32, ws=A, ldws=16, N=5, K=64, x=A, x_type=1, ldx=64, inv=None, M=2, y=A, type=0, ldy=5, space=A, bytes=1 << 20, word=None):
    return lib.lcd_mx_linear_fused(wc, ldwc, ws, ldws, N, K, x, x_type, ldx, inv, M, y, type, ldy, space, bytes, word, None)


def loss(z=A, type=0, T=2, V=50, ldz=50, idx=A, width=4, ldi=3, top=A, top_type=1, ldt=3, k=3, tau=1.0, lse=None, weight=None, loss=A, stats=None,
         d=None, ldd=50):
    return lib.lcd_distill_loss(z, type, T, V, ldz, idx, width, ldi, top, top_type, ldt, k, tau, lse, weight, loss, stats, d, ldd, None)


def grad(z=A, type=0, T=2, V=50, ldz=50, idx=A, width=4, ldi=3, top=A, top_type=1, ldt=3, k=3, tau=1.0, lse=None, weight=None, stats=A, d=ODD, ldd=50):
    return lib.lcd_distill_grad(z, type, T, V, ldz, idx, width, ldi, top, top_type, ldt, k, tau, lse, weight, stats, d, ldd, None)


@pytest.mark.parametrize("call,bad", [
    (quantize, [dict(x=None), dict(type=3), dict(type=-1), dict(M=0), dict(K=0), dict(M=-1), dict(ldx=63), dict(codes=None), dict(scales=None),
                dict(codes=ODD), dict(scales=ODD), dict(ldc=16), dict(ldc=40), dict(lds=8), dict(lds=0), dict(inv=ctypes.c_void_p(2)), dict(x=ctypes.c_void_p(2)),
                dict(M=1 << 31), dict(K=1 << 31, ldx=1 << 31, ldc=1 << 30, lds=1 << 26)]),
    (dequantize, [dict(out=None), dict(type=7), dict(M=0), dict(K=0), dict(ldo=63), dict(codes=ODD), dict(scales=ODD), dict(ldc=16), dict(lds=8)]),
    (linear, [dict(wc=None), dict(ws=None), dict(xc=None), dict(xs=None), dict(y=None), dict(N=0), dict(K=0), dict(M=0), dict(ldy=4), dict(type=3),
              dict(wc=ODD), dict(ws=ODD), dict(xc=ODD), dict(xs=ODD), dict(ldwc=24), dict(ldws=24), dict(ldxc=16), dict(ldxs=8), dict(word=ctypes.c_void_p(2)),
              dict(y=ctypes.c_void_p(2)), dict(K=65), dict(M=1 << 31), dict(N=1 << 31, ldy=1 << 31)]),
    (fused, [dict(wc=None), dict(x=None), dict(x_type=9), dict(ldx=63), dict(M=0), dict(space=ODD), dict(K=65), dict(inv=ctypes.c_void_p(2))]),
    (loss, [dict(z=None), dict(idx=None), dict(top=None), dict(loss=None), dict(type=3), dict(top_type=3), dict(T=0), dict(V=0), dict(k=0), dict(ldz=49),
            dict(ldi=2), dict(ldt=2), dict(width=2), dict(width=8, idx=ctypes.c_void_p(4)), dict(tau=0.0), dict(tau=-1.0), dict(tau=float("nan")),
            dict(tau=float("inf")), dict(tau=1e-39), dict(d=A, ldd=49), dict(d=A, ldz=64, ldd=50), dict(lse=ctypes.c_void_p(2)), dict(weight=ctypes.c_void_p(2)),
            dict(stats=ctypes.c_void_p(2)), dict(z=ctypes.c_void_p(2)), dict(T=1 << 31)]),
    (grad, [dict(stats=None), dict(d=None), dict(z=None), dict(ldd=49), dict(tau=0.0), dict(k=0)])])
def test_invalid_arguments(call, bad):
    for kw in bad:
        assert call(**kw) == 1, kw


def test_too_many_entries_and_short_workspaces():
    assert loss(V=5000, ldz=5000, k=1025, ldi=1025, ldt=1025) == 2
    assert fused(M=20, bytes=20 * 48 - 1) == 3 and fused(M=20, space=None) == 3
    need = ctypes.c_size_t()
    assert lib.lcd_mx_linear_fused_workspace_bytes(20, 64, ctypes.byref(need)) == 0 and need.value == 20 * (32 + 16)
    assert lib.lcd_mx_linear_fused_workspace_bytes(4, 64, ctypes.byref(need)) == 0 and need.value == 0
    assert lib.lcd_mx_linear_fused_workspace_bytes(0, 64, ctypes.byref(need)) == 1
    assert lib.lcd_mx_linear_fused_workspace_bytes(2, 64, None) == 1
    assert lcd.mx_linear_fused_workspace_bytes(33, 33) == 33 * (32 + 16)


def test_binding_refuses_what_is_no_gpu_matrix():
    x, byte = torch.zeros(2, 64), torch.zeros(2, 32, dtype=torch.uint8)
    for call in (lambda: lcd.mx_quantize(x), lambda: lcd.mx_dequantize(byte, byte), lambda: lcd.mx_linear(byte, byte, byte, byte),
                 lambda: lcd.mx_linear_fused(byte, byte, x), lambda: lcd.distill_loss(x, byte.int(), x), lambda: lcd.distill_grad(x, byte.int(), x, x)):
        with pytest.raises(AssertionError):
            call()
    for call in (lambda: lcd.mx_quantize(np.zeros((2, 64))), lambda: lcd.distill_loss(None, None, None), lambda: lcd.mx_linear(1, 2, 3, 4)):
        with pytest.raises(TypeError):
            call()

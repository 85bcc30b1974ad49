"""Refusals of the calls on row groups, experts and adapters, through the C ABI and the binding, before anything is launched (CPU)."""
import ctypes

import pytest
import torch

import paper_2506_12038_b200 as lcd
from paper_2506_12038_b200 import binding

lib = binding.lib
A = ctypes.c_void_p(1 << 20)          # an aligned address that nothing reads
ODD = ctypes.c_void_p((1 << 20) + 8)
TWO = ctypes.c_void_p(2)


def plan(**kw):
    return binding.RowGroupsC(**{**dict(order=1 << 20, groups=1 << 20, offsets=1 << 20, count=6), **kw})


def weights(**kw):
    return binding.AdapterWeights(**{**dict(a=1 << 20, b=1 << 20, type=1, lda=64, adapter_a=64 * 4, ldb=4, adapter_b=4 * 10, G=3, rank=4, K=64, N=10,
                                            scale=None), **kw})


def group(g=A, width=4, count=6, G=3, order=A, groups=A, offsets=A):
    return lib.lcd_group_rows(g, width, count, G, order, groups, offsets, None)


def experts(wc=A, ldwc=32, dwc=32 * 5, ws=A, ldws=16, dws=16 * 5, G=3, N=5, K=64, x=A, x_type=1, T=2, ldx=64, inv=None, rows=None, y=A, y_type=0,
            ldy=5, space=A, bytes=1 << 20, word=None):
    return lib.lcd_mx_linear_grouped(wc, ldwc, dwc, ws, ldws, dws, G, N, K, x, x_type, T, ldx, inv, plan() if rows is None else rows, y, y_type, ldy,
                                     space, bytes, word, None)


def adapters(w=None, x=A, x_type=1, ldx=64, rows=None, base=A, ldbase=10, y=ODD, y_type=0, ldy=10, t=None, ldt=0, space=A, bytes=1 << 20, word=None):
    return lib.lcd_adapters(weights() if w is None else w, x, x_type, ldx, plan() if rows is None else rows, base, ldbase, y, y_type, ldy, t, ldt,
                            space, bytes, word, None)


def grad(w=None, dy=A, lddy=10, x=A, ldx=64, type=1, t=A, ldt=4, rows=None, base=A, ldbase=64, dx=ODD, lddx=64, da=A, db=A, grad_type=0, space=A,
         bytes=1 << 20, word=None):
    return lib.lcd_adapters_grad(weights() if w is None else w, dy, lddy, x, ldx, type, t, ldt, plan() if rows is None else rows, base, ldbase, dx,
                                 lddx, da, db, grad_type, space, bytes, word, None)


PLANS = [dict(rows=plan(order=None)), dict(rows=plan(groups=None)), dict(rows=plan(offsets=None)), dict(rows=plan(count=0)), dict(rows=plan(count=-1)),
         dict(rows=plan(order=2)), dict(rows=plan(count=(1 << 30) + 1))]
WEIGHTS = [dict(w=weights(**kw)) for kw in (dict(a=None), dict(b=None), dict(type=3), dict(lda=63), dict(ldb=3), dict(G=0), dict(rank=0), dict(K=0), dict(N=0),
                                            dict(adapter_a=64 * 4 - 1), dict(adapter_b=39), dict(a=1), dict(scale=2))]


@pytest.mark.parametrize("call,bad", [
    (group, [dict(g=None), dict(width=2), dict(width=8, g=ctypes.c_void_p(4)), dict(g=TWO), dict(count=0), dict(count=-5), dict(count=(1 << 30) + 1),
             dict(G=0), dict(order=None), dict(groups=None), dict(offsets=None), dict(order=TWO), dict(groups=TWO), dict(offsets=TWO)]),
    (experts, PLANS + [dict(wc=None), dict(ws=None), dict(x=None), dict(y=None), dict(wc=ODD), dict(ws=ODD), dict(ldwc=16), dict(ldwc=40), dict(ldws=8),
                       dict(dwc=32 * 5 - 16), dict(dwc=32 * 5 + 8), dict(dws=16 * 4), dict(G=0), dict(N=0), dict(K=0), dict(K=65), dict(T=0), dict(T=4),
                       dict(T=12), dict(ldx=63), dict(ldy=4), dict(x_type=3), dict(y_type=-1), dict(inv=TWO), dict(space=ODD), dict(word=TWO), dict(y=TWO)]),
    (adapters, PLANS + WEIGHTS + [dict(x=None), dict(x_type=5), dict(ldx=63), dict(x=ctypes.c_void_p(1)), dict(y=None), dict(ldy=9), dict(y_type=3),
                                  dict(base=TWO), dict(ldbase=9), dict(y=A, ldy=12), dict(t=A, ldt=3), dict(t=TWO, ldt=4), dict(space=ODD), dict(word=TWO)]),
    (grad, PLANS + WEIGHTS + [dict(dy=None), dict(lddy=9), dict(x=None), dict(ldx=63), dict(type=3), dict(t=None), dict(ldt=3), dict(t=TWO),
                              dict(base=ctypes.c_void_p(1)), dict(ldbase=63), dict(lddx=63), dict(dx=A, lddx=70), dict(dx=A, base=None), dict(dx=A, x=ODD, dy=ODD, lddx=72), dict(dx=None, da=None, db=None),
                              dict(grad_type=3), dict(da=TWO), dict(space=ODD), dict(word=TWO)])])
def test_invalid_arguments(call, bad):
    for kw in bad:
        assert call(**kw) == 1, kw


def test_unsupported_and_short_workspaces():
    assert group(G=1025) == 2 and experts(G=513) == 2
    assert adapters(w=weights(rank=129, lda=64, adapter_a=64 * 129, ldb=129, adapter_b=1290)) == 2
    assert adapters(w=weights(type=2)) == 2 and grad(w=weights(type=2)) == 2              # fp16 beside bf16
    assert adapters(w=weights(G=1025)) == 2 and grad(w=weights(G=1025)) == 2
    assert experts(bytes=6 * 52 - 1) == 3 and experts(space=None) == 3
    assert adapters(bytes=6 * 64 - 1) == 3 and adapters(space=None) == 3 and grad(bytes=6 * 64 - 1) == 3
    need = ctypes.c_size_t()
    assert lib.lcd_adapters_workspace_bytes(6, 129, ctypes.byref(need)) == 2 and lib.lcd_adapters_workspace_bytes(0, 4, ctypes.byref(need)) == 1
    assert lib.lcd_adapters_workspace_bytes(6, 4, None) == 1 and lib.lcd_mx_linear_grouped_workspace_bytes(6, 0, ctypes.byref(need)) == 1
    for rank, padded in ((1, 16), (16, 16), (17, 32), (33, 64), (65, 128), (128, 128)):
        assert lcd.adapters_workspace_bytes(511, rank) == 511 * padded * 4 and lcd.adapters_workspace_bytes(512, rank) == 512 * padded * 10
    assert lcd.mx_linear_grouped_workspace_bytes(6, 64) == 6 * 52


def test_binding_refuses_what_is_no_gpu_tensor():
    x, w, byte, index = torch.zeros(2, 64), torch.zeros(3, 4, 64), torch.zeros(3, 2, 32, dtype=torch.uint8), torch.zeros(2, dtype=torch.int32)
    rows = lcd.RowGroups(index, index, torch.zeros(4, dtype=torch.int32))
    for call in (lambda: lcd.group_rows(index, 3), lambda: lcd.mx_linear_grouped(byte, byte, x, rows), lambda: lcd.adapters(x, w, w, rows),
                 lambda: lcd.adapters_grad(x, x, w, w, x, rows)):
        with pytest.raises(AssertionError):
            call()
    for call in (lambda: lcd.group_rows([0, 1], 3), lambda: lcd.mx_linear_grouped(1, 2, 3, rows), lambda: lcd.adapters(x, None, w, rows)):
        with pytest.raises(TypeError):
            call()

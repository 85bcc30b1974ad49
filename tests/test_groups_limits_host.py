"""The largest sizes of the calls on row groups, experts and adapters: one more is refused before anything is launched (CPU)."""
import ctypes

import paper_2506_12038_b200 as lcd
from test_groups_host import adapters, experts, grad, lib, weights

MOST = 1 << 30


def test_columns_beyond_the_most():
    assert experts(N=MOST + 1, ldy=MOST + 1, dwc=32 * (MOST + 1), dws=16 * (MOST + 1)) == 1
    assert experts(K=MOST + 1, ldx=MOST + 1, ldwc=(MOST // 32 + 1) * 16, dwc=(MOST // 32 + 1) * 80, ldws=MOST // 32 + 16, dws=(MOST // 32 + 16) * 5) == 1
    wide = weights(K=MOST + 1, lda=MOST + 1, adapter_a=4 * (MOST + 1))
    assert adapters(w=wide, ldx=MOST + 1) == 1 and grad(w=wide, ldx=MOST + 1, ldbase=MOST + 1, lddx=MOST + 1) == 1
    high = weights(N=MOST + 1, adapter_b=4 * (MOST + 1))
    assert adapters(w=high, ldbase=MOST + 1, ldy=MOST + 1) == 1 and grad(w=high, lddy=MOST + 1) == 1
    need = ctypes.c_size_t()
    assert lib.lcd_mx_linear_grouped_workspace_bytes(6, MOST + 1, ctypes.byref(need)) == 1


def test_resolve():
    tokens, split, paired = ctypes.c_int(-7), ctypes.c_int(-7), ctypes.c_int(-7)
    out = [ctypes.byref(v) for v in (tokens, split, paired)]
    for bad in ((0, 3, 5, 64), (6, 0, 5, 64), (6, 3, 0, 64), (6, 3, 5, 0), (MOST + 1, 3, 5, 64), (6, 3, MOST + 1, 64), (6, 3, 5, MOST + 1)):
        assert lib.lcd_mx_linear_grouped_resolve(*bad, *out) == 1, bad
    for i in range(3):
        assert lib.lcd_mx_linear_grouped_resolve(6, 3, 5, 64, *out[:i], None, *out[i + 1:]) == 1
    assert lib.lcd_mx_linear_grouped_resolve(6, 513, 5, 64, *out) == 2
    assert (tokens.value, split.value, paired.value) == (-7, -7, -7)
    assert lcd.resolve_mx_linear_grouped(6, 3, 5, 64) == (16, 1, False)

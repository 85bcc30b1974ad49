"""The largest sizes of the calls on row groups, experts and adapters: one more is refused before anything is launched (CPU)."""
import ctypes

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

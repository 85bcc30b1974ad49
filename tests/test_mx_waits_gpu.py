"""The limit of a product's waits counts from when its operands may be read, not from when its blocks began: a kernel before it may let it
begin early and run on for longer than that."""
import pytest
import torch

import paper_2506_12038_b200 as lcd
from test_mx_gpu import random_mx, random_x

pytestmark = pytest.mark.gpu

RUNS_ON = r"""
extern "C" __global__ void runs_on(long long ns) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  long long t0, t;
  asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t0));
  for (unsigned i = 0; i < 4000000000u; ++i) {
    asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(t));
    if (t - t0 >= ns) break;
  }
}
"""


@pytest.mark.parametrize("M,N,K,ready", [(3, 500, 1000, False), (40, 500, 1000, True), (12, 129, 4096, True), (700, 7001, 6000, True)])
def test_behind_a_kernel_that_runs_on(M, N, K, ready):
    runs_on = torch.cuda._compile_kernel(RUNS_ON, "runs_on")
    w, x = random_mx(N, N, K), random_x(M, M, K)
    operands = lcd.mx_quantize(x) if ready else (x,)
    call = lcd.mx_linear if ready else lcd.mx_linear_fused
    want = call(w[0], w[1], *operands)
    y, word = torch.zeros_like(want), torch.full((1,), -5, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    runs_on(grid=(1, 1, 1), block=(32, 1, 1), args=[2_600_000_000])
    call(w[0], w[1], *operands, y=y, status_word=word)
    torch.cuda.synchronize()
    assert word.item() == -5 and torch.equal(y, want)

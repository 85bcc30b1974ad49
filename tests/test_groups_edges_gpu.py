"""Rows of base and y at any alignment, with NaN right before and behind each: what the kernels for few rows load around a row's ends does not
show in results, which equal those of aligned rows."""
import pytest
import torch

import paper_2506_12038_b200 as lcd
from test_groups_gpu import TYPES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("w,out", [("fp32", "bf16"), ("fp32", "fp16"), ("fp32", "fp32"), ("bf16", "bf16"), ("fp16", "fp16")])
@pytest.mark.parametrize("r", [16, 60, 100])
def test_ends_of_rows(w, out, r):
    g = torch.Generator(device="cuda").manual_seed(r)
    M, K, most = 7, 64, 150
    x = torch.randn(M, K, generator=g, device="cuda").to(TYPES["fp32" if w == "fp32" else w])
    a = torch.randn(2, r, K, generator=g, device="cuda").to(TYPES[w])
    rows = lcd.group_rows(torch.arange(M, device="cuda") % 3, 2)
    for N in (23, 24, 31, 32, 33, 36, 44, 47, 64, 100, 149, 150):
        b = torch.randn(2, N, r, generator=g, device="cuda").to(TYPES[w])
        base = torch.randn(M, N, generator=g, device="cuda").to(TYPES[out])
        even = torch.zeros(M, (N + 15) // 16 * 16, dtype=TYPES[out], device="cuda")
        even[:, :N] = base
        want = lcd.adapters(x, a, b, rows, even[:, :N])
        for before, pitch in ((1, N + 1), (2, N + 3), (3, N + 5), (4, N + 4), (5, N + 1), (8, N + 7)):
            room = torch.full((before + M * pitch,), float("nan"), dtype=TYPES[out], device="cuda")
            off = room[before:].view(M, pitch)[:, :N]
            off.copy_(base)
            assert torch.equal(lcd.adapters(x, a, b, rows, off), want)
            assert torch.equal(lcd.adapters(x, a, b, rows, off, y=off), want)
            assert torch.isnan(room[:before]).all() and torch.isnan(room[before:].view(M, pitch)[:, N:]).all()

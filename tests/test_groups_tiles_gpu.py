"""Adapters of many rows whose blocks walk through more tiles than they have buffers for."""
import pytest
import torch

import paper_2506_12038_b200 as lcd
from test_groups_gpu import TYPES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("x,w,N", [("bf16", "bf16", 9000), ("fp16", "fp16", 9001), ("fp32", "bf16", 5003), ("fp32", "fp32", 5000)])
def test_many_tiles_a_block(x, w, N):
    # a row's result depends on its own tile only, so the same rows beside fewer others have to give the same bits
    g = torch.Generator(device="cuda").manual_seed(N)
    M, K, r, G = 5000, 64, 16, 3
    xs, base = torch.randn(M, K, generator=g, device="cuda").to(TYPES[x]), torch.randn(M, N, generator=g, device="cuda").to(TYPES[x])
    a, b = torch.randn(G, r, K, generator=g, device="cuda").to(TYPES[w]), torch.randn(G, N, r, generator=g, device="cuda").to(TYPES[w])
    group = torch.randint(-1, G, (M,), generator=g, device="cuda")
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    y, t = lcd.adapters(xs, a, b, lcd.group_rows(group, G), base, want_t=True, status_word=word)
    part = torch.cat([lcd.adapters(xs[i:i + 1250], a, b, lcd.group_rows(group[i:i + 1250], G), base[i:i + 1250], status_word=word)
                      for i in range(0, M, 1250)])
    assert torch.equal(part, y) and torch.equal(y[group < 0], base[group < 0])
    dx = lcd.adapters_grad(y, None, a, b, None, lcd.group_rows(group, G), xs, want_weights=False, status_word=word)[0]
    # (y is about (K r)^(1/2) = 32, dt that times N^(1/2), dx that times r^(1/2): 12000, and five times that is more than fp16 has)
    assert not torch.isnan(dx).any() and word.item() == 0

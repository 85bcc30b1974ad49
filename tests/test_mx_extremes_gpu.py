"""Products of microscaled matrices at the ends of the scales' range, and what one launch and two make of infinities, NaN and subnormal numbers."""
import numpy as np
import pytest
import torch

import paper_2506_12038_b200 as lcd
from oracle import train_oracle as O
from test_mx_gpu import TYPES, host, random_mx

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M", [255, 3])
def test_scales_whose_product_is_one(M):
    # token m's scale 2^(m - 127) against weight rows of 2^(127 - m): only where both meet is the sum of ordinary size
    N, K = 255, 64
    w, x = random_mx(1, N, K), random_mx(2, M, K)
    bytes_ = torch.arange(255, dtype=torch.uint8, device="cuda")
    w[1].copy_((254 - bytes_)[:, None].expand(-1, 2))
    x[1].copy_(bytes_[:M, None].expand(-1, 2))
    y64, _ = O.mx_linear(w[2], w[1].cpu().numpy(), x[2], x[1].cpu().numpy())
    got = host(lcd.mx_linear(w[0], w[1], x[0], x[1]))
    at = np.arange(M)
    assert np.array_equal(got[at, at], y64[at, at])
    fine = (np.abs(y64) < 2.0 ** 127) & ((np.abs(y64) > 2.0 ** -100) | (y64 == 0))
    assert np.array_equal(got[fine], y64[fine])


@pytest.mark.parametrize("type", sorted(TYPES))
@pytest.mark.parametrize("M,K", [(1, 700), (4, 4096), (3, 33)])
def test_one_launch_and_two_agree_on_every_kind_of_number(M, K, type):
    assert lcd.mx_linear_fused_workspace_bytes(M, K) == 0
    rng = np.random.default_rng(K)
    bits = rng.integers(0, 2 ** 32, size=(M, K), dtype=np.uint64).astype(np.uint32)
    x = torch.from_numpy(bits.view(np.float32).copy()).to(TYPES[type]).cuda() if type != "fp32" else torch.from_numpy(bits.view(np.float32).copy()).cuda()
    x[:, 32 * (K // 64):] = (torch.rand(M, K - 32 * (K // 64), device="cuda") * 1e-7).to(x.dtype)        # subnormal in fp16
    w = random_mx(K, 300, K)
    for inv in (None, torch.full((K,), 0.37, device="cuda"), torch.full((K,), 3e38, device="cuda")):
        y = lcd.mx_linear_fused(w[0], w[1], x, inv)
        z = lcd.mx_linear(w[0], w[1], *lcd.mx_quantize(x, inv))
        assert torch.equal(y.isnan(), z.isnan()) and torch.equal(torch.nan_to_num(y, nan=1.0), torch.nan_to_num(z, nan=1.0))
    x[:, :32 * (K // 64)] = x[:, -1:]
    y = lcd.mx_linear_fused(w[0], w[1], x)
    assert torch.isfinite(y).all() and torch.equal(y, lcd.mx_linear(w[0], w[1], *lcd.mx_quantize(x)))

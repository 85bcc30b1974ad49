"""Products of microscaled matrices whose tiles are shared by pairs of CTAs, while other work delays their copies: every result is exact."""
import pytest
import torch

import paper_2506_12038_b200 as lcd
from test_mx_gpu import random_mx, random_x

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N,K", [(700, 7001, 6000), (1100, 7001, 6000), (1537, 9001, 40), (2100, 2600, 9000)])     # 192 and 256 tokens a tile
def test_pairs_under_load(M, N, K):
    # scales 2^0: every sum is a multiple of 1/4 below 2^24 of them, so that results are exact whatever the order
    w, x = random_mx(N + K, N, K), random_mx(M, M, K)
    w[1].fill_(127)
    x[1].fill_(127)
    a, b = (lcd.mx_dequantize(t[0], t[1], K).double() for t in (x, w))
    want, size = (a @ b.t()).float(), (a.abs() @ b.abs().t()).max()
    assert size * 4 < 2 ** 24
    load = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(60):
            load[: 1 << 27].copy_(load[1 << 27:])
    results = [lcd.mx_linear(w[0], w[1], x[0], x[1]) for _ in range(12)]
    for y in results:
        assert torch.equal(y, want)
    torch.cuda.synchronize()


@pytest.mark.parametrize("M,N,K", [(700, 7001, 6000), (1100, 7001, 6000)])
def test_pairs_whose_weights_are_copied_ahead(M, N, K):
    # the one-call form asks for the weights before the tokens have been quantised, by both CTAs of a pair
    w = random_mx(3, N, K)
    xs = [random_x(s, M, K, "bf16") for s in range(2)]
    want = [lcd.mx_linear(w[0], w[1], *lcd.mx_quantize(x)) for x in xs]
    torch.cuda.synchronize()
    for _ in range(10):
        for x, y in zip(xs, want):
            assert torch.equal(lcd.mx_linear_fused(w[0], w[1], x), y)
    word = torch.full((1,), -5, dtype=torch.int32, device="cuda")
    assert torch.equal(lcd.mx_linear_fused(w[0], w[1], xs[0], status_word=word), want[0]) and word.item() == -5

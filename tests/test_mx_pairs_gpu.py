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


@pytest.mark.parametrize("M,N,K", [(65, 128000, 256), (97, 128000, 600), (193, 38000, 600), (200, 28672, 4096), (150, 14001, 4096)])
def test_pairs_of_a_large_vocabulary(M, N, K):
    # fewer tokens than a tile's first half, one more than it, one more than a tile; weight rows that end in a pair's second half
    w, x = random_mx(N + K, N, K), random_mx(M, M, K)
    w[1].fill_(127)
    x[1].fill_(127)
    a, b = (lcd.mx_dequantize(t[0], t[1], K).double() for t in (x, w))
    y = torch.full((M + 1, N + 3), 7.0, device="cuda")
    lcd.mx_linear(w[0], w[1], x[0], x[1], y=y[:M, :N])
    assert torch.equal(y[:M, :N], (a @ b.t()).float()) and (y[M] == 7).all() and (y[:, N:] == 7).all()


def test_pairs_beside_other_products_and_in_a_graph():
    # several streams, narrow tiles and pairs at once; then the same pairs' calls captured and replayed
    work = [(700, 7001, 2000), (1100, 7001, 2000), (12, 5000, 4096), (300, 2600, 777)]
    w = [random_mx(i, N, K) for i, (M, N, K) in enumerate(work)]
    x = [random_x(i, M, K, "bf16") for i, (M, N, K) in enumerate(work)]
    want = [lcd.mx_linear_fused(a[0], a[1], b) for a, b in zip(w, x)]
    streams = [torch.cuda.Stream() for _ in work]
    torch.cuda.synchronize()
    got = [[] for _ in work]
    for _ in range(15):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(lcd.mx_linear_fused(w[i][0], w[i][1], x[i]))
    torch.cuda.synchronize()
    assert all(torch.equal(y, want[i]) for i in range(len(work)) for y in got[i])
    out = [torch.zeros_like(y) for y in want]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        for i in range(len(work)):
            lcd.mx_linear_fused(w[i][0], w[i][1], x[i], y=out[i])
    for _ in range(3):
        for y in out:
            y.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))

"""t and dt enter the products behind them with all their 24 bits: terms that cancel leave what only the last of those bits hold."""
import pytest
import torch

import paper_2506_12038_b200 as lcd
from test_groups_gpu import PAIRS, TYPES

pytestmark = pytest.mark.gpu

# In each of these sums two terms cancel but for 2^-18: 1 + 2^-9 + 2^-18 takes 19 bits, which no single 16-bit number and no two bf16 parts of
# 8 bits hold; everything else is exact in every type, so the results are too.
REST = 2.0 ** -18


def filled(shape, type, entries):
    t = torch.zeros(shape, dtype=TYPES[type], device="cuda")
    for at, v in entries.items():
        t[at] = v
    return t


def wanted(shape, entries):
    return filled(shape, "fp32", entries).double()


SHAPES = [(2, 2, 3, 2), (8, 64, 72, 16), (40, 67, 33, 30), (70, 96, 130, 64), (64, 64, 72, 128), (600, 64, 136, 16), (600, 256, 200, 40), (520, 128, 264, 64),
          (1100, 67, 131, 24), (700, 64, 72, 128), (1500, 65, 129, 100)]


@pytest.mark.parametrize("x,w", PAIRS)
@pytest.mark.parametrize("M,K,N,r", SHAPES)
def test_t_enters_with_all_its_bits(x, w, M, K, N, r):
    K = max(K, 3)
    xs = filled((M, K), x, {(slice(None), 0): 1.0, (slice(None), 1): 2.0 ** -9, (slice(None), 2): 2.0 ** -9})
    a = filled((1, r, K), w, {(0, 0, 0): 1.0, (0, 0, 1): 1.0, (0, 0, 2): 2.0 ** -9, (0, r - 1, 0): 1.0, (0, r - 1, 1): 1.0})
    b = filled((1, N, r), w, {(0, slice(None), 0): 1.0, (0, slice(None), r - 1): -1.0})
    rows = lcd.group_rows(torch.zeros(M, dtype=torch.int32, device="cuda"), 1)
    for out in TYPES.values():
        y, t = lcd.adapters(xs, a, b, rows, dtype=out, want_t=True)
        assert (t[:, 0] == 1 + 2.0 ** -9 + REST).all() and (y.double() == REST).all()


@pytest.mark.parametrize("x,w", PAIRS)
@pytest.mark.parametrize("M,N,K,r", SHAPES)
def test_t_and_dt_enter_the_gradients_with_all_their_bits(x, w, M, N, K, r):
    N = max(N, 3)
    # rows 0 and M - 1 differ in the last of three columns of dy, so dt does by REST; x is 1 and -1 there
    dy = filled((M, N), x, {(slice(None), 0): 1.0, (slice(None), 1): 2.0 ** -9, (0, 2): 2.0 ** -9})
    b = filled((1, N, r), w, {(0, 0, 0): 1.0, (0, 1, 0): 1.0, (0, 2, 0): 2.0 ** -9, (0, 0, r - 1): 1.0, (0, 1, r - 1): 1.0})
    a = filled((1, r, K), w, {(0, 0, slice(None)): 1.0, (0, r - 1, slice(None)): -1.0})
    xs = filled((M, K), x, {(0, slice(None)): 1.0, (M - 1, slice(None)): -1.0})
    rows = lcd.group_rows(torch.zeros(M, dtype=torch.int32, device="cuda"), 1)
    sums = filled((M, N), x, {(0, slice(None)): 1.0, (M - 1, slice(None)): -1.0})
    t = filled((M, r), "fp32", {(0, slice(None)): 1.0 + 2.0 ** -9 + REST, (M - 1, slice(None)): 1.0 + 2.0 ** -9})
    for out in TYPES.values():
        dx, da, _ = lcd.adapters_grad(dy, xs, a, b, t, rows, grad_dtype=out)
        assert torch.equal(dx.double(), wanted((M, K), {0: REST}))
        assert torch.equal(da.double(), wanted((1, r, K), {(0, 0): REST}))
        assert (lcd.adapters_grad(sums, xs, a, b, t, rows, grad_dtype=out, want_dx=False)[2].double() == REST).all()


@pytest.mark.parametrize("x,w", [("fp32", "fp32"), ("fp16", "fp16"), ("bf16", "bf16"), ("bf16", "fp32")])
@pytest.mark.parametrize("r,most", [(16, 76), (40, 172), (64, 172), (128, 172)])
@pytest.mark.parametrize("positive", [False, True])
def test_long_sums_of_every_rank(x, w, r, most, positive):
    # 8192 terms: 128 stages of four instructions, in turn to seven accumulators (ranks to 32) or three: `most` additions one after the other, each of
    # which cuts off less than a step of its sum, 2^-23 of it.  Accumulators and parts are joined by ten additions at most (10 * 2^-24) and products
    # of fp32 numbers are within 2^-21: together less than 2^-19.  Signed terms cancel: there errors are shares of the terms' root of squares, which
    # the random walk of a sum does not exceed by more than a few times; all positive ones they are shares of the sum itself.
    g = torch.Generator(device="cuda").manual_seed(r)
    M = K = 8192
    draw = (lambda *s: torch.rand(*s, generator=g, device="cuda")) if positive else (lambda *s: torch.randn(*s, generator=g, device="cuda"))
    xs, dy, t = draw(M, K).to(TYPES[x]), draw(M, 64).to(TYPES[x]), draw(M, r)
    a, b = draw(1, r, K).to(TYPES[w]), draw(1, 64, r).to(TYPES[w])
    rows = lcd.group_rows(torch.zeros(M, dtype=torch.int32, device="cuda"), 1)
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    _, got_t = lcd.adapters(xs, a, b, rows, want_t=True, dtype=torch.float32, status_word=word)
    _, da, db = lcd.adapters_grad(dy, xs, a, b, t, rows, want_dx=False, grad_dtype=torch.float32, status_word=word)
    want_t, dt = xs.double() @ a[0].double().t(), dy.double() @ b[0].double()
    for got, want in ((got_t, want_t), (da[0], dt.t() @ xs.double()), (db[0], dy.double().t() @ t.double())):
        assert (got.double() - want).norm() <= (most * 2.0 ** -23 + 2.0 ** -19) * want.norm()
    assert word.item() == 0

"""Microscaled 4-bit floating point on the GPU against the float64 oracle.  Codes and scales are bit-exact; what they stand for is
exact up to the output type's rounding; products are held to the bound derived at check_product."""
import numpy as np
import pytest
import torch

import paper_2506_12038_b200 as lcd
from oracle import train_oracle as O

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


def host(t):
    return t.detach().double().cpu().numpy()


def random_x(seed, M, K, type="fp32", pitch=0):
    """Values of many magnitudes, zeros and whole zero blocks among them; rows `pitch` elements longer than K."""
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(M, K)) * np.exp(rng.normal(size=(M, K))) * 2.0 ** rng.integers(-6, 6, size=(M, 1))
    x[rng.random((M, K)) < 0.05] = 0.0
    if K > 64:
        x[:, 32:64] = 0.0
    full = torch.full((M, K + pitch), float("nan"), dtype=TYPES[type], device="cuda")
    full[:, :K] = torch.from_numpy(x).to(TYPES[type])
    return full[:, :K]


def random_mx(seed, rows, K):
    """Microscaled rows as a checkpoint holds them: any codes, scales within 2^+-8; columns beyond K hold code 0."""
    rng = np.random.default_rng(seed)
    blocks = -(-K // 32)
    codes = rng.integers(0, 16, size=(rows, blocks * 32), dtype=np.uint8)
    codes[:, K:] = 0
    scales = rng.integers(119, 136, size=(rows, blocks), dtype=np.uint8)
    packed = O.mx_codes(codes)
    room = torch.full((rows, -(-blocks // 16) * 16), 255, dtype=torch.uint8, device="cuda")      # what lies between rows is NaN
    room[:, :blocks] = torch.from_numpy(scales)
    return torch.from_numpy(packed).cuda(), room[:, :blocks], packed, scales


def check_quantize(x, inv=None):
    codes, scales = lcd.mx_quantize(x, inv)
    ref, bytes_ = O.mx_quantize(host(x), None if inv is None else host(inv))
    assert np.array_equal(scales.cpu().numpy(), bytes_)
    assert np.array_equal(codes.cpu().numpy(), O.mx_codes(ref))
    return codes, scales


@pytest.mark.parametrize("type", sorted(TYPES))
@pytest.mark.parametrize("M,K,pitch,smooth", [(1, 1, 0, False), (1, 31, 0, True), (3, 32, 0, False), (2, 33, 0, True), (5, 250, 0, True),
                                              (4, 256, 8, True), (3, 511, 1, False), (1, 4096, 0, True), (7, 2056, 0, True), (333, 1001, 0, True),
                                              (2, 11008, 3, False)])
def test_quantize_bit_exact(type, M, K, pitch, smooth):
    x = random_x(M + K, M, K, type, pitch)
    inv = torch.from_numpy((0.05 + np.random.default_rng(K).random(K)).astype(np.float32)).cuda() if smooth else None
    codes, scales = check_quantize(x, inv)
    assert codes.shape == (M, 16 * -(-K // 32)) and scales.shape == (M, -(-K // 32)) and scales.stride(0) % 16 == 0


@pytest.mark.parametrize("type", sorted(TYPES))
@pytest.mark.parametrize("M,K,pitch", [(9600, 40, 0), (5000, 256, 0), (1300, 1100, 0), (1300, 1101, 0), (1237, 2050, 6), (700, 4097, 3)])
def test_many_rows(type, M, K, pitch):
    # several rows a thread, aligned and not, there and back
    x = random_x(M + K, M, K, type, pitch)
    codes, scales = check_quantize(x)
    v = O.mx_values(codes.cpu().numpy(), scales.cpu().numpy(), K)
    for out in sorted(TYPES):
        room = torch.full((M + 1, K + pitch), 7.0, dtype=TYPES[out], device="cuda")
        lcd.mx_dequantize(codes, scales, K, out=room[:M, :K])
        assert torch.equal(room[:M, :K], torch.from_numpy(v).cuda().to(TYPES[out])) and (room[M] == 7).all() and (room[:, K:] == 7).all()


@pytest.mark.parametrize("offset", range(8))
def test_quantize_rows_at_every_offset(offset):
    room = random_x(7, 1, 3 * 300 + 8, "fp16")[0]
    check_quantize(room[offset:offset + 900].view(3, 300))


def test_quantize_ties_and_extremes():
    x = torch.zeros(12, 64, device="cuda")
    x[0, :8] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0])
    x[1, :8] = -x[0, :8]
    x[2, 0], x[2, 1] = 7.999, 4.9999995
    x[3, 3] = float("inf")
    x[4, 40] = float("nan")
    x[5, 0] = 3.4028234663852886e38
    x[6, 0] = 2.0 ** -149
    x[7, :3] = torch.tensor([2.0 ** -126, 2.0 ** -127, 2.0 ** -140])
    x[8, :2] = torch.tensor([2.0 ** 30, 1e-30])
    x[9, 0] = -0.0
    x[10, 0] = -float("inf")
    x[11, 0] = -float("nan")
    codes, scales = check_quantize(x)
    v = lcd.mx_dequantize(codes, scales)
    for row, half in ((3, 0), (4, 1), (10, 0), (11, 0)):
        assert v[row, 32 * half:32 * half + 32].isnan().all() and not v[row, 32 * (1 - half):32 * (1 - half) + 32].isnan().any()
    # a factor that takes a value beyond the range makes its block NaN, as an infinity does
    check_quantize(x, torch.full((64,), 1e3, device="cuda"))


def test_quantize_writes_its_rows_only():
    x = random_x(3, 5, 70)
    codes, scales = torch.full((5, 64), 77, dtype=torch.uint8, device="cuda"), torch.full((5, 16), 77, dtype=torch.uint8, device="cuda")
    c, s = lcd.mx_quantize(x, codes=codes[:, :48], scales=scales[:, :3])
    want = lcd.mx_quantize(x)
    assert torch.equal(c, want[0]) and torch.equal(s, want[1])
    assert (codes[:, 48:] == 77).all() and (scales[:, 3:] == 77).all()


@pytest.mark.parametrize("type", sorted(TYPES))
@pytest.mark.parametrize("M,K,pitch", [(1, 1, 0), (3, 33, 0), (5, 250, 6), (2, 4096, 0), (9, 1001, 7)])
def test_dequantize(type, M, K, pitch):
    codes, scales, packed, bytes_ = random_mx(K, M, K)
    out = torch.full((M, K + pitch), 7.0, dtype=TYPES[type], device="cuda")
    got = lcd.mx_dequantize(codes, scales, K, out=out[:, :K])
    # every value of these scales has two significant bits and lies in the normal range of all three types
    assert np.array_equal(host(got), O.mx_values(packed, bytes_, K)) and (out[:, K:] == 7).all()
    assert torch.equal(lcd.mx_dequantize(codes, scales, K, dtype=TYPES[type]), got)


def test_dequantize_every_code_and_scale():
    codes = torch.tensor([[(2 * i) % 16 | ((2 * i + 1) % 16) << 4 for i in range(8)] * 2], dtype=torch.uint8, device="cuda").repeat(256, 1)
    scales = torch.zeros(256, 16, dtype=torch.uint8, device="cuda")
    scales[:, 0] = torch.arange(256)
    v = O.mx_values(codes.cpu().numpy(), scales[:, :1].cpu().numpy())
    got = host(lcd.mx_dequantize(codes, scales[:, :1]))
    assert np.isnan(got[255]).all() and np.isnan(v[255]).all()
    with np.errstate(over="ignore"):
        want = v.astype(np.float32).astype(np.float64)           # 6 * 2^126 and the like are infinite in binary32
    assert np.array_equal(got[:255], want[:255])
    half = lcd.mx_dequantize(codes, scales[:, :1], dtype=torch.float16)
    assert torch.equal(half[:255], torch.from_numpy(want[:255]).to(torch.float32).half().cuda())


# --------------------------------------------------------------------------------------------------------- the product
def check_product(y, w, x, product=None):
    """The error of binary32 sums.  Products of elements are exact; S is the sum of the products' magnitudes.  A tensor-core
    instruction adds the 64 columns of two blocks to the sum: it aligns their terms to the largest and keeps at least 24 bits of
    it, so each of the 64 + 1 terms loses less than 2^-23 of at most S: together, for K / 64 instructions, less than
    (K / 64) * 65 * 2^-23 * S if every term were as large as S.  Terms are S / 64 on average, and what is lost is a share of the
    largest term of an instruction or of the sum so far: (K / 32 + 8) * 2^-22 * S bounds it with room for the sums of K's parts.
    The rounding to y's type adds half a step, and its smallest subnormal half of itself."""
    y64, size = O.mx_linear(w[2], w[3], x[2], x[3]) if product is None else product
    got = host(y)
    step = 0.0 if y.dtype == torch.float32 else torch.finfo(y.dtype).eps / 2
    blocks = w[3].shape[1]
    bound = (blocks + 8) * 2.0 ** -22 * size + step * np.abs(y64) * 1.001 + (2.0 ** -25 if y.dtype == torch.float16 else 0.0)
    assert got.shape == y64.shape and np.isfinite(got).all()
    assert (np.abs(got - y64) <= bound).all(), (np.abs(got - y64) / np.maximum(bound, 1e-300)).max()


SHAPES = [(1, 1, 1), (1, 8, 32), (3, 128, 64), (1, 130, 500), (2, 257, 1024), (5, 40, 4096), (8, 129, 544), (16, 384, 512), (17, 100, 96),
          (33, 300, 1500), (64, 128, 2048), (100, 250, 333), (129, 511, 640), (300, 200, 250), (513, 640, 1000)]


@pytest.mark.parametrize("M,N,K", SHAPES)
def test_product(M, N, K):
    w, x = random_mx(N * 7 + K, N, K), random_mx(M + K, M, K)
    check_product(lcd.mx_linear(w[0], w[1], x[0], x[1]), w, x)


@pytest.mark.parametrize("type", ["fp32", "bf16"])
@pytest.mark.parametrize("M,N,K", [(577, 5003, 2049), (1537, 9001, 40), (1000, 14001, 3000), (2050, 2600, 777)])
def test_product_of_many_tokens(M, N, K, type):
    # several tiles a CTA, pairs of CTAs, the widest tiles, the last of them ragged (the oracle's product in float64 on the GPU)
    w, x = random_mx(N * 7 + K, N, K), random_mx(M + K, M, K)
    a, b = (torch.from_numpy(O.mx_values(t[2], t[3])).cuda() for t in (x, w))
    product = (host(a @ b.t()), host(a.abs() @ b.abs().t()))
    y = torch.full((M + 1, N), 7.0, dtype=TYPES[type], device="cuda")
    lcd.mx_linear(w[0], w[1], x[0], x[1], y=y[:M])
    check_product(y[:M], w, x, product)
    assert (y[M] == 7).all()
    again = torch.zeros_like(y[:M])
    for _ in range(3):
        lcd.mx_linear(w[0], w[1], x[0], x[1], y=again)
        assert torch.equal(again, y[:M])


@pytest.mark.parametrize("type", ["fp16", "bf16"])
@pytest.mark.parametrize("M,N,K", [(1, 130, 500), (7, 128, 4096), (200, 333, 700)])
def test_product_types(type, M, N, K):
    w, x = random_mx(N * 7 + K, N, K), random_mx(M + K, M, K)
    x[1].sub_(8)                  # within fp16's range
    x = (*x[:3], x[3] - 8)
    check_product(lcd.mx_linear(w[0], w[1], x[0], x[1], dtype=TYPES[type]), w, x)


@pytest.mark.parametrize("M,N,K", [(1, 4096, 4096), (4, 300, 28672), (40, 256, 11008), (300, 260, 5001)])
def test_product_of_whole_numbers_is_exact(M, N, K):
    # scales 2^0, so that every product is a multiple of 1/4 and every sum less than 2^24 of them: exact in any order
    w, x = random_mx(N + K, N, K), random_mx(M, M, K)
    w[1].fill_(127)
    x[1].fill_(127)
    y64, size = O.mx_linear(w[2], np.full_like(w[3], 127), x[2], np.full_like(x[3], 127))
    assert size.max() * 4 < 2 ** 24
    assert np.array_equal(host(lcd.mx_linear(w[0], w[1], x[0], x[1])), y64)


@pytest.mark.parametrize("M", [1, 20, 200])
def test_product_of_every_scale(M):
    # one row per scale byte pair: the power of two of the product is right over the range of binary32
    N, K = 255, 64
    w, x = random_mx(1, N, K), random_mx(2, M, K)
    bytes_ = torch.arange(255, dtype=torch.uint8, device="cuda")
    w[1].copy_(bytes_[:, None].expand(-1, 2))
    x[1].fill_(127)
    y64, size = O.mx_linear(w[2], w[1].cpu().numpy(), x[2], x[1].cpu().numpy())
    got = host(lcd.mx_linear(w[0], w[1], x[0], x[1]))
    fine = (size < 2.0 ** 127) & (size > 2.0 ** -100)
    assert fine.sum() > 200 * M and np.array_equal(got[fine], y64[fine])
    # below: a flush to zero loses less than the smallest normal number a term
    small = size <= 2.0 ** -100
    assert (np.abs(got - y64)[small] <= 65 * 2.0 ** -126).all()


@pytest.mark.parametrize("M", [1, 12, 150])
def test_nan_stays_in_its_row(M):
    w, x = random_mx(5, 200, 600), random_mx(6, M, 600)
    w[1][17, 3] = 255
    x[1][M - 1, 18] = 255
    y = lcd.mx_linear(w[0], w[1], x[0], x[1])
    nan = torch.zeros_like(y, dtype=torch.bool)
    nan[:, 17] = True
    nan[M - 1] = True
    assert torch.equal(y.isnan(), nan)


@pytest.mark.parametrize("M,N,K", [(1, 300, 1000), (12, 129, 4096), (70, 200, 333), (260, 513, 777)])
@pytest.mark.parametrize("type", sorted(TYPES))
def test_fused_call_equals_two_calls(M, N, K, type):
    w = random_mx(N, N, K)
    x = random_x(M, M, K, type, 3)
    inv = torch.rand(K, device="cuda") + 0.1
    y = lcd.mx_linear_fused(w[0], w[1], x, inv)
    codes, scales = lcd.mx_quantize(x, inv)
    assert torch.equal(y, lcd.mx_linear(w[0], w[1], codes, scales))
    check_product(y, w, (None, None, codes.cpu().numpy(), scales.cpu().numpy()))


@pytest.mark.parametrize("M", [1, 9, 130])
def test_outputs_and_operands_with_longer_rows(M):
    N, K = 140, 992
    w, x = random_mx(1, N, K), random_mx(2, M, K)
    wide = lambda t, more: torch.cat([t, torch.full((t.shape[0], more), 255, dtype=torch.uint8, device="cuda")], dim=1)[:, :t.shape[1]]
    room = torch.full((M + 2, N + 5), 7.0, device="cuda")
    y = room[1:M + 1, :N]
    out = lcd.mx_linear(wide(w[0], 32), wide(w[1], 16 - 31 % 16 + 16), wide(x[0], 16), wide(x[1], 1), y=y)
    assert out is y and torch.equal(y, lcd.mx_linear(w[0], w[1], x[0], x[1]))
    assert (room[0] == 7).all() and (room[M + 1] == 7).all() and (room[:, N:] == 7).all()


def test_results_do_not_change_from_run_to_run():
    for M, N, K in ((1, 4096, 4096), (16, 1000, 5000), (300, 1000, 700)):
        w, x = random_mx(N, N, K), random_mx(M, M, K)
        y = lcd.mx_linear(w[0], w[1], x[0], x[1])
        assert all(torch.equal(y, lcd.mx_linear(w[0], w[1], x[0], x[1])) for _ in range(5))


@pytest.mark.parametrize("M", [1, 200])
def test_weights_that_the_call_before_wrote(M):
    # a training loop's order: weights quantised, used at once, quantised again
    x = random_x(9, M, 2048)
    w0, w1 = random_x(1, 1024, 2048), random_x(2, 1024, 2048)
    codes, scales = lcd.mx_quantize(w0)
    want = [lcd.mx_linear_fused(*lcd.mx_quantize(w), x) for w in (w0, w1)]
    torch.cuda.synchronize()
    for _ in range(20):
        for w, y in ((w1, want[1]), (w0, want[0])):
            lcd.mx_quantize(w, codes=codes, scales=scales)
            assert torch.equal(lcd.mx_linear_fused(codes, scales, x), y)


@pytest.mark.parametrize("M", [3, 40])           # one launch, two
def test_on_another_stream_and_in_a_graph(M):
    w = random_mx(3, 500, 1000)
    xs = [random_x(s, M, 1000) for s in (1, 2)]
    want = [lcd.mx_linear_fused(w[0], w[1], x) for x in xs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = lcd.mx_linear_fused(w[0], w[1], xs[0], stream=side)
    side.synchronize()
    assert torch.equal(y, want[0])
    x, out = xs[0].clone(), torch.empty_like(want[0])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        lcd.mx_linear_fused(w[0], w[1], x, y=out)
    for k in (1, 0, 1):
        x.copy_(xs[k])
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[k])


def test_status_word_untouched():
    w, x = random_mx(3, 500, 1000), random_mx(4, 40, 1000)
    word = torch.full((1,), 7, dtype=torch.int32, device="cuda")
    lcd.mx_linear(w[0], w[1], x[0], x[1], status_word=word)
    assert word.item() == 7


def test_offsets_beyond_32_bits():
    # 2.3 GB of codes: rows behind the 2^31st byte, against the same rows alone (whole-number sums, exact in any order)
    N, K = 140_032, 32768
    codes = torch.randint(0, 256, (N, K // 2), dtype=torch.uint8, device="cuda")
    scales = torch.full((N, K // 32), 127, dtype=torch.uint8, device="cuda")
    x = random_mx(1, 3, K)
    x[1].fill_(127)
    y = lcd.mx_linear(codes, scales, x[0], x[1])
    for lo in (0, 65536, N - 300):
        part = lcd.mx_linear(codes[lo:lo + 300], scales[lo:lo + 300], x[0], x[1])
        assert torch.equal(y[:, lo:lo + 300], part)
    v = lcd.mx_dequantize(codes, scales, dtype=torch.bfloat16)         # 4.6e9 values
    assert torch.equal(v[N - 2:], lcd.mx_dequantize(codes[N - 2:], scales[N - 2:], dtype=torch.bfloat16))
    again = lcd.mx_quantize(v)
    assert torch.equal(lcd.mx_dequantize(*again, dtype=torch.bfloat16)[N - 2:], v[N - 2:])
    wide = torch.zeros(2, 2 ** 31 + 64, dtype=torch.bfloat16, device="cuda")[:, :100]     # rows further apart than 2^31 elements
    wide.copy_(v[:2, :100])
    c, s = lcd.mx_quantize(wide)
    assert torch.equal(lcd.mx_dequantize(c, s, 100, dtype=torch.bfloat16), lcd.mx_dequantize(*lcd.mx_quantize(wide.contiguous()), 100, dtype=torch.bfloat16))


def test_calls_of_several_threads_and_streams_at_once():
    import concurrent.futures
    work = [(1, 700, 3000), (12, 384, 4096), (50, 500, 1000), (300, 512, 2048)]
    w = [random_mx(i, N, K) for i, (M, N, K) in enumerate(work)]
    x = [random_x(i, M, K, "bf16") for i, (M, N, K) in enumerate(work)]
    want = [lcd.mx_linear_fused(a[0], a[1], b) for a, b in zip(w, x)]
    torch.cuda.synchronize()

    def loop(i):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            got = [lcd.mx_linear_fused(w[i][0], w[i][1], x[i]) for _ in range(50)]
            stream.synchronize()
            return all(torch.equal(g, want[i]) for g in got)
    with concurrent.futures.ThreadPoolExecutor(4) as pool:
        assert all(pool.map(loop, range(4)))


def test_between_the_lookup_kernels():
    # kernels that begin before the one ahead of them has ended, of both kinds, in turn
    from synth import gen
    L = gen.random_case(seed=9, N=512, K=2048, bits=3, M=12)
    pw = lcd.PackedWeights(lcd.pack_weights(L.idx, L.codebook, 3))
    xh, inv = torch.from_numpy(L.x).cuda(), torch.from_numpy(L.inv_s).cuda()
    w = random_mx(2, 512, 2048)

    def both():
        a, s = lcd.smooth_quantize_act(xh, inv)
        y = lcd.lut_linear(pw, a, s)
        z = lcd.mx_linear_fused(w[0], w[1], y[:, :512].repeat(1, 4), inv)
        return y, z, lcd.mx_linear_fused(w[0], w[1], xh, inv)
    want = both()
    torch.cuda.synchronize()
    for _ in range(30):
        assert all(torch.equal(g, v) for g, v in zip(both(), want))

"""Plans, experts' products and adapters on the GPU against the float64 oracle: plans are exact, whole numbers are exact, everything else is held
to bounds derived at `close`."""
import numpy as np
import pytest
import torch

import paper_2506_12038_b200 as lcd
from oracle import groups_oracle as O
from oracle import train_oracle as MX

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "fp16": torch.float16, "bf16": torch.bfloat16}


def host(t):
    return t.detach().double().cpu().numpy()


def cuda(a, type="fp32"):
    return torch.from_numpy(np.ascontiguousarray(a)).to(TYPES[type]).cuda()


def wide(t, pitch):
    """The same matrix (or matrices) with rows `pitch` elements longer, NaN between them."""
    room = torch.full((*t.shape[:-1], t.shape[-1] + pitch), float("nan"), dtype=t.dtype, device="cuda")
    room[..., :t.shape[-1]] = t
    return room[..., :t.shape[-1]]


def step(dtype):
    return 0.0 if dtype == torch.float32 else torch.finfo(dtype).eps / 2


def close(got, want, bound):
    """bound: of the value before it is rounded to its type; that rounding adds half a step, fp16's smallest step half of itself."""
    v = host(got)
    bound = bound + step(got.dtype) * (np.abs(want) + bound) + np.abs(want) * 2.0 ** -24 + (2.0 ** -25 if got.dtype == torch.float16 else 1e-37)
    worst = (np.abs(v - want) - bound).max()
    assert (np.abs(v - want) <= bound).all(), worst


def plan_of(group, G):
    rows = lcd.group_rows(torch.from_numpy(np.asarray(group)).cuda(), G)
    for got, want in zip(rows, O.group_rows(group, G)):
        assert np.array_equal(got.cpu().numpy(), want)
    return rows


# ------------------------------------------------------------------------------------------------------------ the plan
@pytest.mark.parametrize("count,G", [(1, 1), (1, 1024), (5, 3), (31, 2), (32, 32), (33, 7), (257, 1), (1000, 64), (1025, 1000), (4096, 8), (4097, 8),
                                     (9001, 1024), (70000, 129)])
@pytest.mark.parametrize("dtype", [np.int32, np.int64])
def test_plan(count, G, dtype):
    rng = np.random.default_rng(count + G)
    group = rng.integers(-2, G + 2, size=count).astype(dtype)
    if dtype == np.int64 and count > 3:
        group[1], group[2] = 1 << 32, -(1 << 32)           # low words that would be groups
    plan_of(group, G)
    plan_of(np.full(count, G - 1, dtype=dtype), G)
    plan_of(np.full(count, -1, dtype=dtype), G)
    plan_of(np.sort(group), G)


def test_plan_into_given_tensors_and_shapes():
    group = torch.tensor([[2, 0], [-1, 2]], device="cuda")
    order, groups, offsets = (torch.full((n,), 77, dtype=torch.int32, device="cuda") for n in (6, 6, 6))
    rows = lcd.group_rows(group, 3, order[1:5], groups[1:5], offsets[1:5])
    assert rows.order.tolist() == [1, 0, 3, 2] and rows.groups.tolist() == [0, 2, 2, -1] and rows.offsets.tolist() == [0, 1, 1, 3]
    for t in (order, groups, offsets):
        assert t[0] == 77 and t[5] == 77
    with pytest.raises(lcd.LcdError):
        lcd.group_rows(group, 1025)
    with pytest.raises(lcd.LcdError):
        lcd.group_rows(group[:0], 3)


# ------------------------------------------------------------------------------------------------------------ experts
def random_experts(seed, G, N, K):
    """Experts as a checkpoint holds them: any codes, scales within 2^+-4; columns beyond K hold code 0, NaN lies between rows of scales."""
    rng = np.random.default_rng(seed)
    blocks = -(-K // 32)
    codes = rng.integers(0, 16, size=(G, N, blocks * 32), dtype=np.uint8)
    codes[:, :, K:] = 0
    scales = rng.integers(123, 132, size=(G, N, blocks), dtype=np.uint8)
    packed = (codes[:, :, 0::2] | (codes[:, :, 1::2] << 4)).astype(np.uint8)
    room = torch.full((G, N, -(-blocks // 16) * 16), 255, dtype=torch.uint8, device="cuda")
    room[:, :, :blocks] = torch.from_numpy(scales)
    values = np.stack([MX.mx_values(packed[g], scales[g], K) for g in range(G)])
    return torch.from_numpy(packed).cuda(), room[:, :, :blocks], values


def check_experts(T, k, G, N, K, type="fp32", out="fp32", smooth=False, pitch=0, group=None, seed=0, y=None):
    rng = np.random.default_rng(seed + T + N + K)
    codes, scales, w = random_experts(seed + N, G, N, K)
    x = wide(cuda(rng.normal(size=(T, K)) * np.exp(rng.normal(size=(T, K))), type), pitch)
    inv = cuda(0.05 + rng.random(K)) if smooth else None
    if group is None:
        group = rng.integers(-1, G + 1, size=(T, k))
    group = np.asarray(group).reshape(-1)
    rows = plan_of(group, G)
    got = lcd.mx_linear_grouped(codes, scales, x, rows, inv, y=y, dtype=TYPES[out])
    xc, xs = MX.mx_quantize(host(x), None if inv is None else host(inv))
    want, size = O.grouped(MX.mx_values(MX.mx_codes(xc), xs, K), w, group, k)
    # as for lcd.mx_linear: an instruction of 64 columns keeps 24 bits of its largest term and the sum so far
    close(got, want, (-(-K // 32) + 8) * 2.0 ** -22 * size)
    assert (got[torch.from_numpy((group < 0) | (group >= G)).cuda()] == 0).all()
    return got


@pytest.mark.parametrize("type,out", [("fp32", "fp32"), ("fp16", "bf16"), ("bf16", "fp16")])
@pytest.mark.parametrize("T,k,G,N,K,pitch", [(1, 1, 1, 1, 1, 0), (1, 4, 8, 130, 600, 0), (1, 2, 3, 1000, 64, 3), (3, 2, 5, 127, 250, 0), (7, 1, 2, 128, 2048, 8),
                                             (40, 3, 4, 300, 511, 1), (200, 2, 6, 200, 320, 0), (333, 4, 3, 257, 1001, 0), (5, 8, 40, 64, 96, 0)])
def test_experts(type, out, T, k, G, N, K, pitch):
    check_experts(T, k, G, N, K, type, out, smooth=K % 2 == 0, pitch=pitch)


@pytest.mark.parametrize("sizes", [[0, 0, 0], [17, 0, 0, 5], [0, 1, 0, 0, 300, 2], [128, 16, 33, 64, 1], [257, 256, 255], [600, 0, 1]])
def test_ragged_experts(sizes):
    group = np.concatenate([np.full(n, g) for g, n in enumerate(sizes)] + [np.full(3, -1)])
    np.random.default_rng(1).shuffle(group)
    check_experts(len(group), 1, len(sizes), 200, 288, group=group)


def test_every_width_of_tiles():
    # the mean size of an expert's batch picks the width
    for T in (9, 60, 120, 250, 400, 900):
        check_experts(T, 1, 4, 130, 544, group=np.random.default_rng(T).integers(0, 4, size=T))


@pytest.mark.parametrize("type", sorted(TYPES))
def test_many_tokens_of_several_choices(type):
    # a token is quantised once for its choices
    check_experts(700, 3, 5, 96, 2048, type, smooth=True)
    check_experts(1100, 4, 6, 40, 1001, type, pitch=1)
    check_experts(1100, 2, 3, 40, 2016, type, group=np.full(2200, -1))


def test_more_experts_than_a_warp_and_than_rows():
    check_experts(50, 2, 200, 40, 96)
    check_experts(2, 2, 512, 16, 64)


def test_many_tiles_a_cta():
    check_experts(64, 2, 16, 20000, 64, group=np.arange(128) % 16)


def test_experts_write_their_rows_only():
    room = torch.full((9, 50), 7.0, device="cuda")
    check_experts(4, 2, 3, 40, 64, y=room[:8, :40])
    assert (room[8] == 7).all() and (room[:, 40:] == 7).all()


def test_experts_whole_numbers_are_exact():
    rng = np.random.default_rng(3)
    T, k, G, N, K = 100, 2, 5, 140, 512
    x = rng.choice([0.0, 1.0, 2.0, -1.0, -2.0], size=(T, K))
    x[:, ::32] = 2.0                                       # the block's largest: elements are exact
    w = rng.choice([0.0, 1.0, -1.0, 4.0, -4.0], size=(G, N, K))
    w[:, :, ::32] = 4.0
    made = [lcd.mx_quantize(cuda(w[g])) for g in range(G)]
    codes = torch.stack([c for c, _ in made])
    scales = torch.zeros(G, N, 16, dtype=torch.uint8, device="cuda")
    for g, (_, s) in enumerate(made):
        scales[g] = s
    group = rng.integers(-1, G, size=(T * k))
    got = lcd.mx_linear_grouped(codes, scales, cuda(x), plan_of(group, G))
    assert np.array_equal(host(got), O.grouped(x, w, group, k)[0])


def test_experts_of_one_group_are_the_shared_product():
    codes, scales, _ = random_experts(5, 1, 333, 1024)
    x = torch.randn(77, 1024, device="cuda")
    rows = lcd.group_rows(torch.zeros(77, dtype=torch.int32, device="cuda"), 1)
    got, want = lcd.mx_linear_grouped(codes, scales, x, rows), lcd.mx_linear_fused(codes[0], scales[0], x)
    assert (got - want).abs().max() <= 2e-6 * want.abs().max()


def test_nan_stays_in_its_token_and_expert():
    codes, scales, _ = random_experts(6, 3, 64, 128)
    room = scales.clone(memory_format=torch.preserve_format)
    scales = torch.zeros(3, 64, 16, dtype=torch.uint8, device="cuda")
    scales[:, :, :4] = room
    scales[1, 5, 2] = 255
    x = torch.randn(10, 128, device="cuda")
    x[4, 7] = float("nan")
    x[6, 100] = float("inf")
    group = np.array([0, 1, 2, 0, 1, 2, 0, 1, 2, -1])
    y = host(lcd.mx_linear_grouped(codes, scales[:, :, :4], x, plan_of(group, 3)))
    bad = np.isnan(y)
    assert bad[4].all() and bad[6].all() and bad[group == 1][:, 5].all()
    bad[[4, 6]] = False
    bad[group == 1, 5] = False
    assert not bad.any() and (y[9] == 0).all()


# ------------------------------------------------------------------------------------------------------------ adapters
def loss_of(n):
    """What fp32 sums of n products lose at most, as a share of the products' magnitudes.  A tensor-core instruction of 8 or 16 columns aligns
    its addends to the largest of them and of the sum so far, which no magnitudes exceed, and keeps at least 24 bits: it loses 17 * 2^-23 for
    16 columns, or 9 * 2^-23 for each of up to three products of 8 columns' parts; the warps' and CTAs' 64 sums 2^-24 each."""
    return n / 8 * 27 * 2.0 ** -23 + 27 * 2.0 ** -23 + 64 * 2.0 ** -24


def cut_of(types, out):
    """What the parts of t or dt and of an fp32 operand beside it leave out: two bf16 parts 2^-15 (the first is cut off: at most 2^-7, the second
    rounded: 2^-9 of it, doubled for the product), three or two tf32 parts 2^-20 and 2^-20."""
    return 2.0 ** -15 if "bf16" in types and out != torch.float32 else 2.0 ** -19


def make_adapters(seed, M, G, r, K, N, x="fp32", w="fp32", out=None, pitch=0, scale=True, group=None, base=True, whole=False):
    rng = np.random.default_rng(seed)
    draw = (lambda *s: rng.integers(-2, 3, size=s).astype(np.float64)) if whole else (lambda *s: rng.normal(size=s))
    c = dict(x=wide(cuda(draw(M, K), x), pitch), a=wide(cuda(draw(G, r, K), w), pitch), b=wide(cuda(draw(G, N, r), w), pitch),
             group=rng.integers(-1, G, size=M) if group is None else np.asarray(group),
             scale=cuda(np.exp2(rng.integers(-1, 2, size=G)) if whole else 0.5 + rng.random(G)) if scale else None,
             base=wide(cuda(draw(M, N), out or x), pitch) if base else None)
    c["rows"] = plan_of(c["group"], G)
    return c


def check_adapters(c, types=(), dtype=None, exact=False, **kw):
    y, t = lcd.adapters(c["x"], c["a"], c["b"], c["rows"], c["base"], scale=c["scale"], want_t=True, dtype=dtype, **kw)
    want, t_want, t_size, y_size, y_deep = O.adapters(host(c["x"]), host(c["a"]), host(c["b"]), c["group"], None if c["base"] is None else host(c["base"]),
                                                      None if c["scale"] is None else host(c["scale"]))
    if exact:
        assert np.array_equal(host(t), t_want) and np.array_equal(host(y), want)
        return y, t
    K, r = c["x"].shape[1], c["a"].shape[1]
    lost = loss_of(K) + 2.0 ** -19 * ("fp32" in types)
    close(t, t_want, lost * t_size)
    cut = cut_of(types, y.dtype)
    close(y, want, lost * y_deep + (loss_of(r) + cut) * y_size * (1 + lost) + 2.0 ** -23 * (np.abs(want) + y_size))
    # the bound adds up worst cases; on the whole errors are much smaller (independent ones of at most the cut, or 2^-19 from sums of a few hundred)
    rms = np.linalg.norm(host(y) - want) / max(np.linalg.norm(want), 1e-30)
    assert rms <= step(y.dtype) + cut + 2.0 ** -18 + (1e-3 if y.dtype == torch.float16 and np.abs(want).max() < 1e-3 else 0)
    return y, t


PAIRS = [("fp32", "fp32"), ("fp16", "fp16"), ("bf16", "bf16"), ("fp16", "fp32"), ("bf16", "fp32"), ("fp32", "fp16"), ("fp32", "bf16")]


@pytest.mark.parametrize("x,w", PAIRS)
@pytest.mark.parametrize("M,G,r,K,N,pitch", [(1, 1, 1, 1, 1, 0), (1, 3, 16, 256, 200, 0), (2, 8, 8, 70, 33, 0), (9, 2, 12, 100, 65, 3), (40, 5, 33, 320, 130, 8),
                                             (64, 64, 16, 64, 64, 0), (100, 3, 64, 333, 129, 0), (70, 2, 100, 96, 90, 1), (130, 4, 128, 512, 264, 0)])
def test_adapters(x, w, M, G, r, K, N, pitch):
    c = make_adapters(M + r, M, G, r, K, N, x, w, pitch=pitch)
    check_adapters(c, (x, w))


@pytest.mark.parametrize("x,w", PAIRS)
@pytest.mark.parametrize("out", sorted(TYPES))
def test_adapters_types_of_y(x, w, out):
    check_adapters(make_adapters(7, 50, 3, 24, 200, 300, x, w, out), (x, w))
    check_adapters(make_adapters(8, 50, 3, 48, 200, 300, x, w, base=False), (x, w), dtype=TYPES[out])


@pytest.mark.parametrize("x,w", PAIRS)
@pytest.mark.parametrize("M,G,r,K,N", [(1, 2, 16, 4096, 1000), (33, 4, 8, 256, 700), (600, 3, 64, 128, 130), (257, 2, 128, 64, 100)])
def test_adapters_whole_numbers_are_exact(x, w, M, G, r, K, N):
    # |t| <= 4 K, |y| <= 16 K r + 2 times a power of two: below 2^24, and in two bf16 parts up to 2^16
    c = make_adapters(M, M, G, r, K, N, x, w, "fp32", whole=True)
    check_adapters(c, exact=True)


@pytest.mark.parametrize("sizes", [[0, 0, 5], [1, 1, 1, 1, 1, 1, 1], [31, 1, 0, 33, 8], [300, 7, 0, 0, 1], [16, 16, 16, 16]])
def test_adapters_ragged(sizes):
    for left in (0, 4):
        group = np.concatenate([np.full(n, g) for g, n in enumerate(sizes)] + [np.full(left, -1)])
        np.random.default_rng(2).shuffle(group)
        check_adapters(make_adapters(3, len(group), len(sizes), 20, 130, 150, "bf16", "bf16", group=group), ("bf16",))
        check_adapters(make_adapters(3, len(group), len(sizes), 20, 130, 150, "fp16", "fp16", "fp32", group=group, scale=False), ("fp16",))


MANY = [(512, 1, 16, 96, 64), (700, 3, 8, 96, 264), (1500, 9, 33, 64, 128), (513, 2, 64, 64, 520), (640, 4, 128, 64, 200), (600, 700, 12, 32, 48), (600, 5, 12, 333, 131),
        (512, 1, 64, 130, 259), (777, 3, 128, 201, 1001), (530, 2, 31, 1000, 1)]


@pytest.mark.parametrize("x,w", PAIRS)
@pytest.mark.parametrize("M,G,r,K,N", MANY)
def test_adapters_of_many_rows(x, w, M, G, r, K, N):
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    c = make_adapters(M + r, M, G, r, K, N, x, w)
    check_adapters(c, (x, w), status_word=word)
    whole = make_adapters(M + r, M, G, r, K, N, x, w, "fp32", whole=True, pitch=8)
    check_adapters(whole, exact=True, status_word=word)
    assert word.item() == 0


def test_adapters_of_many_rows_without_base_and_in_place():
    for group in (None, np.full(600, -1), np.arange(600) % 3 - 1):
        c = make_adapters(13, 600, 2, 16, 64, 136, "bf16", "bf16", base=False, group=group)
        check_adapters(c, ("bf16",))
        c["base"] = torch.randn(600, 136, device="cuda").bfloat16()
        y, _ = check_adapters(c, ("bf16",))
        room = torch.full((601, 144), 7.0, dtype=torch.bfloat16, device="cuda")
        room[:600, :136] = c["base"]
        got = lcd.adapters(c["x"], c["a"], c["b"], c["rows"], room[:600, :136], y=room[:600, :136], scale=c["scale"])
        assert torch.equal(got, y) and (room[600] == 7).all() and (room[:, 136:] == 7).all()


def test_adapters_in_place_and_beyond_their_rows():
    c = make_adapters(5, 20, 3, 16, 64, 72, "bf16", "bf16")
    y, _ = check_adapters(c, ("bf16",))
    room = torch.full((21, 80), 7.0, dtype=torch.bfloat16, device="cuda")
    room[:20, :72] = c["base"]
    t_room = torch.full((21, 20), 7.0, device="cuda")
    got, t = lcd.adapters(c["x"], c["a"], c["b"], c["rows"], room[:20, :72], y=room[:20, :72], scale=c["scale"], t=t_room[:20, :16])
    assert torch.equal(got, y) and got.data_ptr() == room.data_ptr() and (room[20] == 7).all() and (room[:, 72:] == 7).all()
    assert (t_room[20] == 7).all() and (t_room[:, 16:] == 7).all() and t.data_ptr() == t_room.data_ptr()
    none = torch.from_numpy(c["group"] < 0).cuda()
    assert torch.equal(got[none], c["base"][none]) and (t[none] == 0).all()


@pytest.mark.parametrize("times", [4, 120])
@pytest.mark.parametrize("x,w", [("bf16", "bf16"), ("fp16", "fp16"), ("fp32", "fp32")])
def test_adapters_keep_what_is_not_finite_in_its_row_and_adapter(x, w, times):
    c = make_adapters(9, 6 * times, 4, 16, 96, 80, x, w, group=[0, 1, 2, 3, -1, 0] * times)
    for key, at in (("x", (0, 5)), ("x", (4, 6)), ("a", (1, 3, 7)), ("b", (2, 9, 1))):
        c[key][at] = float("nan")
    c["x"][9, 1] = float("inf")
    y, t = lcd.adapters(c["x"], c["a"], c["b"], c["rows"], c["base"], scale=c["scale"], want_t=True)
    bad = ~torch.isfinite(y).cpu().numpy()
    group = c["group"]
    assert bad[0].all() and bad[9].all() and bad[group == 1].all() and bad[group == 2][:, 9].all()
    bad[[0, 9]] = False
    bad[group == 1] = False
    bad[group == 2, 9] = False
    assert not bad.any()
    assert torch.equal(y[4], c["base"][4]) and (t[4] == 0).all()
    assert torch.isinf(t[9]).all()                         # an infinity stays one (its other parts are left out)


@pytest.mark.parametrize("scale", [1e-30, 1e-12, 1e12, 1e30])
def test_adapters_range_of_t(scale):
    # t lies anywhere in fp32's range whatever the operands' types
    c = make_adapters(11, 12, 2, 16, 64, 40, "fp32", "bf16", base=False)
    c["x"].mul_(scale)
    y, t = lcd.adapters(c["x"], c["a"], c["b"], c["rows"], scale=c["scale"], want_t=True)
    want = O.adapters(host(c["x"]), host(c["a"]), host(c["b"]), c["group"], None, host(c["scale"]))[0]
    assert np.linalg.norm(host(y) - want) <= 2.0 ** -18 * np.linalg.norm(want)


def check_grad(c, x, types=(), exact=False, grad_dtype=None, base=True, seed=0, whole=False, **kw):
    rng = np.random.default_rng(seed + 100)
    M, K, (G, N, r) = c["x"].shape[0], c["x"].shape[1], c["b"].shape
    draw = (lambda *s: rng.integers(-2, 3, size=s).astype(np.float64)) if whole else (lambda *s: rng.normal(size=s))
    dy, t = cuda(draw(M, N), x), cuda(draw(M, r))
    dx_base = cuda(draw(M, K), x) if base else None
    got = lcd.adapters_grad(dy, c["x"], c["a"], c["b"], t, c["rows"], dx_base, scale=c["scale"], grad_dtype=grad_dtype, **kw)
    (dx, dx_size, dx_deep), (da, da_size, da_deep), (db, db_size) = O.adapters_grad(
        host(dy), host(c["x"]), host(c["a"]), host(c["b"]), host(t), c["group"], None if dx_base is None else host(dx_base),
        None if c["scale"] is None else host(c["scale"]))
    if exact:
        for g, want in zip(got, (dx, da, db)):
            assert np.array_equal(host(g), want)
        return got
    lost = loss_of(N) + 2.0 ** -19 * ("fp32" in types) + 2.0 ** -23
    close(got[0], dx, lost * dx_deep + (loss_of(r) + cut_of(types, got[0].dtype)) * dx_size * (1 + lost) + 2.0 ** -23 * (np.abs(dx) + dx_size))
    most = max(1, np.bincount(c["group"][c["group"] >= 0], minlength=1).max())
    cut = cut_of((x,), got[1].dtype)
    close(got[1], da, lost * da_deep + (loss_of(most) + cut) * da_size * (1 + lost))
    close(got[2], db, (loss_of(most) + cut + 2.0 ** -23) * db_size)
    for g, want in zip(got, (dx, da, db)):
        assert np.linalg.norm(host(g) - want) <= (step(g.dtype) + 2.0 ** -14 * ("bf16" in types and g.dtype != torch.float32) + 2.0 ** -17) * max(np.linalg.norm(want), 1e-3)
    return got


@pytest.mark.parametrize("x,w", PAIRS)
@pytest.mark.parametrize("M,G,r,K,N,pitch", [(1, 1, 1, 1, 1, 0), (1, 3, 16, 256, 200, 0), (9, 2, 12, 100, 65, 3), (40, 5, 33, 320, 130, 8),
                                             (64, 64, 16, 64, 64, 0), (100, 3, 64, 333, 129, 0), (70, 2, 100, 96, 90, 1), (600, 2, 8, 72, 520, 0)])
def test_grad(x, w, M, G, r, K, N, pitch):
    check_grad(make_adapters(M + r, M, G, r, K, N, x, w, pitch=pitch), x, (x, w))


@pytest.mark.parametrize("x,w", PAIRS)
@pytest.mark.parametrize("M,G,r,K,N", MANY)
def test_grad_of_many_rows(x, w, M, G, r, K, N):
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    c = make_adapters(M + r, M, G, r, N, K, x, w)
    check_grad(c, x, (x, w), status_word=word)
    check_grad(c, x, (x, w), status_word=word, grad_dtype=torch.float32, base=False)
    whole = make_adapters(M + r, M, G, r, N, K, x, w, whole=True, pitch=8)
    check_grad(whole, x, whole=True, exact=x == "fp32", grad_dtype=torch.float32, types=(x, w), status_word=word)
    assert word.item() == 0


@pytest.mark.parametrize("x,w", PAIRS)
@pytest.mark.parametrize("M,G,r,K,N", [(3000, 1, 16, 64, 72), (2500, 2, 40, 136, 64), (2100, 1, 8, 63, 65), (1300, 30, 32, 1000, 72), (1500, 2, 128, 200, 72),
                                       (1100, 3, 100, 137, 65)])
def test_grad_of_long_groups(x, w, M, G, r, K, N):
    # a sum over more rows than the stages in flight hold, several times around them; rows of one group against sums in whole numbers
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    whole = make_adapters(M + r, M, G, r, K, N, x, w, whole=True)
    whole["scale"] = None
    check_grad(whole, x, whole=True, exact=x == "fp32", grad_dtype=torch.float32, types=(x, w), status_word=word)
    check_grad(make_adapters(M + r, M, G, r, K, N, x, w), x, (x, w), status_word=word)
    assert word.item() == 0


@pytest.mark.parametrize("x,w", [("fp32", "fp32"), ("fp16", "fp16"), ("bf16", "fp32")])
def test_long_sums_keep_fp32s_precision(x, w):
    # 8192 terms: 128 stages of four instructions, each of which cuts its sum off (2^-24 of it at most).  They go to seven accumulators in turn:
    # 76 of them one after the other; the parts' products, the joining of the sums and what the parts leave out are within 2^-20
    g = torch.Generator(device="cuda").manual_seed(3)
    M = K = 8192
    xs, dy, t = (torch.randn(M, n, generator=g, device="cuda") for n in (K, 64, 16))
    a, b = torch.randn(1, 16, K, generator=g, device="cuda") / 64, torch.randn(1, 64, 16, generator=g, device="cuda")
    xs, dy, a, b = xs.to(TYPES[x]), dy.to(TYPES[x]), a.to(TYPES[w]), b.to(TYPES[w])
    rows = lcd.group_rows(torch.zeros(M, dtype=torch.int32, device="cuda"), 1)
    _, got_t = lcd.adapters(xs, a, b, rows, want_t=True)
    _, da, db = lcd.adapters_grad(dy, xs, a, b, t, rows, want_dx=False, grad_dtype=torch.float32)
    want_t, dt = xs.double() @ a[0].double().t(), dy.double() @ b[0].double()
    for got, want in ((got_t, want_t), (da[0], dt.t() @ xs.double()), (db[0], dy.double().t() @ t.double())):
        assert (got.double() - want).norm() <= (76 * 2.0 ** -24 + 2.0 ** -20) * want.norm()


@pytest.mark.parametrize("x,w", PAIRS)
@pytest.mark.parametrize("M,G,r,K,N", [(1, 2, 16, 1000, 256), (33, 4, 8, 700, 256), (600, 3, 64, 130, 96), (257, 2, 128, 100, 64), (2000, 1, 16, 128, 64)])
def test_grad_whole_numbers_are_exact(x, w, M, G, r, K, N):
    # |dt| <= 8 N, |da| <= 16 N M: below 2^24; dx rounds to its type, exactly where it is fp32
    c = make_adapters(M, M, G, r, K, N, x, w, whole=True)
    got = check_grad(c, x, whole=True, exact=x == "fp32", grad_dtype=torch.float32, types=(x, w))
    if x != "fp32":
        dy_seed = np.random.default_rng(100)
        dy, t = (dy_seed.integers(-2, 3, size=s).astype(np.float64) for s in ((M, N), (M, r)))
        _, (da, *_), (db, _) = O.adapters_grad(dy, host(c["x"]), host(c["a"]), host(c["b"]), t, c["group"], None, host(c["scale"]))
        assert np.array_equal(host(got[1]), da) and np.array_equal(host(got[2]), db)


@pytest.mark.parametrize("grad", sorted(TYPES))
def test_grad_types(grad):
    for x, w in PAIRS:
        check_grad(make_adapters(2, 60, 3, 24, 90, 70, x, w), x, (x, w), grad_dtype=TYPES[grad], base=grad != "fp16")


def test_grad_parts_and_given_tensors():
    c = make_adapters(4, 30, 4, 16, 64, 48, "bf16", "bf16", group=[0, 2] * 15)
    dx, da, db = check_grad(c, "bf16", ("bf16",), base=False)
    assert (da[1] == 0).all() and (db[3] == 0).all()
    dy_seed = np.random.default_rng(100)
    dy, t = cuda(dy_seed.normal(size=(30, 48)), "bf16"), cuda(dy_seed.normal(size=(30, 16)))
    args = (dy, c["x"], c["a"], c["b"], t, c["rows"])
    only = lcd.adapters_grad(dy, None, c["a"], c["b"], None, c["rows"], scale=c["scale"], want_weights=False)
    assert torch.equal(only[0], dx) and only[1] is None and only[2] is None
    only = lcd.adapters_grad(*args, scale=c["scale"], want_dx=False)
    assert only[0] is None and torch.equal(only[1], da) and torch.equal(only[2], db)
    room = torch.full((31, 72), 7.0, dtype=torch.bfloat16, device="cuda")
    room[:30, :64] = 0
    given = lcd.adapters_grad(*args, room[:30, :64], dx=room[:30, :64], scale=c["scale"], da=torch.full_like(da, 9), db=torch.full_like(db, 9))
    assert torch.equal(given[0], dx) and torch.equal(given[1], da) and torch.equal(given[2], db)
    assert (room[30] == 7).all() and (room[:, 64:] == 7).all()


def test_gradient_against_differences():
    M, G, r, K, N = 12, 2, 4, 20, 16
    c = make_adapters(21, M, G, r, K, N, base=False)
    w = torch.randn(M, N, device="cuda")

    def loss(x, a, b):
        return float((lcd.adapters(x, a, b, c["rows"], scale=c["scale"]).double() * w.double()).sum())

    x, a, b = (v.contiguous() for v in (c["x"], c["a"], c["b"]))
    _, t = lcd.adapters(x, a, b, c["rows"], scale=c["scale"], want_t=True)
    grads = lcd.adapters_grad(w, x, a, b, t, c["rows"], scale=c["scale"])
    rng = np.random.default_rng(0)
    for i, grad in enumerate(grads):
        for _ in range(6):
            d = torch.from_numpy(rng.normal(size=grad.shape)).float().cuda()
            h = 2.0 ** -6
            up, down = [[v + s * h * d if j == i else v for j, v in enumerate((x, a, b))] for s in (1, -1)]
            slope = (loss(*up) - loss(*down)) / (2 * h)          # linear in each: the difference is exact up to rounding
            want = float((grad.double() * d.double()).sum())
            size = float((grad.double() * d.double()).abs().sum()) + abs(want)
            # y is off by about 2^-20 of its terms, of which there are some M N r K^(1/2) / 2 h; an ample bound is 2^-9 of the products' magnitudes
            assert abs(slope - want) <= 2.0 ** -9 * size


# ------------------------------------------------------------------------------------------------------------ in a program
def test_streams_devices_and_repeats():
    c = make_adapters(31, 200, 6, 16, 256, 320, "bf16", "bf16")
    codes, scales, _ = random_experts(8, 4, 96, 256)
    x = torch.randn(64, 256, device="cuda")
    choice = torch.randint(-1, 4, (64, 2), device="cuda")

    def work(stream=None):
        rows = lcd.group_rows(choice, 4, stream=stream)
        y = lcd.mx_linear_grouped(codes, scales, x, rows, stream=stream)
        z, t = lcd.adapters(c["x"], c["a"], c["b"], c["rows"], c["base"], scale=c["scale"], want_t=True, stream=stream)
        return (*rows, y, z, t, *lcd.adapters_grad(z, c["x"], c["a"], c["b"], t, c["rows"], scale=c["scale"], stream=stream))

    first = work()
    for _ in range(5):
        assert all(torch.equal(a, b) for a, b in zip(first, work()))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = [work(s) for s in streams for _ in range(4)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for g in got for a, b in zip(first, g))


@pytest.mark.parametrize("x,w,r", [("fp16", "fp16", 16), ("fp16", "fp32", 64), ("bf16", "bf16", 64), ("fp32", "fp32", 32), ("bf16", "bf16", 128)])
def test_right_before_and_behind_products_that_begin_early(x, w, r):
    # kernels that hold tensor memory and let the next one begin while they run, one behind the other, of several sizes
    c = make_adapters(41, 640, 3, r, 256, 264, x, w)
    few, many, xs = (torch.randn(n, 256, device="cuda") for n in (1, 700, 40))
    codes, scales, _ = random_experts(9, 3, 300, 256)
    dy, t = torch.randn(640, 264, device="cuda").to(TYPES[x]), torch.randn(640, r, device="cuda")
    plan = lcd.group_rows(torch.arange(40, device="cuda") % 3, 3)
    word = torch.zeros(1, dtype=torch.int32, device="cuda")

    def work():
        out = []
        for v in (few, many, xs):
            out.append(lcd.adapters(c["x"], c["a"], c["b"], c["rows"], c["base"], scale=c["scale"], status_word=word))
            out.append(lcd.mx_linear_fused(codes[0], scales[0], v, status_word=word))
            out += lcd.adapters_grad(dy, c["x"], c["a"], c["b"], t, c["rows"], scale=c["scale"], status_word=word)
            out.append(lcd.mx_linear_fused(codes[1], scales[1], v, status_word=word))
            out.append(lcd.mx_linear_grouped(codes, scales, xs, plan, status_word=word))
            out += lcd.adapters_grad(dy, c["x"], c["a"], c["b"], t, c["rows"], scale=c["scale"], want_dx=False, status_word=word)[1:]
        return out

    first = work()
    torch.cuda.synchronize()
    for _ in range(20):
        again = work()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, again)) and word.item() == 0


def test_captured_and_replayed():
    codes, scales, _ = random_experts(8, 4, 96, 256)
    c = make_adapters(33, 48, 6, 16, 256, 96, "fp16", "fp16", "fp32")
    x, choice, which = c["x"].contiguous(), torch.randint(-1, 4, (48, 1), device="cuda"), torch.from_numpy(c["group"]).cuda()

    def work():
        y = lcd.mx_linear_grouped(codes, scales, x, lcd.group_rows(choice, 4))
        rows = lcd.group_rows(which, 6)
        z, t = lcd.adapters(x, c["a"], c["b"], rows, y, scale=c["scale"], want_t=True)
        return y, z, t, *lcd.adapters_grad(z.half(), x, c["a"], c["b"], t, rows, scale=c["scale"])

    work()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = work()
    for seed in range(3):
        g = torch.Generator(device="cuda").manual_seed(seed)
        x.copy_(torch.randn(48, 256, generator=g, device="cuda"))
        choice.copy_(torch.randint(-1, 4, (48, 1), generator=g, device="cuda"))
        which.copy_(torch.randint(-1, 6, (48,), generator=g, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, work()))


def test_offsets_beyond_32_bits():
    # rows of x and y, and an adapter and an expert, that begin beyond 2^31 and 2^32 elements
    free = torch.cuda.mem_get_info()[0]
    if free < 40 << 30:
        pytest.skip("needs 40 GB")
    pitch = (1 << 31) + 64
    x = torch.zeros(2 * pitch + 64, dtype=torch.bfloat16, device="cuda").as_strided((3, 64), (pitch, 1))
    x.copy_(torch.randn(3, 64, device="cuda"))
    a = torch.zeros(2 * pitch + 16 * 64, dtype=torch.bfloat16, device="cuda").as_strided((3, 16, 64), (pitch, 64, 1))
    a.copy_(torch.randn(3, 16, 64, device="cuda"))
    b = torch.randn(3, 80, 16, device="cuda").bfloat16()
    rows = plan_of(np.array([2, 1, 0]), 3)
    want = lcd.adapters(x.contiguous(), a.contiguous(), b, rows)
    y = torch.zeros(2 * pitch + 80, dtype=torch.bfloat16, device="cuda").as_strided((3, 80), (pitch, 1))
    assert torch.equal(lcd.adapters(x, a, b, rows, y=y), want) and torch.equal(y, want)
    del y, a
    codes, scales, _ = random_experts(2, 3, 40, 64)
    far = torch.zeros(2 * pitch + 40 * 32, dtype=torch.uint8, device="cuda").as_strided((3, 40, 32), (pitch, 32, 1))
    far.copy_(codes)
    room = torch.zeros(2 * pitch + 40 * 16, dtype=torch.uint8, device="cuda").as_strided((3, 40, 2), (pitch, 16, 1))
    room.copy_(scales)
    assert torch.equal(lcd.mx_linear_grouped(far, room, x, rows), lcd.mx_linear_grouped(codes, scales, x.contiguous(), rows))


def test_a_layer_of_experts_and_a_step_of_adapters():
    """As they are used together: two products of experts with an activation between them, weighted and summed; adapters beside a clustered
    layer, trained a step on the distillation loss."""
    g = torch.Generator(device="cuda").manual_seed(5)
    T, k, G, D, H = 24, 2, 6, 128, 96
    x = torch.randn(T, D, generator=g, device="cuda")
    up, down = random_experts(1, G, 2 * H, D), random_experts(2, G, D, H)
    weight, choice = torch.softmax(torch.randn(T, G, generator=g, device="cuda"), dim=1).topk(k, dim=1)
    rows = lcd.group_rows(choice, G)
    h = lcd.mx_linear_grouped(up[0], up[1], x, rows)
    h = torch.nn.functional.silu(h[:, :H]) * h[:, H:]
    y = (lcd.mx_linear_grouped(down[0], down[1], h, rows).view(T, k, D) * weight[:, :, None]).sum(dim=1)
    want = np.zeros((T, D))
    for t in range(T):
        for j in range(k):
            p, e = t * k + j, int(choice[t, j])
            xc = MX.mx_quantize(host(x[t:t + 1]))
            v = up[2][e] @ MX.mx_values(MX.mx_codes(xc[0]), xc[1], D)[0]
            hc = MX.mx_quantize(host(h[p:p + 1]))                # the kernel's own h: its 4-bit rounding is a step function
            assert np.allclose(host(h[p]), v[:H] / (1 + np.exp(-v[:H])) * v[H:], rtol=1e-4, atol=1e-4 * np.abs(v).max())
            want[t] += float(weight[t, j]) * (down[2][e] @ MX.mx_values(MX.mx_codes(hc[0]), hc[1], H)[0])
    assert np.linalg.norm(host(y) - want) <= 1e-5 * np.linalg.norm(want)

    rng = np.random.default_rng(0)
    V, r, A = 200, 8, 3
    w = lcd.PackedWeights(lcd.pack_weights(rng.integers(0, 4, size=(V, D), dtype=np.uint8), np.sort(rng.normal(size=(V, 4)), axis=1).astype(np.float16), 2))
    xh = x.half()
    idx, scale = lcd.smooth_quantize_act(xh)
    base = lcd.lut_linear(w, idx, scale)
    which = torch.randint(-1, A, (T,), generator=g, device="cuda")
    plan = lcd.group_rows(which, A)
    a = (torch.randn(A, r, D, generator=g, device="cuda") / 8).half()
    b = (torch.randn(A, V, r, generator=g, device="cuda") / 8).half()
    logits, t = lcd.adapters(xh, a, b, plan, base, want_t=True)
    top, at = torch.randn(T, V, generator=g, device="cuda").topk(5, dim=1)
    loss, dz = lcd.distill_loss(logits, at.int(), top, want_grad=True)
    dx, da, db = lcd.adapters_grad(dz.half(), xh, a, b, t, plan, grad_dtype=torch.float32)
    # the same by torch's own differentiation
    x_, a_, b_ = (v.double().requires_grad_() for v in (xh, a, b))
    z = base.double()
    for e in range(A):
        z = z + torch.where((which == e)[:, None], x_ @ a_[e].t() @ b_[e].t(), torch.zeros_like(z))
    q, p = torch.log_softmax(z, dim=1).gather(1, at), torch.softmax(top.double(), dim=1)
    total = (p * (p.log() - q)).sum(dim=1)
    total.sum().backward()
    assert torch.allclose(loss.double(), total, rtol=1e-4, atol=1e-4)
    for got, ref in ((dx, x_.grad), (da, a_.grad), (db, b_.grad)):
        assert (got.double() - ref).norm() <= 2e-3 * ref.norm()      # dz in fp16: 2^-11, and its small entries

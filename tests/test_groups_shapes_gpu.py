"""Every form of the product of experts that its plan can choose (tiles of 16 to 256 tokens, pairs of CTAs, columns cut over a cluster), each asserted by
name, with ragged experts: none, one token, a box of rows and one less or more, a whole tile and one less or more."""
import numpy as np
import pytest
import torch

import paper_2506_12038_b200 as lcd
from oracle import train_oracle as MX
from test_groups_gpu import TYPES

pytestmark = pytest.mark.gpu

# (tokens of a tile, CTAs that share its columns, pairs): rows, experts, N, K
SHAPES = {
    (16, 1, False): [(24, 8, 300, 250), (1, 3, 129, 64)], (16, 2, False): [(8, 8, 520, 8200), (2, 8, 4096, 14336)], (16, 4, False): [(8, 5, 300, 8200)],
    (16, 8, False): [(16, 5, 40, 4090)],
    (32, 1, False): [(512, 5, 520, 100), (300, 5, 1000, 100)], (32, 2, False): [(200, 5, 520, 14300)], (32, 4, False): [(128, 5, 300, 8200)],
    (32, 8, False): [(40, 8, 40, 4090)],
    (64, 1, False): [(1500, 8, 520, 100), (700, 12, 1000, 100)], (64, 2, False): [(512, 5, 520, 14300)], (64, 4, False): [(300, 5, 300, 8200)],
    (64, 8, False): [(64, 8, 40, 14300)],
    (128, 1, False): [(3000, 8, 520, 100), (2048, 5, 1000, 100), (8192, 32, 4096, 2048)], (128, 2, False): [(2048, 5, 300, 14300)],
    (128, 4, False): [(700, 5, 300, 14300)],
    (192, 1, False): [(8192, 12, 300, 2000), (3000, 5, 1000, 2000)], (192, 2, False): [(12000, 5, 40, 14300)],
    (192, 4, False): [(4096, 12, 40, 14300), (1500, 5, 300, 14300)],
    (256, 1, False): [(12000, 5, 300, 14300)], (256, 2, False): [(16384, 1, 40, 28000)], (256, 4, False): [(8192, 5, 40, 14300)],
    (192, 1, True): [(3000, 8, 1000, 4090), (12000, 5, 130, 4090)], (256, 1, True): [(4096, 5, 1000, 8200), (16384, 12, 130, 14300)],
}
CASES = [(form, *size) for form, sizes in SHAPES.items() for size in sizes]
E2M1 = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], dtype=torch.float64)


def decoded(codes, scales, K):
    """What codes [..., bytes] and scales [..., blocks] stand for, in 64 bits."""
    table = E2M1.to(codes.device)
    v = torch.stack([table[(codes & 15).long()], table[(codes >> 4).long()]], dim=-1).flatten(-2)
    return (v.unflatten(-1, (-1, 32)) * torch.exp2(scales.double() - 127)[..., None]).flatten(-2)[..., :K]


def ragged(rows, G, tile, seed):
    """A group for every row: experts of the sizes where a tile or one of its boxes ends, the last one with what is left, some rows without."""
    wish = [1, 0, tile + 1, tile - 1, tile, 33, 64, 65, 31, 2 * tile + 1, 63, 32]
    sizes, left = [], rows - rows // 17
    for g in range(G - 1):
        sizes.append(min(wish[g % len(wish)], max(0, left // 2)))
        left -= sizes[-1]
    group = np.concatenate([np.full(n, g) for g, n in enumerate(sizes + [left])] + [np.full(rows // 17, -1)])
    np.random.default_rng(seed).shuffle(group)
    return torch.from_numpy(group).cuda()


def product(x, w, group, k):
    want, size = (torch.zeros(len(group), w.shape[1], dtype=torch.float64, device="cuda") for _ in range(2))
    for e in range(w.shape[0]):
        p = (group == e).nonzero().flatten()
        if len(p):
            want[p] = x[p // k] @ w[e].t()
            size[p] = x[p // k].abs() @ w[e].abs().t()
    return want, size


def experts(seed, G, N, K, plain):
    g = torch.Generator(device="cuda").manual_seed(seed)
    blocks = -(-K // 32)
    codes = torch.randint(0, 256, (G, N, blocks * 16), dtype=torch.uint8, device="cuda", generator=g)
    cut = torch.zeros(blocks * 32, dtype=torch.uint8, device="cuda")
    cut[:K] = 15
    codes &= cut[::2] | cut[1::2] << 4
    room = torch.full((G, N, -(-blocks // 16) * 16), 255, dtype=torch.uint8, device="cuda")
    room[:, :, :blocks] = 127 if plain else torch.randint(123, 132, (G, N, blocks), dtype=torch.uint8, device="cuda", generator=g)
    return codes, room[:, :, :blocks]


def test_decoding_is_the_oracles():
    codes, scales = experts(1, 2, 5, 70, False)
    for e in range(2):
        assert np.array_equal(decoded(codes[e], scales[e], 70).cpu().numpy(), MX.mx_values(codes[e].cpu().numpy(), scales[e].cpu().numpy(), 70))


@pytest.mark.parametrize("form,rows,G,N,K", CASES)
def test_forms(form, rows, G, N, K):
    assert lcd.resolve_mx_linear_grouped(rows, G, N, K) == form
    k = 2 if rows % 2 == 0 else 1
    group = ragged(rows, G, form[0], rows)
    plan = lcd.group_rows(group, G)
    none = group < 0
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(N)
    # random numbers, into rows off 16 bytes with others around
    codes, scales = experts(K, G, N, K, False)
    x = torch.randn(rows // k, K, device="cuda", generator=g) * torch.exp(torch.randn(rows // k, 1, device="cuda", generator=g))
    room = torch.full((rows + 1, N + 3), 7.0, device="cuda")
    y = lcd.mx_linear_grouped(codes, scales, x, plan, y=room[:rows, :N], status_word=word)
    w = torch.stack([decoded(codes[e], scales[e], K) for e in range(G)])
    want, size = product(decoded(*lcd.mx_quantize(x), K), w, group, k)
    # an instruction of 64 columns keeps 24 bits of its largest term and the sum so far; a cluster adds up to eight sums
    bound = (-(-K // 32) + 8) * 2.0 ** -22 * size + want.abs() * 2.0 ** -24
    assert ((y.double() - want).abs() <= bound).all()
    assert (y[none] == 0).all() and (room[rows] == 7).all() and (room[:, N:] == 7).all()
    # whole numbers (halves) are exact in fp32, and rounded once to every type of y
    codes, scales = experts(K + 1, G, N, K, True)
    x = torch.randint(-2, 3, (rows // k, K), device="cuda", generator=g).float()
    x[:, ::32] = 2.0
    w = torch.stack([decoded(codes[e], scales[e], K) for e in range(G)])
    want, size = product(x.double(), w, group, k)
    assert size.max() < 2 ** 22
    for type in TYPES.values():
        y = lcd.mx_linear_grouped(codes, scales, x.to(type), plan, dtype=type, status_word=word)
        assert torch.equal(y, want.float().to(type))
    assert word.item() == 0


@pytest.mark.parametrize("form,rows,G,N,K", [c for c in CASES if c[0] in [(16, 8, False), (64, 4, False), (128, 4, False), (192, 1, True), (256, 4, False)]])
def test_forms_side_by_side(form, rows, G, N, K):
    # several streams and a replayed graph: the same bits every time
    codes, scales = experts(K, G, N, K, False)
    x = torch.randn(rows, K, device="cuda").bfloat16()
    group = ragged(rows, G, form[0], 3)
    plan = lcd.group_rows(group, G)
    want = lcd.mx_linear_grouped(codes, scales, x, plan)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = [lcd.mx_linear_grouped(codes, scales, x, plan, stream=s) for s in streams for _ in range(2)]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        y = lcd.mx_linear_grouped(codes, scales, x, lcd.group_rows(group, G))
    for _ in range(2):
        y.zero_()
        graph.replay()
        assert torch.equal(y, want)
    assert all(torch.equal(v, want) for v in got)

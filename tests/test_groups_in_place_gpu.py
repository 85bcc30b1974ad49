"""base that is y (dx): rows without an adapter are left as they are, to the bit, whatever they hold and however many rows there are."""
import pytest
import torch

import paper_2506_12038_b200 as lcd
from test_groups_gpu import TYPES

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("type", ["bf16", "fp16"])
@pytest.mark.parametrize("M", [9, 700, 1500])
@pytest.mark.parametrize("N,pitch", [(136, 136), (131, 133)])
@pytest.mark.parametrize("absent", ["some", "most", "all"])
def test_rows_without_an_adapter_keep_their_bits(type, M, N, pitch, absent):
    g = torch.Generator(device="cuda").manual_seed(M + N)
    K, r, G = 64, 16, 3
    group = torch.randint(0, G, (M,), generator=g, device="cuda")
    group[torch.rand(M, generator=g, device="cuda") < {"some": 0.25, "most": 0.95, "all": 2.0}[absent]] = -1
    none = group < 0
    x, a = torch.randn(M, K, generator=g, device="cuda").to(TYPES[type]), torch.randn(G, r, K, generator=g, device="cuda").to(TYPES[type])
    b = torch.randn(G, N, r, generator=g, device="cuda").to(TYPES[type])
    rows = lcd.group_rows(group, G)
    bits = torch.randint(-2 ** 15, 2 ** 15, (M, pitch), generator=g, device="cuda", dtype=torch.int16)        # NaN of every kind among them
    base = torch.randn(M, N, generator=g, device="cuda").to(TYPES[type])
    room = bits.clone().view(TYPES[type])
    room[~none, :N] = base[~none]
    want = lcd.adapters(x, a, b, rows, base)
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    y = lcd.adapters(x, a, b, rows, room[:, :N], y=room[:, :N], status_word=word)
    assert y.data_ptr() == room.data_ptr() and torch.equal(y[~none], want[~none])
    assert torch.equal(room.view(torch.int16)[none], bits[none]) and torch.equal(room.view(torch.int16)[:, N:], bits[:, N:])
    # the same of dx: b in a's place
    dy = torch.randn(M, K, generator=g, device="cuda").to(TYPES[type])
    at, bt = b.transpose(1, 2).contiguous(), a.transpose(1, 2).contiguous()
    want = lcd.adapters_grad(dy, None, at, bt, None, rows, base, want_weights=False)[0]
    room = bits.clone().view(TYPES[type])
    room[~none, :N] = base[~none]
    dx = lcd.adapters_grad(dy, None, at, bt, None, rows, room[:, :N], dx=room[:, :N], want_weights=False, status_word=word)[0]
    assert torch.equal(dx[~none], want[~none]) and torch.equal(room.view(torch.int16)[none], bits[none]) and word.item() == 0

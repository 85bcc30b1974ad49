"""Plans that lcd_group_rows did not write: results are unspecified, but nothing is read or written outside the buffers, and the calls
behind are as ever."""
import pytest
import torch

import paper_2506_12038_b200 as lcd
from test_groups_gpu import random_experts

pytestmark = pytest.mark.gpu


def surrounded(bytes, fill):
    """A workspace in the middle of a larger allocation, filled, and the whole of it."""
    room = torch.full((bytes + 2 * 4096,), fill, dtype=torch.uint8, device="cuda")
    return room[4096:4096 + bytes], room


@pytest.mark.parametrize("fill", [0x7f, 0x10, 0x00, 0xff])
@pytest.mark.parametrize("T,k,K", [(1100, 4, 1001), (2100, 2, 2048), (40, 3, 256)])
def test_rows_twice_and_rows_that_are_none(T, k, K, fill):
    # of several choices a token: quantised once from 2^22 values on, its places noted in the workspace; what the workspace held is no place
    G, N = 6, 200
    codes, scales, _ = random_experts(T, G, N, K)
    x = torch.randn(T, K, device="cuda")
    count = T * k
    rows = lcd.group_rows(torch.randint(-1, G, (count,), device="cuda"), G)
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    want = lcd.mx_linear_grouped(codes, scales, x, rows, status_word=word)
    order = rows.order.clone()
    order[::2] = order[1::2][:order[::2].numel()] if count % 2 == 0 else order[::2]
    twice = rows._replace(order=order)
    none = order.clone()
    none[::3], none[1::7], none[2::11] = -1, count, 2 ** 31 - 1
    for plan in (twice, rows._replace(order=none)):
        space, room = surrounded(lcd.mx_linear_grouped_workspace_bytes(count, K), fill)
        y_room = torch.full((count + 2, N + 8), 7.0, device="cuda")
        lcd.mx_linear_grouped(codes, scales, x, plan, y=y_room[1:-1, :N], workspace=space, status_word=word)
        torch.cuda.synchronize()
        assert (room[:4096] == fill).all() and (room[-4096:] == fill).all()
        assert (y_room[0] == 7).all() and (y_room[-1] == 7).all() and (y_room[:, N:] == 7).all()
        assert torch.equal(lcd.mx_linear_grouped(codes, scales, x, rows, workspace=space, status_word=word), want)
    assert word.item() == 0


@pytest.mark.parametrize("M,G", [(20, 5), (700, 5), (1500, 1024)])
@pytest.mark.parametrize("kind", ["descending", "to and fro", "beyond", "negative", "none"])
def test_offsets_that_do_not_ascend(M, G, kind):
    # only rows that the batch has are read and written, and the calls end
    offsets = {"descending": torch.arange(G, -1, -1) * M // G, "to and fro": torch.arange(G + 1) % 2 * M, "beyond": torch.full((G + 1,), 2 ** 31 - 1),
               "negative": torch.full((G + 1,), -2 ** 31), "none": torch.zeros(G + 1, dtype=torch.int64)}[kind].int().cuda()
    K, N, r = 64, 136, 16
    x, dy = torch.randn(M, K, device="cuda").bfloat16(), torch.randn(M, N, device="cuda").bfloat16()
    a, b = torch.randn(G, r, K, device="cuda").bfloat16(), torch.randn(G, N, r, device="cuda").bfloat16()
    codes, scales, _ = random_experts(M, 5, 40, K)
    rows = lcd.group_rows(torch.randint(-1, G, (M,), device="cuda"), G)
    few = lcd.group_rows(torch.randint(-1, 5, (M,), device="cuda"), 5)
    foreign = rows._replace(offsets=offsets)
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    want = lcd.adapters(x, a, b, rows, dy, status_word=word)

    def room(m, n, type=torch.bfloat16):
        whole = torch.full((m + 2, n + 8), 7.0, dtype=type, device="cuda")
        return whole, whole[1:m + 1, :n]

    space, around = surrounded(lcd.adapters_workspace_bytes(M, r), 0x7f)
    (ys, y), (ts, t), (ds, dx) = room(M, N), room(M, r, torch.float32), room(M, K)
    da, db = torch.full((G + 2, r, K), 7.0, device="cuda"), torch.full((G + 2, N, r), 7.0, device="cuda")
    lcd.adapters(x, a, b, foreign, dy, y=y, t=t, workspace=space, status_word=word)
    lcd.adapters_grad(dy, x, a, b, t, foreign, dx=dx, da=da[1:G + 1], db=db[1:G + 1], workspace=space, status_word=word)
    es, e = room(M, 40, torch.float32)
    lcd.mx_linear_grouped(codes, scales, x, few._replace(offsets=offsets[:6].contiguous()), y=e, status_word=word)
    torch.cuda.synchronize()
    assert (around[:4096] == 0x7f).all() and (around[-4096:] == 0x7f).all()
    for whole, part in ((ys, y), (ts, t), (ds, dx), (es, e)):
        m, n = part.shape
        assert (whole[0] == 7).all() and (whole[m + 1:] == 7).all() and (whole[:, n:] == 7).all()
    for whole in (da, db):
        assert (whole[0] == 7).all() and (whole[G + 1] == 7).all()
    assert torch.equal(lcd.adapters(x, a, b, rows, dy, workspace=space, status_word=word), want) and word.item() == 0

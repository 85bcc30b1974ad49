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

"""Products of experts at the largest sizes that the calls take."""
import pytest
import torch

import paper_2506_12038_b200 as lcd

pytestmark = pytest.mark.gpu


def test_most_weight_rows():
    N = 1 << 30
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("needs 30 GB")
    # codes 15 (-6) and 7 (6) in turn; their bytes serve as scales too: 127 stands for 1
    codes = torch.full((1, N, 16), 127, dtype=torch.uint8, device="cuda")
    x = torch.zeros(2, 32, device="cuda")
    x[:, 0], x[:, 3] = 2.0, 0.5
    rows = lcd.group_rows(torch.tensor([0, -1], device="cuda"), 1)
    y = torch.full((2, N), 5.0, dtype=torch.bfloat16, device="cuda")
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    lcd.mx_linear_grouped(codes, codes[:, :, :1], x, rows, y=y, status_word=word)
    assert word.item() == 0
    for part in y[0].split(1 << 28):
        assert (part == -9).all()
    for part in y[1].split(1 << 28):
        assert (part == 0).all()

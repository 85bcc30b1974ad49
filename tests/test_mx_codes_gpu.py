"""Codes and what they stand for, all of them, in every type and on every path to memory."""
import numpy as np
import pytest
import torch

import paper_2506_12038_b200 as lcd
from oracle import train_oracle as O
from test_mx_gpu import TYPES, host

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("type", sorted(TYPES))
@pytest.mark.parametrize("M,K,pitch", [(3, 4096, 0), (3, 4095, 1), (30000, 64, 0), (30000, 61, 0), (2000, 1000, 3)])
def test_every_code_under_every_scale(type, M, K, pitch):
    # few and many rows, on 16 bytes and off them; the values of 2^128 and beyond (bytes 253 and 254) are infinite
    rng = np.random.default_rng(K)
    blocks = -(-K // 32)
    codes = rng.integers(0, 16, size=(M, blocks * 32), dtype=np.uint8)
    scales = rng.integers(0, 256, size=(M, blocks), dtype=np.uint8)
    scales[:, 0] = np.arange(M) % 256
    packed = torch.from_numpy(O.mx_codes(codes)).cuda()
    room = torch.zeros(M, -(-blocks // 16) * 16, dtype=torch.uint8, device="cuda")
    room[:, :blocks] = torch.from_numpy(scales)
    out = torch.full((M, K + pitch), 7.0, dtype=TYPES[type], device="cuda")
    got = lcd.mx_dequantize(packed, room[:, :blocks], K, out=out[:, :K])
    with np.errstate(over="ignore"):
        want = torch.from_numpy(O.mx_values(packed.cpu().numpy(), scales, K).astype(np.float32)).to(TYPES[type]).cuda()
    assert torch.equal(got.isnan(), want.isnan()) and torch.equal(torch.nan_to_num(got, nan=9.0), torch.nan_to_num(want, nan=9.0))
    assert torch.equal(got.signbit() | got.isnan(), want.signbit() | want.isnan()) and (out[:, K:] == 7).all()


@pytest.mark.parametrize("type", ["fp16", "bf16"])
@pytest.mark.parametrize("K", [2048, 2047])
def test_every_16_bit_number_under_every_scale_of_its_block(type, K):
    # every number of the type, in blocks whose largest magnitude is 1, 2, 4 ... 64 times as large as it or more
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(TYPES[type]).cuda()
    for times in (1.0, 3.0, 8.0, 64.0):
        x = bits.repeat_interleave(32).view(65536, 32)
        place = torch.arange(65536, device="cuda") % 32
        x[torch.arange(65536, device="cuda"), place] = (bits.float() * times).to(x.dtype)
        x = x.reshape(-1, 2048)[:, :K]
        codes, scales = lcd.mx_quantize(x)
        ref, bytes_ = O.mx_quantize(host(x))
        assert np.array_equal(scales.cpu().numpy(), bytes_) and np.array_equal(codes.cpu().numpy(), O.mx_codes(ref))

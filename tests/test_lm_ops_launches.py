"""Matrices of more than 2^32 elements, or pieces of eight of them, a replica: more than a launch has threads along one axis."""
import pytest
import torch

import ops_reference as R
import paper_2604_24708_amd as H

pytestmark = pytest.mark.gpu
ROWS = 1 << 21            # the most a call takes


def test_zeros_of_a_gradient_without_rows():
    width = 2049
    assert ROWS * width > 1 << 32
    dw = torch.full((1, ROWS, width), 7.0, dtype=torch.bfloat16, device=R.DEV)
    h, labels = torch.empty(1, 0, width, dtype=torch.bfloat16, device=R.DEV), torch.empty(1, 0, dtype=torch.int32, device=R.DEV)
    mean = torch.ones(1, device=R.DEV)
    H.hdet_vocab_loss(h, dw, labels, torch.empty(1, 0, device=R.DEV), mean, dw=dw)             # (W is read by no row)
    assert float(mean) == 0
    for part in dw[0].split(1 << 18):
        assert not bool(part.any())
    torch.cuda.empty_cache()


def test_rows_read_back():
    width = 16392
    assert ROWS * (width // 8) > 1 << 32
    codes, scale = H.hdet_codes_empty(1, ROWS, width), torch.empty(1, ROWS, device=R.DEV)
    row = torch.arange(ROWS, device=R.DEV)
    scale[0] = torch.exp2((row % 7).float())
    codes.copy_((row % 251 - 125).to(torch.int8)[None, :, None].expand(1, ROWS, width))
    values = torch.full((1, ROWS, width), float("nan"), dtype=torch.bfloat16, device=R.DEV)
    H.hdet_restore_rows(codes, scale, values)
    want = ((row % 251 - 125).float() * scale[0]).to(torch.bfloat16)[:, None]
    for part, w in zip(values[0].split(1 << 17), want.split(1 << 17)):
        assert torch.all(part == w)
    del codes, values
    torch.cuda.empty_cache()

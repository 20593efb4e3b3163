"""Rotation tables of bases that 32 bits do not hold."""
import numpy as np
import pytest
import torch

import paged_model as M
from paper_2406_17808_amd import paged
from test_gpu_paged import f64, i32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
STRETCHED = 10000.0 * 8.0 ** (128 / 126)      # a base as context extension makes it: 82684.62...


@pytest.mark.parametrize("base", [STRETCHED, 10000.0, 0.3, 1e-3, 123456789.0])
@pytest.mark.parametrize("d", [2, 64, 128])
def test_table_entries(base, d):
    """Both tables against cosines and sines of the host: an angle p * theta is off by the roundings of the quotient, the power (one step of 2^-52 each, the
    former times log(base)) and the product."""
    n = 100000
    rope = paged.RopeTable(n, d, base, DEV)
    got = rope.table.cpu().numpy().view(np.float64).reshape(-1, d // 2, 2)
    p = np.concatenate([np.arange(256), 256 * np.arange(-(-n // 256))]).astype(np.float64)
    angle = p[:, None] * base ** (-np.arange(d // 2) / (d // 2))
    tol = np.abs(angle) * 2.0 ** -52 * (4 + abs(np.log(base))) + 2.0 ** -51
    assert (np.abs(got[..., 0] - np.cos(angle)) <= tol).all() and (np.abs(got[..., 1] - np.sin(angle)) <= tol).all()


def test_rotation_by_a_base_that_32_bits_do_not_hold():
    gen = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn((5, 2, 128), generator=gen, device=DEV)
    pos = i32([1, 1000, 65537, 131071, 99991])
    got, _ = paged.qk_norm_rope(x, norm=False, positions=pos, rope=paged.RopeTable(1 << 17, 128, STRETCHED, DEV))
    y = f64(x)
    size = np.concatenate([np.abs(y[..., :64]) + np.abs(y[..., 64:])] * 2, -1)
    want = M.rotate(y, pos.cpu().numpy(), STRETCHED)
    # cosine and sine, two products and their sum in 32 bits, the rounding of the result
    assert (np.abs(f64(got) - want) <= 2.0 ** -24 * np.abs(want) + 4 * 2.0 ** -24 * size).all()

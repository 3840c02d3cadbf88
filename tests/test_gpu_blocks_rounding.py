"""fp32 numbers whose quotient by the block's largest lies next to a border between two codes, on the GPU: the codes are those of a multiplication and a division in
fp32, rounded to nearest even."""
import numpy as np
import pytest
import torch

from oracle import beside_oracle as O
from paper_2603_01875_amd import kdloss as K
from tests.test_gpu_blocks import values

pytestmark = pytest.mark.gpu


def quotient(x, m):
    return np.float32(448) * x / m                                        # (numpy's fp32: each operation rounded)


def near_borders(rng, m, n):
    """n numbers of magnitude at most m whose quotient 448 x / m is a border between two codes, or as near to one as fp32 has them."""
    unit = rng.integers(16, 32, n) * 2.0 ** rng.integers(-14, 5, n)        # (all borders are odd multiples of a 32nd of a power of two, or of 2^-10)
    x = (np.longdouble(m) * unit / 448).astype(np.float32)
    x = (x.view(np.int32) + rng.integers(-1, 2, n).astype(np.int32)).view(np.float32)
    return np.where(np.abs(x) <= m, x, np.float32(m)) * rng.choice(np.array([-1, 1], np.float32), n)


def rows(seed, R, blocks):
    """[R, 128 blocks] with a largest element of its own in each block of 128."""
    rng = np.random.default_rng(seed)
    x = np.empty((R, blocks, 128), np.float32)
    for r in range(R):
        for b in range(blocks):
            m = np.float32(np.ldexp(rng.integers(1 << 23, 1 << 24), int(rng.integers(-60, 40))))
            x[r, b] = near_borders(rng, m, 128)
            x[r, b, rng.integers(0, 128)] = m
    return x.reshape(R, -1)


def check(got, x, m, some=True):
    want = O.e4m3(quotient(x, m))
    assert (got == want).all(), (np.argwhere(got != want)[:3], (got != want).sum())
    # (a quotient that is rounded once from 64 bits gives other codes: these numbers are near enough to a border)
    assert not some or (O.e4m3((x.astype(np.float64) * 448 / m).astype(np.float32)) != want).sum() > 0.002 * x.size


def largest(x):
    return np.repeat(np.abs(x).reshape(x.shape[0], -1, 128).max(2), 128, 1)


def test_blocks_of_rows():
    x = rows(1, 384, 4)
    m = largest(x)
    check(values(K.quantize_e4m3_blocks(torch.from_numpy(x).cuda()), 512), x, m)
    q, qt = K.quantize_e4m3_blocks(torch.from_numpy(x).cuda(), both=True)
    check(values(q, 512), x, m)
    other = K.quantize_e4m3_blocks(torch.from_numpy(x.T.copy()).cuda(), transpose=True)
    assert torch.equal(other.codes, q.codes) and torch.equal(other.scales, q.scales)


def test_blocks_of_tiles():
    rng = np.random.default_rng(2)
    for i in range(40):
        m = np.float32(np.ldexp(rng.integers(1 << 23, 1 << 24), int(rng.integers(-60, 40))))
        x = near_borders(rng, m, 128 * 128).reshape(128, 128)
        x[i, 5] = -m
        q, qt = K.quantize_e4m3_blocks(torch.from_numpy(x).cuda(), K.BLOCK_TILE, both=True)
        check(values(q, 128), x, m, False)
        assert torch.equal(qt.codes, q.codes.t())


@pytest.mark.parametrize("R", [1, 4])
def test_few_rows_of_a_linear_layer(R):
    """By a matrix of 448 on the diagonal, whose scale is 1: a result is 448 times the code times the scale."""
    x = rows(3, 12 * R, 1)
    w = K.quantize_e4m3_blocks(448 * torch.eye(128, device="cuda"), K.BLOCK_TILE)
    m = largest(x)
    scale = (m / np.float32(448)).astype(np.float64)
    want = (448 * O.e4m3(quotient(x, m)) * scale).astype(np.float32)
    for i in range(0, x.shape[0], R):
        y = K.kd_linear_e4m3(torch.from_numpy(x[i:i + R]).cuda(), w, out_dtype=K.F32)
        assert (y.cpu().numpy() == want[i:i + R]).all()


def test_bf16_codes_do_not_depend_on_the_kernel():
    """Few rows are quantised inside the product, more in front of it: the same codes."""
    g = torch.Generator().manual_seed(5)
    x = torch.randn(32, 128, generator=g).to(torch.bfloat16).cuda()
    w = K.quantize_e4m3_blocks(448 * torch.eye(128, device="cuda"), K.BLOCK_TILE)
    q = K.quantize_e4m3_blocks(x)
    assert torch.equal(K.kd_linear_e4m3(x, w, out_dtype=K.F32), K.kd_matmul_e4m3(q, w, out_dtype=K.F32))

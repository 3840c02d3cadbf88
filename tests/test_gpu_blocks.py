"""e4m3 in blocks of 128 on the GPU: the quantiser against the definition, the product against 64 bits on the same codes, the linear
layer with its gradients."""
import numpy as np
import pytest
import torch

from oracle import beside_oracle as O
from paper_2603_01875_amd import autograd as A
from paper_2603_01875_amd import kdloss as K

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}


def np64(t):
    return t.detach().cpu().double().numpy()


def matrix(seed, R, C, dtype, spread=3.0):
    """Entries of many magnitudes, some blocks empty."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((R, C)) * np.exp(rng.standard_normal((R, 1)) * spread)
    x[:, C // 2:C // 2 + 128] *= (rng.random((R, 1)) < 0.7)
    return torch.from_numpy(x.astype(np.float32)).to(DT[dtype])


def values(q, cols):
    """What the codes stand for, without the scales."""
    return np64(q.codes.view(torch.float8_e4m3fn).float())[:, :cols]


def check_codes(q, x, tile):
    """x: what was quantised, fp64."""
    R, C = x.shape
    codes, scales = O.blocks(x, tile)
    assert (np64(q.scales) == scales).all()
    got = values(q, C)
    # the quotient is rounded to fp32 (and 7 x in front of it, for fp32 x) before it is rounded to e4m3
    m = np.maximum(O.expand(scales, R, C, tile) * 448.0, O.LEAST)
    exact = x * 448.0 / m
    unit = np.ldexp(1.0, np.frexp(np.maximum(np.abs(exact), 2.0 ** -6))[1] - 4)
    assert (np.abs(got - exact) <= unit / 2 + np.abs(exact) * 2.0 ** -22).all()
    if np.array_equal(x, x.astype(np.float32).view(np.uint32).__and__(0xffff0000).view(np.float32)):      # bf16: nothing but the last rounding
        assert (got == codes).all()
    assert (q.codes[:, C:] == 0).all()


@pytest.mark.parametrize("R,C", [(1, 1), (1, 128), (3, 16), (2, 129), (128, 128), (129, 255), (130, 1000), (257, 130), (500, 24)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("block", [K.BLOCK_ROW, K.BLOCK_TILE])
def test_quantiser(R, C, dtype, block):
    x = matrix(R * 1000 + C, R, C, dtype)
    q, qt = K.quantize_e4m3_blocks(x.cuda(), block, both=True)
    tile = block == K.BLOCK_TILE
    check_codes(q, np64(x), tile)
    check_codes(qt, np64(x).T.copy(), tile)
    one, other = K.quantize_e4m3_blocks(x.cuda(), block), K.quantize_e4m3_blocks(x.cuda(), block, transpose=True)
    assert torch.equal(one.codes, q.codes) and torch.equal(other.codes, qt.codes)
    assert torch.equal(one.scales, q.scales) and torch.equal(other.scales, qt.scales)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_quantiser_rows_of_a_wider_array_at_an_odd_offset(dtype):
    wide = matrix(5, 70, 403, dtype).cuda()
    x = wide[1:, 3:304]
    check_codes(K.quantize_e4m3_blocks(x), np64(x), False)


def test_quantiser_extremes():
    x = torch.zeros(6, 256)
    x[0, 0], x[0, 1] = 3.4e38, 1e38
    x[1, 5] = 1e-45                                     # far below what a scale resolves: the code is 0
    x[2, 3], x[2, 200] = float("inf"), 1.0
    x[3, 130] = float("nan")
    x[4, 0], x[4, 1] = -2.0 ** -126, 2.0 ** -127
    q = K.quantize_e4m3_blocks(x.cuda())
    s = q.scales.cpu()
    assert torch.isnan(s[2, 0]) and torch.isfinite(s[2, 1]) and torch.isnan(s[3, 1]) and torch.isfinite(s[3, 0])
    keep = [0, 1, 4, 5]
    check_codes(K.E4m3Blocks(q.codes[keep], q.scales[keep], K.BLOCK_ROW), np64(x[keep]), False)
    t = K.quantize_e4m3_blocks(x.cuda(), K.BLOCK_TILE)
    assert torch.isnan(t.scales).all()
    w = K.quantize_e4m3_blocks(torch.ones(16, 256, device="cuda"), K.BLOCK_TILE)
    y = K.kd_matmul_e4m3(q, w, out_dtype=K.F32).cpu()
    assert torch.isnan(y[2]).all() and torch.isnan(y[3]).all() and torch.isfinite(y[[1, 4, 5]]).all() and (y[5] == 0).all()
    assert torch.isinf(y[0]).all()                      # 3.4e38 + 1e38 is beyond fp32


def reference(a, b, K_, b_tile):
    """(product, sum of magnitudes) of two E4m3Blocks in fp64."""
    M, N = a.codes.shape[0], b.codes.shape[0]
    va = values(a, K_) * O.expand(np64(a.scales), M, K_, False)
    vb = values(b, K_) * O.expand(np64(b.scales), N, K_, b_tile)
    return va @ vb.T, np.abs(va) @ np.abs(vb).T


def check_product(y, ref, size, K_, dtype, before=None):
    """A block's 128 products are added in fp32, the scale's two roundings and the sum over blocks on top: (128 + blocks + 4)
    half steps of fp32 of the sum of magnitudes, twice that for a matrix pipe that cuts off instead of rounding.  For a bf16 result the e4m3 pipe
    cuts seven of eight products at 2^-13 of the largest of them.  The result is rounded once."""
    if before is not None:
        ref, size = ref + before, size + np.abs(before)
    err = ((128 + K_ / 128 + 4) * 2.0 ** -23 + (7 * 2.0 ** -13 if dtype == "bf16" else 0)) * size
    off = np.abs(np64(y) - ref) - err - HALF[dtype] * (np.abs(ref) + err) - 1e-40
    assert (off <= 0).all(), (off.max(), np.unravel_index(off.argmax(), off.shape))


SIZES = [(1, 1, 1), (1, 16, 128), (1, 300, 256), (3, 17, 100), (8, 128, 1024), (16, 130, 272), (17, 64, 640), (33, 257, 384), (64, 100, 2000),
         (100, 1000, 128), (128, 256, 512), (129, 255, 144), (200, 520, 1040), (257, 515, 333), (300, 31, 4096), (500, 777, 1000),
         (513, 1024, 896), (1, 4096, 4096), (5, 2048, 8192),
         (13, 5000, 8192), (16, 16, 16), (17, 40, 30_000), (32, 1000, 3000), (2, 33_000, 256), (1, 15, 100_000), (31, 300, 4080)]


@pytest.mark.parametrize("M,N,K_", SIZES)
@pytest.mark.parametrize("tile", [True, False])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_product(M, N, K_, tile, out):
    a = K.quantize_e4m3_blocks(matrix(M + K_, M, K_, "f32", 1.0).cuda())
    b = K.quantize_e4m3_blocks(matrix(N + K_ + 1, N, K_, "f32", 1.0).cuda(), K.BLOCK_TILE if tile else K.BLOCK_ROW)
    ref, size = reference(a, b, K_, tile)
    y = K.kd_matmul_e4m3(a, b, out_dtype=K.F32 if out == "f32" else K.BF16)
    assert y.dtype == DT[out]
    check_product(y, ref, size, K_, out)
    assert torch.equal(y, K.kd_matmul_e4m3(a, b, out_dtype=K.F32 if out == "f32" else K.BF16))
    into = matrix(7, M, N, out).cuda()
    before = np64(into)
    K.kd_matmul_e4m3(a, b, out=into, accumulate=True)
    check_product(into, ref, size, K_, out, before)


@pytest.mark.parametrize("M,N,K_", [(40, 217, 2100), (33, 1, 2048), (64, 130, 4200), (70, 131, 16_400), (500, 1027, 2176), (130, 64, 40_000),
                                    (3000, 3001, 200)])
@pytest.mark.parametrize("tile", [True, False])
@pytest.mark.parametrize("out", ["bf16", "f32"])
def test_product_of_a_long_axis_in_parts(M, N, K_, tile, out):
    """Parts that are shorter than the others, or empty (16,400: 129 blocks are 15 parts of nine); the last size has none, in 128 x 128 tiles."""
    test_product(M, N, K_, tile, out)


@pytest.mark.parametrize("tile", [True, False])
@pytest.mark.parametrize("out", ["bf16", "f32"])
@pytest.mark.parametrize("M,N,K_", [(4096, 5000, 128), (4000, 4800, 100), (2300, 9000, 272), (20_000, 300, 130)])
def test_more_tiles_than_workgroups(M, N, K_, tile, out):
    """Workgroups that take several tiles, each with the loads of the next under way: a row of tiles with scales of NaN touches nothing
    but itself."""
    a = K.quantize_e4m3_blocks(matrix(M, M, K_, "f32", 1.0).cuda())
    b = K.quantize_e4m3_blocks(matrix(N, N, K_, "f32", 1.0).cuda(), K.BLOCK_TILE if tile else K.BLOCK_ROW)
    a.scales[300:301] = float("nan")
    b.scales[1, -1] = float("nan")
    y = K.kd_matmul_e4m3(a, b, out_dtype=K.F32 if out == "f32" else K.BF16)
    bad = torch.zeros(M, N, dtype=torch.bool)
    bad[300] = True
    bad[:, 128:256 if tile else 129][:, :] = True
    if not tile:
        bad[:, 128:] = False
        bad[:, 1] = True
        bad[300] = True
    assert torch.equal(torch.isnan(y).cpu(), bad)
    rows = [0, 1, 255, 256, 299, M // 2, M - 1]
    some = K.E4m3Blocks(a.codes[rows], a.scales[rows], K.BLOCK_ROW)
    b.scales[1, -1] = 0.0
    ref, size = reference(some, b, K_, tile)
    good = ~bad[rows].numpy()
    check_product(torch.where(torch.from_numpy(good), y[rows].cpu(), 0.0), np.where(good, ref, 0), np.where(good, size, 0), K_, out)


@pytest.mark.parametrize("M,N,K_,dtype,out", [(1, 1000, 512, "bf16", "f32"), (2, 48, 1000, "f32", "f32"), (9, 515, 200, "bf16", "bf16"),
                                              (16, 1024, 1024, "bf16", "f32"), (31, 130, 77, "f32", "bf16"), (65, 300, 640, "bf16", "f32"),
                                              (300, 200, 250, "f32", "f32"), (1, 256, 8192, "f32", "f32"), (8, 151936, 64, "bf16", "bf16")])
def test_linear_is_quantiser_and_product(M, N, K_, dtype, out):
    x = matrix(M + N, M, K_, dtype, 1.0).cuda()
    w = K.quantize_e4m3_blocks(matrix(N + 1, N, K_, "bf16", 0.5).cuda(), K.BLOCK_TILE)
    a = K.quantize_e4m3_blocks(x)
    ref, size = reference(a, w, K_, True)
    y = K.kd_linear_e4m3(x, w, out_dtype=K.F32 if out == "f32" else K.BF16)
    check_product(y, ref, size, K_, out)
    into = torch.full((M, N), 2.0, device="cuda", dtype=DT[out])
    K.kd_linear_e4m3(x, w, out=into, accumulate=True)
    check_product(into, ref, size, K_, out, np.full((M, N), 2.0))


def test_linear_of_an_input_at_an_odd_offset():
    flat = torch.randn(5 * 333 + 1, device="cuda").to(torch.bfloat16)
    x = flat[1:].view(5, 333)
    w = K.quantize_e4m3_blocks(matrix(1, 50, 333, "bf16", 0.5).cuda(), K.BLOCK_TILE)
    assert torch.equal(K.kd_linear_e4m3(x, w), K.kd_linear_e4m3(x.clone(), w))


@pytest.mark.parametrize("T,H,V", [(1, 128, 64), (7, 200, 130), (130, 256, 515), (300, 1000, 77)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_layer_and_its_gradients(T, H, V, dtype):
    x, W, gy = (matrix(i + T, *s, dtype, 0.5).cuda() for i, s in enumerate(((T, H), (V, H), (T, V))))
    x.requires_grad_(), W.requires_grad_()
    y = A.linear_e4m3(x, W)
    gx, gW = torch.autograd.grad(y, (x, W), gy)
    assert y.dtype == gx.dtype == gW.dtype == DT[dtype]
    xd, Wd = x.detach(), W.detach()
    q, w, g, gt, xt = (K.quantize_e4m3_blocks(xd), K.quantize_e4m3_blocks(Wd, K.BLOCK_TILE), K.quantize_e4m3_blocks(gy),
                       K.quantize_e4m3_blocks(gy, transpose=True), K.quantize_e4m3_blocks(xd, transpose=True))
    wt = K.quantize_e4m3_blocks(Wd, K.BLOCK_TILE, transpose=True)
    check_product(y, *reference(q, w, H, True), H, dtype)
    check_product(gx, *reference(g, wt, V, True), V, dtype)
    check_product(gW, *reference(gt, xt, T, False), T, dtype)
    # and all of it against the products of the numbers themselves: each factor is off by at most 2^-4 of itself, or, below the normal
    # range, by half a step of 2^-9 where the block's largest is 448: 2^-18.8 of that
    for got, a, b in ((y, np64(xd), np64(Wd)), (gx, np64(gy), np64(Wd).T), (gW, np64(gy).T, np64(xd).T)):
        da, db = (np.abs(m) * 2.0 ** -4 + np.abs(m).max() * 2.0 ** -18 for m in (a, b))
        bound = da @ np.abs(b).T + np.abs(a) @ db.T + da @ db.T
        ref = a @ b.T
        assert (np.abs(np64(got) - ref) <= 1.01 * bound + HALF[dtype] * (np.abs(ref) + bound) + 1e-30).all()
    # only what is asked for
    gx2, = torch.autograd.grad(A.linear_e4m3(x, Wd), (x,), gy)
    gW2, = torch.autograd.grad(A.linear_e4m3(xd, W), (W,), gy)
    assert torch.equal(gx2, gx) and torch.equal(gW2, gW)


def test_gradient_against_differences():
    """The layer's value changes as its gradient says, on numbers that e4m3 holds exactly (so that the layer is linear in them)."""
    rng = np.random.default_rng(3)
    steps = np.array([-2.0, -1.0, 1.0, 2.0])
    x, W, gy = (torch.from_numpy(rng.choice(steps, s)).float().cuda() for s in ((5, 128), (128, 128), (5, 128)))
    for t in (x, W, gy):
        t[:, 0] = 448.0                                 # every block's scale is 1, whichever way it is cut ...
        t[0, :] = 448.0
    x.requires_grad_(), W.requires_grad_()
    gx, gW = torch.autograd.grad(A.linear_e4m3(x, W), (x, W), gy)

    def value(x_, W_):
        return float((A.linear_e4m3(x_, W_).double() * gy.double()).sum())
    for i, j in ((1, 5), (4, 127), (2, 64)):
        d = torch.zeros_like(x)
        d[i, j] = 1.0
        with torch.no_grad():
            diff = (value(torch.where(d > 0, 4.0 * torch.ones_like(x), x), W) - value(torch.where(d > 0, 2.0 * torch.ones_like(x), x), W)) / 2
        assert abs(diff - float(gx[i, j])) <= 1e-5 * (abs(diff) + 448 * 448)
    for i, j in ((1, 5), (100, 127)):
        d = torch.zeros_like(W)
        d[i, j] = 1.0
        with torch.no_grad():
            diff = (value(x, torch.where(d > 0, 4.0 * torch.ones_like(W), W)) - value(x, torch.where(d > 0, 2.0 * torch.ones_like(W), W))) / 2
        assert abs(diff - float(gW[i, j])) <= 1e-5 * (abs(diff) + 448 * 448)

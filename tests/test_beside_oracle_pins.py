"""Pins of the fp64 reference of what stands beside the losses, by hand-made cases and by another way of computing the same."""
import numpy as np
import torch

from oracle import beside_oracle as O
from oracle import e4m3 as E


def test_e4m3_is_the_nearest_of_the_table():
    rng = np.random.default_rng(1)
    tab = E.e4m3_values()
    x = np.concatenate([rng.standard_normal(20000) * 60, rng.standard_normal(20000) * 0.01, tab[np.isfinite(tab)], [1.0625, 1.1875, 464., 1e9]])
    mine = O.e4m3(x)
    codes = E.quantize_e4m3(x, 1.0)
    near32 = x.astype(np.float32) == x
    assert (mine[near32] == tab[codes][near32]).all()
    pos = tab[:127]
    best = np.abs(np.abs(x)[:, None] - pos[None]).min(1)
    assert np.allclose(np.abs(np.abs(x) - np.abs(mine)), best, rtol=0, atol=1e-12)


def test_blocks():
    x = np.zeros((130, 300))
    x[0, 0], x[0, 1], x[1, 130], x[129, 299] = 448.0, 17.0, -2.0, 1e-3
    codes, scales = O.blocks(x, False)
    assert scales.shape == (130, 3) and scales[0, 0] == 1.0 and codes[0, 1] == 16.0 and codes[1, 130] == -448.0
    assert scales[5, 0] == 2.0 ** -126                      # an empty block
    codes, scales = O.blocks(x, True)
    assert scales.shape == (2, 3) and codes[129, 299] == 448.0 and scales[1, 2] == np.float32(1e-3 / 448)
    assert (O.expand(scales, 130, 300, True)[:128, 128:256] == scales[0, 1]).all()


def test_top_logits_and_log_sum_exp():
    z = np.array([[1.0, 3.0, 3.0, -np.inf], [np.nan, 0.0, 5.0, 1.0], [-np.inf] * 4])
    top, index, lse = O.top_logits(z, 4, 2.0)
    assert index[0].tolist() == [1, 2, 0, -1] and top[0].tolist() == [3, 3, 1, -np.inf]
    assert index[1].tolist() == [0, 2, 3, 1] and np.isnan(lse[1]) and index[2].tolist() == [-1] * 4 and lse[2] == -np.inf
    assert np.isclose(lse[0], float(torch.logsumexp(torch.tensor([0.5, 1.5, 1.5], dtype=torch.float64), 0)))


def test_sampling():
    z = np.log(np.array([0.1, 0.4, 0.2, 0.3]))
    assert [O.sample(z, u)[0] for u in (0.0, 0.099, 0.11, 0.49, 0.51, 0.69, 0.71, 0.999)] == [0, 0, 1, 1, 2, 2, 3, 3]
    assert O.kept(z, 1.0, 2, 1.0, 0.0)[0].tolist() == [1, 3]
    assert O.kept(z, 1.0, 0, 0.65, 0.0)[0].tolist() == [1, 3] and O.kept(z, 1.0, 0, 0.75, 0.0)[0].tolist() == [1, 2, 3]
    assert O.kept(z, 1.0, 3, 0.75, 0.0)[0].tolist() == [1, 3]                      # of 0.4 / 0.9, 0.3 / 0.9, 0.2 / 0.9
    assert O.kept(z, 1.0, 0, 1.0, 0.6)[0].tolist() == [1, 3] and O.kept(z, 1.0, 0, 1e-9, 0.0)[0].tolist() == [1]
    assert O.kept(np.zeros(5), 1.0, 3, 1.0, 0.0)[0].tolist() == [0, 1, 2]          # equal ones: the lower index first
    token, logp = O.sample(z, 0.5, top_k=2)
    assert token == 1 and np.isclose(logp, np.log(4 / 7))
    assert O.sample(z, 0.5, temperature=0.0) == (1, 0.0) and O.sample(np.full(3, -np.inf), 0.5)[0] == -1


def test_clip():
    g = [np.array([3.0, 0.0]), np.array([[4.0]])]
    norm, c = O.clip(g, 1.0)
    assert norm == 5 and np.allclose(c[0], [0.6, 0]) and np.allclose(c[1], 0.8)
    assert O.clip(g, 1.0, True)[0] == 4 and (O.clip(g, 10.0)[1][0] == g[0]).all()

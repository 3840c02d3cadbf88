"""Tokens of rows with one large entry and a long tail of equal small ones, all of whose weights are rounded the same way, on the GPU against fp64: the
sums stay within V 2^-52 of the largest weight, without a filter within V 2^-51 and 2^-34 (weights of a drawn chunk, at most 2^14 of them, are rounded to 2^-48,
sums of a thread's four entries and more as well, chunks' sums to 2^-37 and less, 1024 of them)."""
import numpy as np
import pytest
import torch

from paper_2603_01875_amd import kdloss as K
from tests.test_gpu_rows import DT

pytestmark = pytest.mark.gpu
FEW = 2.0 ** -36                      # u's or top_p's product with a sum, exp (2^-39), relative to the sum
SETTINGS = [dict(), dict(min_p=1e-30), dict(top_p=1 - 2.0 ** -24), dict(top_p=1 - 2.0 ** -24, min_p=1e-30)]


def off(V, settings):
    return V * 2.0 ** -52 if settings else V * 2.0 ** -51 + 2.0 ** -34


def check(z, u, out, settings):
    """Each token's share of the sum holds u times the whole, and its logp is that share's, as far as the sums are known.  Indices in order, one peak."""
    z = z.double().numpy()
    top_p = float(np.float32(settings.get("top_p", 1.0)))
    for t in range(z.shape[0]):
        w = np.exp(z[t] - z[t].max())
        run = np.cumsum(w.astype(np.longdouble))
        S, err = float(run[-1]), off(z.shape[1], settings) + FEW * float(run[-1])
        # the nucleus: the peak, whose weight is 1, and of the tail the first ones, as many as reach top_p of the whole
        low = max(1.0, S * top_p) - err
        high = min(S, max(1.0, S * top_p + w.min() + err)) + err
        token, logp = int(out["token"][t]), float(out["logp"][t])
        assert 0 <= token < z.shape[1]
        before, behind = float(run[token] - w[token]), float(run[token])
        # (in order of the index the kept tail entries are the first ones: run is theirs as far as it goes)
        assert before - err <= float(u[t]) * high and float(u[t]) * low <= behind + err, (t, token, before, behind, float(u[t]))
        for total in (low, high):
            want = z[t][token] - z[t].max() - np.log(total)
            assert abs(logp - want) <= 2.0 ** -24 * abs(want) + 2 * err + (high - low), (t, token, logp, want)


@pytest.mark.parametrize("settings", SETTINGS, ids=lambda s: ",".join(s) or "all")
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V", [(64, 151_936), (3, 50_257), (8, 5000), (8, 4000)])
def test_a_peak_over_a_flat_tail(T, V, dtype, settings):
    tail = torch.linspace(-34.0, -8.0, T).to(DT[dtype])
    z = tail.view(-1, 1).expand(T, V).contiguous()
    z[:, 0] = 0
    u = 1 - 2.0 ** -torch.linspace(1, 24, T)
    check(z, u, K.kd_sample(z.cuda(), u.cuda(), **settings), settings)


@pytest.mark.parametrize("settings", SETTINGS, ids=lambda s: ",".join(s) or "all")
def test_a_peak_over_the_longest_tail(settings):
    """2^24 entries of 2^-38.5: a part in 2^14.5 of the row, which u passes."""
    V = 1 << 24
    z = torch.full((1, V), -26.75, dtype=torch.bfloat16)
    z[0, 0] = 0
    for u in (1 - 2.0 ** -15, 1 - 2.0 ** -17, 1 - 2.0 ** -24):
        u = torch.tensor([u])
        check(z, u, K.kd_sample(z.cuda(), u.cuda(), **settings), settings)


def test_a_long_top_k_over_a_flat_tail():
    """More entries than a list of the largest holds, of which top_k are kept: the sums are those of the whole row's passes."""
    V, k = 151_936, 100_000
    z = torch.full((2, V), -31.5)
    z[:, 0] = 0
    u = torch.tensor([0.5, 1 - 2.0 ** -24])
    out = K.kd_sample(z.cuda(), u.cuda(), top_k=k)
    total = 1 + (k - 1) * np.exp(-31.5)
    want = -np.log(total)
    assert out["token"].tolist() == [0, 0]
    assert (np.abs(out["logp"].cpu().double().numpy() - want) <= 2.0 ** -24 * abs(want) + k * 2.0 ** -52 + FEW * (total - 1) + 2.0 ** -50).all()

"""Tokens of rows with many equal logits on the GPU against the fp64 reference: which of them are kept, and in which order they are drawn."""
import numpy as np
import pytest
import torch

from oracle import beside_oracle as O
from paper_2603_01875_amd import kdloss as K
from tests.test_gpu_rows import np64, rows

pytestmark = pytest.mark.gpu
SURE = 2.0 ** -36                     # of the whole: the sums' error, as far as these lengths have it (V 2^-52 and exp's 2^-39)


def check(z, u, s, out):
    """Every token is a kept one and its logp its share, wherever the kept ones are sure; it is the reference's wherever u is.  An entry that equals the largest has
    a weight of 1, exactly: min_p of 1 keeps it.  Returns how many rows were sure, and how many of their tokens."""
    z, u = np64(z), np64(u)
    token, logp = out["token"].cpu().numpy(), np64(out["logp"])
    sure = pinned = 0
    for t in range(z.shape[0]):
        f = {k: float(np.float32(s.get(k, d))) for k, d in (("temperature", 1.0), ("top_p", 1.0), ("min_p", 0.0))}
        order = np.lexsort((np.arange(z[t].size), -z[t]))[:s.get("top_k", 0) or z[t].size]
        w = np.exp((z[t][order] - z[t].max()) / f["temperature"])
        run = np.cumsum(w)
        near = [np.abs(run / run[-1] - f["top_p"]).min()] if f["top_p"] < 1 else []
        near += [np.abs(w[w < 1] - f["min_p"]).min()] if f["min_p"] > 0 and (w < 1).any() else []
        if near and min(near) < SURE:
            continue
        sure += 1
        ids, wk = O.kept(z[t], f["temperature"], s.get("top_k", 0), f["top_p"], f["min_p"])
        at = np.searchsorted(ids, token[t])
        assert at < ids.size and ids[at] == token[t], (t, s, token[t])
        lp = np.log(wk[at] / wk.sum())
        assert abs(logp[t] - lp) <= 2.0 ** -24 * abs(lp) + 2.0 ** -34, (t, s, logp[t], lp)
        run = np.cumsum(wk) / wk.sum()
        if run.size == 1 or np.abs(run[:-1] - u[t]).min() >= SURE:
            pinned += 1
            assert token[t] == ids[np.searchsorted(run, u[t], side="right")], (t, s)
    return sure, pinned


SETTINGS = [dict(), dict(min_p=1.0), dict(min_p=0.05), dict(top_p=0.9), dict(top_p=0.31), dict(top_k=40), dict(top_k=700), dict(top_k=2000),
            dict(top_k=2000, min_p=1.0), dict(top_k=30, min_p=1.0), dict(top_p=0.77, min_p=1.0), dict(top_k=600, top_p=0.63, min_p=0.3), dict(temperature=0.5, top_p=0.9)]


@pytest.mark.parametrize("kind", ["equal", "zeros", "steps", "masked", "one", "lowest"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [101, 3001, 12_345])
def test_equal_logits(kind, dtype, V):
    T = 24
    z = rows(V, T, V, kind, dtype)
    u = torch.from_numpy(np.random.default_rng(V).random(T).astype(np.float32))
    for s in SETTINGS:
        sure, pinned = check(z, u, s, K.kd_sample(z.cuda(), u.cuda(), **s))
        assert sure == T and pinned >= T - 1, (s, sure, pinned)


@pytest.mark.parametrize("V", [101, 12_345])
def test_each_of_the_largest_is_drawn_in_order(V):
    """Seven entries share the largest logit: min_p of 1 leaves these, and each seventh of u draws one."""
    at = np.sort(np.random.default_rng(V).permutation(V)[:7])
    z = torch.randn(7, V)
    z[:, at] = 6.0
    u = ((torch.arange(7) + 0.5) / 7).float()
    for s in (dict(min_p=1.0), dict(min_p=1.0, top_p=0.999), dict(min_p=1.0, top_k=9), dict(min_p=1.0, top_k=1500), dict(top_k=7)):
        out = K.kd_sample(z.cuda(), u.cuda(), **s)
        assert out["token"].tolist() == at.tolist(), s
        assert (np.abs(np64(out["logp"]) + np.log(7)) <= 2.0 ** -24 * np.log(7) + 2.0 ** -34).all()
    out = K.kd_sample(z.cuda(), u.cuda(), top_k=3)                        # of equal ones the lower indices
    assert out["token"].tolist() == [at[i] for i in (0, 0, 1, 1, 1, 2, 2)]

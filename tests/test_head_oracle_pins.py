"""Pins of the fp64 reference of the one-head losses: closed forms, scipy, central differences."""
import numpy as np
import pytest
from scipy.special import logsumexp
from scipy.stats import entropy

from oracle import head_oracle as O

RNG = np.random.default_rng(5)
T, H, V, K = 6, 8, 24, 5


def _inputs():
    h, W = RNG.standard_normal((T, H)), RNG.standard_normal((V, H))
    return h, W


def _top():
    ids = np.stack([RNG.permutation(V)[:K] for _ in range(T)])
    return RNG.standard_normal((T, K)) * 2, ids


def test_uniform_student_costs_log_V():
    y = np.arange(T) % V
    assert O.cross_entropy(np.zeros((T, H)), np.ones((V, H)), y)["loss"] == pytest.approx(np.log(V), rel=1e-14)


def test_cross_entropy_is_the_divergence_from_its_smoothed_target():
    h, W = _inputs()
    y = RNG.integers(0, V, T)
    for eps in (0.0, 0.2):
        z = h @ W.T
        p = np.exp(z - logsumexp(z, axis=1, keepdims=True))
        q = np.full((T, V), eps / V)
        q[np.arange(T), y] += 1 - eps
        want = [entropy(q[t], p[t]) + entropy(q[t]) for t in range(T)]
        assert O.cross_entropy(h, W, y, smoothing=eps)["per_token_loss"] == pytest.approx(want, rel=1e-12)
    z_loss = O.cross_entropy(h, W, y, z_loss=0.5)["per_token_loss"] - O.cross_entropy(h, W, y)["per_token_loss"]
    assert z_loss == pytest.approx(0.5 * logsumexp(h @ W.T, axis=1) ** 2, rel=1e-12)


@pytest.mark.parametrize("tau", [1.0, 2.5])
def test_top_logits_renormalised_and_with_the_rest(tau):
    h, W = _inputs()
    a, ids = _top()
    z = h @ W.T / tau
    p = np.exp(z - logsumexp(z, axis=1, keepdims=True))
    q = np.exp(a / tau - logsumexp(a / tau, axis=1, keepdims=True))
    want = [entropy(q[t], p[t][ids[t]]) - np.log(p[t][ids[t]].sum()) for t in range(T)]      # scipy normalises p
    assert O.topk(a, ids, h, W, tau=tau)["per_token_loss"] == pytest.approx(want, rel=1e-12)
    lse = logsumexp(a / tau, axis=1) + 0.3
    q = q * np.exp(-0.3)
    cat = lambda x, full: np.append(x, full - x.sum())
    want = [entropy(cat(q[t], 1.0), cat(p[t][ids[t]], 1.0)) for t in range(T)]
    assert O.topk(a, ids, h, W, lse, tau=tau, tail=O.REST)["per_token_loss"] == pytest.approx(want, rel=1e-10)
    want = [(q[t] * np.log(q[t] / p[t][ids[t]])).sum() for t in range(T)]
    assert O.topk(a, ids, h, W, lse, tau=tau, tail=O.DROP)["per_token_loss"] == pytest.approx(want, rel=1e-12)


def test_all_logits_are_the_forward_divergence():
    """K = V, or the whole teacher split into a list and the rest of one entry."""
    from oracle import kd_oracle as KD
    h, W = _inputs()
    h_t, W_t = _inputs()
    z = h_t @ W_t.T
    ids = np.tile(np.arange(V), (T, 1))
    ref = KD.kd_loss_fwd_bwd(h_t, W_t, h, W, None, 1.0, 0, 0.5, KD.W_VH)
    for got in (O.topk(z, ids, h, W), O.topk(z[:, 1:], ids[:, 1:], h, W, logsumexp(z, axis=1), tail=O.REST)):
        for k, name in (("loss", "loss"), ("per_token_loss", "per_token_loss"), ("grad_h", "grad_h_s"), ("grad_W", "grad_W_s")):
            np.testing.assert_allclose(got[k], ref[name], rtol=1e-9, atol=1e-12)


def test_one_certain_entry_is_cross_entropy():
    h, W = _inputs()
    y = RNG.integers(0, V, T)
    ce, tk = O.cross_entropy(h, W, y), O.topk(np.zeros((T, 1)), y[:, None], h, W)
    for k in ("loss", "grad_h", "grad_W"):
        np.testing.assert_allclose(ce[k], tk[k], rtol=1e-12, atol=1e-15)


def test_same_row_twice_adds_up_and_absent_entries_do_not_count():
    h, W = _inputs()
    a, ids = _top()
    twice = O.topk(np.concatenate([a, a[:, :1]], 1), np.concatenate([ids, ids[:, :1]], 1), h, W)
    once = a.copy()
    once[:, 0] += np.log(2.0)
    np.testing.assert_allclose(twice["grad_h"], O.topk(once, ids, h, W)["grad_h"], rtol=1e-10)
    gone = O.topk(np.concatenate([a, np.full((T, 2), [9.0, -np.inf])], 1),
                  np.concatenate([ids, np.tile([-1, 3], (T, 1))], 1), h, W)
    np.testing.assert_allclose(gone["grad_W"], O.topk(a, ids, h, W)["grad_W"], rtol=1e-12)


@pytest.mark.parametrize("what", ["ce", "renorm", "rest", "drop"])
def test_gradients_are_the_slopes(what):
    h, W = _inputs()
    a, ids = _top()
    y = RNG.integers(0, V, T)
    y[2] = -100
    mask = np.ones(T)
    mask[4] = 0
    lse = logsumexp(a / 1.5, axis=1) + 0.4

    def f(h, W):
        if what == "ce":
            return O.cross_entropy(h, W, y, mask, 0.1, 0.01, scale=0.5)
        return O.topk(a, ids, h, W, lse, mask, 1.5, {"renorm": O.RENORM, "rest": O.REST, "drop": O.DROP}[what], tau2=True)
    out, eps = f(h, W), 1e-6
    for x, g, call in ((h, out["grad_h"], lambda x: f(x, W)), (W, out["grad_W"], lambda x: f(h, x))):
        for _ in range(12):
            i = tuple(RNG.integers(0, s) for s in x.shape)
            up, down = x.copy(), x.copy()
            up[i] += eps
            down[i] -= eps
            assert (call(up)["loss"] - call(down)["loss"]) / (2 * eps) == pytest.approx(g[i], abs=1e-8)
    assert (out["grad_h"][4] == 0).all() and (what != "ce" or (out["grad_h"][2] == 0).all())

"""The one-head losses at the ends of what their parameters allow: hardly a token that counts among many, the least and the largest
temperature, gradients of logits that share a large part."""
import numpy as np
import pytest
import torch

from oracle import head_oracle as O
from paper_2603_01875_amd import kdloss as K
from tests import head_util as U

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("count", [0, 1, 2])
@pytest.mark.parametrize("layout", ["vh", "hv"])
@pytest.mark.parametrize("grad", ["bf16", "f32"])
def test_hardly_a_token_counts(count, layout, grad):
    """Twelve token tiles, of which at most one has tokens, logits made twice: as a call on those tokens alone."""
    T, H, V, k = 3000, 64, 40000, 9
    h, W, y, rng = U.make(7, T, H, V, "bf16")
    a, ids = U.top_lists(rng, 8, V, k, y[:8])
    a, ids = a.repeat(T // 8, 1).cuda(), ids.repeat(T // 8, 1).cuda()
    hd, Wd = U.device(h, W, layout)
    mask, at = torch.zeros(T, dtype=torch.uint8, device="cuda"), [2999, 1234][:count]
    mask[at] = 1
    lse = torch.full((T,), 6.0, device="cuda")
    kw = dict(w_layout=U.LAYOUT[layout], grad_dtype=U.GRAD[grad])
    outs = [K.kd_ce_fwd_bwd(hd, Wd, y.cuda(), mask, 0.1, 1e-3, **kw), K.kd_topk_fwd_bwd(a, ids, hd, Wd, lse, mask, tail=K.TAIL_REST, **kw)]
    torch.cuda.synchronize()
    refs = [O.cross_entropy(U.np64(h[at]), U.np64(W), y[at].numpy(), None, 0.1, 1e-3),
            O.topk(U.np64(a[at]), ids[at].cpu().numpy(), U.np64(h[at]), U.np64(W), U.np64(lse[at]), tail=O.REST)] if count else [None, None]
    for out, ref, (gh, gW) in zip(outs, refs, (("grad_h", "grad_W"), ("grad_h_s", "grad_W_s"))):
        assert not out[gh][mask == 0].any() and not out["per_token_loss"][mask == 0].any()
        if not count:
            assert not out[gW].any() and float(out["loss"].item()) == 0
            continue
        some = dict(loss=out["loss"], per_token_loss=out["per_token_loss"][at], grad_h=out[gh][at], grad_W=out[gW])
        U.check(some, ref, U.np64(h[at]), U.np64(W), grad_dtype=grad, layout=layout, coefficient=2.5)


def _exact_logits(T, V, H=64, common=0.0, tau=1.0):
    """Hidden states and head whose logits over tau are `common` and sixteen bits behind it, exact in fp32."""
    rng = np.random.default_rng(T + V)
    W, h = np.zeros((V, H)), np.zeros((T, H))
    W[:, 0], h[:, 0] = 1.0, common * tau
    W[:, 1:9] = rng.integers(-8, 9, (V, 8)) / 8
    h[:, 1:9] = rng.integers(-4, 5, (T, 8)) / 4 * tau
    return rng, U.rounded(h, "bf16"), U.rounded(W, "bf16")


@pytest.mark.parametrize("T,chunk", [(20, 0), (100, 0), (300, 0), (300, 256)])
@pytest.mark.parametrize("tail", [O.RENORM, O.REST, O.DROP])
@pytest.mark.parametrize("common,tau", [(65536.0, 1.0), (0.0, 2.0 ** -19), (0.0, 2.0 ** 19), (65536.0, 2.0 ** -10)])
def test_gradients_of_large_parts_and_far_temperatures(T, chunk, tail, common, tau):
    """2^-19 and 2^19 are the powers of two next to 1e-6 and 1e6.  Logits over tau are exact, so only exp2's errors are left: dL/dz within
    2^-19 of its terms, as in head_util.bounds."""
    V, H, k = 1024, 64, 40
    rng, h, W = _exact_logits(T, V, H, common, tau)
    ids = torch.from_numpy(np.stack([rng.permutation(V)[:k] for _ in range(T)]))
    a = torch.from_numpy((rng.standard_normal((T, k)) * tau).astype(np.float32))
    lse = torch.from_numpy((np.log(np.exp(U.np64(a) / tau).sum(1)) + 0.5).astype(np.float32))
    n64 = U.np64(h), U.np64(W)
    ref = O.topk(U.np64(a), ids.numpy(), *n64, U.np64(lse), tau=tau, tail=tail, tau2=True)
    out = K.kd_topk_fwd_bwd(a.cuda(), ids.cuda(), *U.device(h, W), lse=None if tail == O.RENORM else lse.cuda(), tau=tau, tail=tail,
                            flags=K.FLAG_TAU2, grad_dtype=K.F32, vocab_chunk=chunk)
    tol = (2.0 ** -19 + 8 * U.F32 * 40) * tau * tau
    assert (np.abs(U.np64(out["per_token_loss"]) - ref["per_token_loss"]) <= tol).all()
    # terms of dz: p, q and rest p / p_rest, of which p / p_rest is at most p / (1 - P)
    p = np.exp(O.log_softmax(n64[0] @ n64[1].T / tau))
    on = np.zeros((T, V), bool)
    np.put_along_axis(on, ids.numpy(), True, 1)
    err = (p + p / np.where(on, 0, p).sum(1, keepdims=True)) * 2.0 ** -18 + np.abs(ref["dz"]) * 2.0 ** -21 + 2.0 ** -40
    s, whole = abs(ref["s"]), np.abs(ref["dz"]) + err
    sets = 6
    for g, want, bound in ((out["grad_h_s"], ref["grad_h"], s * (err @ np.abs(n64[1]) + (V * sets + 64) * U.F32 * (whole @ np.abs(n64[1])))),
                           (out["grad_W_s"], ref["grad_W"], s * (err.T @ np.abs(n64[0]) + (T * sets + 64) * U.F32 * (whole.T @ np.abs(n64[0]))))):
        assert (np.abs(U.np64(g) - want) <= bound + 5 * U.F32 * np.abs(want) + 1e-38).all()


@pytest.mark.parametrize("T", [20, 300])
def test_cross_entropy_gradients_of_a_large_common_part(T):
    V, H = 1024, 64
    rng, h, W = _exact_logits(T, V, H, 65536.0)
    y = torch.from_numpy(rng.integers(0, V, T))
    n64 = U.np64(h), U.np64(W)
    ref = O.cross_entropy(*n64, y.numpy())
    out = K.kd_ce_fwd_bwd(*U.device(h, W), y.cuda(), grad_dtype=K.F32)
    assert (np.abs(U.np64(out["per_token_loss"]) - ref["per_token_loss"]) <= 2.0 ** -19 + 8 * U.F32 * 40).all()
    p = np.exp(O.log_softmax(n64[0] @ n64[1].T))
    err = p * 2.0 ** -18 + np.abs(ref["dz"]) * 2.0 ** -21 + 2.0 ** -40
    whole, s = np.abs(ref["dz"]) + err, abs(ref["s"])
    bound = s * (err.T @ np.abs(n64[0]) + (T * 6 + 64) * U.F32 * (whole.T @ np.abs(n64[0]))) + 5 * U.F32 * np.abs(ref["grad_W"])
    assert (np.abs(U.np64(out["grad_W"]) - ref["grad_W"]) <= bound).all()

"""KD_TAIL_REST where the student is sure of the list: its mass beside it is far below what a float holds, while the gradient of what
lies there keeps adding up to the teacher's rest."""
import numpy as np
import pytest
import torch

from oracle import head_oracle as O
from paper_2603_01875_amd import kdloss as K
from tests import head_util as U

pytestmark = pytest.mark.gpu

GAPS = [1.0, 20.0, 60.0, 86.0, 88.0, 95.0, 120.0, 200.0, 400.0]      # nats between the list and the rest, at the temperature


def _inputs(T, dtype, tau, H=64, V=1024):
    g = torch.Generator().manual_seed(T)
    h, W = torch.zeros(T, H), torch.zeros(V, H)
    W[:, 0] = torch.linspace(-1, 1, V) * 0.1
    W[7, 1] = 1.0
    h[:, 0] = torch.randn(T, generator=g)
    h[:, 1] = torch.tensor(GAPS).repeat(T)[:T] * tau
    h[:, 2] = 1 + torch.rand(T, generator=g)               # (a column of grad_W that every token has a part in)
    return U.rounded(h, dtype), U.rounded(W, dtype)


def _bounds(h, W, ref, on, rest, tau, in_dtype, grad_dtype):
    """As head_util.bounds, with the errors of what lies beside the list relative to its own sum: dz = p - rest p / p_rest there, whose
    second term knows the logits beside the list only, and whose first is as far off as any p."""
    absh, absW = np.abs(h), np.abs(W)
    sets, parts = (1 if grad_dtype == "bf16" else 6), (6 if in_dtype == "f32" else 1)
    e = (h.shape[1] * parts + 11) * U.F32 * (absh @ absW.T) / tau
    worst, beside = e.max(1, keepdims=True), np.where(on, 0, e).max(1, keepdims=True)
    lp = O.log_softmax(h @ W.T / tau)
    p = np.exp(lp)
    out = np.where(on, 0.0, p)
    out /= out.sum(1, keepdims=True)
    dz_round = U.BF16 if grad_dtype == "bf16" else 2.0 ** -22
    dz_err = (p * (worst + e + 2.0 ** -19) + rest * out * (beside + e + 2.0 ** -19)
              + np.abs(ref["dz"]) * (dz_round + 2.0 ** -22) + 2.0 ** -40)
    dz_all = np.abs(ref["dz"]) + dz_err
    op = U.BF16 if in_dtype == "f32" and grad_dtype == "bf16" else 3 * U.F32 if in_dtype == "f32" else 0.0
    last = (U.BF16 if grad_dtype == "bf16" else U.F32) + 4 * U.F32
    T, V = ref["dz"].shape
    s = abs(ref["s"])
    gh = s * ((dz_err + op * dz_all) @ absW + (V * sets + 64) * U.F32 * (dz_all @ absW)) + last * np.abs(ref["grad_h"])
    gW = s * ((dz_err + op * dz_all).T @ absh + (T * sets + 64) * U.F32 * (dz_all.T @ absh)) + last * np.abs(ref["grad_W"])
    return 2 * worst[:, 0] + 2.0 ** -19 + 8 * U.F32 * max(GAPS), gh + 1e-38, gW + 1e-38


@pytest.mark.parametrize("T", [9, 40, 200, 300])
@pytest.mark.parametrize("chunk", [0, 256])
@pytest.mark.parametrize("tau", [1.0, 0.125])
@pytest.mark.parametrize("dtype,grad,layout", [("bf16", "bf16", "vh"), ("bf16", "f32", "hv"), ("f32", "f32", "vh"), ("bf16", "bf16", "hv")])
def test_the_rest_keeps_its_gradient(T, chunk, tau, dtype, grad, layout):
    h, W = _inputs(T, dtype, tau)
    V, rest = W.shape[0], 0.4
    a, ids = torch.zeros(T, 2), torch.tensor([[7, 3]]).repeat(T, 1)
    lse = torch.full((T,), float(np.log(2.0 / (1 - rest))))
    n64 = U.np64(h), U.np64(W)
    ref = O.topk(a.numpy(), ids.numpy(), *n64, U.np64(lse), tau=tau, tail=O.REST)
    assert np.isfinite(ref["dz"]).all()
    on = np.zeros((T, V), bool)
    on[:, [7, 3]] = True
    rows, gh, gW = _bounds(*n64, ref, on, rest, tau, dtype, grad)
    out = K.kd_topk_fwd_bwd(a.cuda(), ids.cuda(), *U.device(h, W, layout), lse.cuda(), tau=tau, tail=K.TAIL_REST,
                            w_layout=U.LAYOUT[layout], grad_dtype=U.GRAD[grad], vocab_chunk=chunk)
    torch.cuda.synchronize()
    assert (np.abs(U.np64(out["per_token_loss"]) - ref["per_token_loss"]) <= rows).all()
    got_W = U.np64(out["grad_W_s"] if layout == "vh" else out["grad_W_s"].T)
    assert np.isfinite(got_W).all() and (np.abs(U.np64(out["grad_h_s"]) - ref["grad_h"]) <= gh).all()
    assert (np.abs(got_W - ref["grad_W"]) <= gW).all()

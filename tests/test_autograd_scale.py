"""What the autograd front ends do with the factor that comes in from behind the loss: it is an fp32 number, and a gradient in bf16
is rounded once, after the product."""
import numpy as np
import pytest
import torch

from paper_2603_01875_amd import autograd as A
from paper_2603_01875_amd import kdloss as K

FACTORS = [0.3, -1.7, 1 / 3, 1e-4, 1.0]


def _tensors(device="cpu", T=70, H=128, V=1000, dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(5)
    return [(torch.randn(n, H, generator=g) * s).to(dtype).to(device).requires_grad_(True) for n, s in ((T, 1.0), (V, 0.05))]


def _check(got, stored, factor):
    want = stored.double() * float(np.float32(factor))
    once = want.float().to(stored.dtype)                   # (the product of a bf16 and an fp32 number has 32 bits: fp32, then bf16)
    assert got.dtype == stored.dtype
    step = torch.finfo(stored.dtype).eps / 2
    assert ((got.double() - want).abs() <= step * want.abs() * 1.0001 + 1e-38).all()
    assert (got == once).double().mean() > 0.999
    # no common shift: what the roundings leave is of both signs
    if want.abs().sum() > 0:
        assert abs(float((got.double() - want).sum() / want.abs().sum())) < 0.05 * step or factor == 1.0


@pytest.mark.parametrize("factor", FACTORS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_one_head_losses_multiply_once_rounded(factor, dtype):
    h, W = _tensors(dtype=dtype)
    grads = dict(grad_h=h.detach() * 0.7, grad_W=W.detach() * 0.9, loss=torch.ones(1))
    loss = A._HeadLossFn.apply(h, W, lambda gh, gW: grads, ("grad_h", "grad_W"))
    (factor * loss).backward()
    _check(h.grad, grads["grad_h"], factor)
    _check(W.grad, grads["grad_W"], factor)
    only = A._HeadLossFn.apply(h.detach(), W, lambda gh, gW: dict(grads, grad_h=None), ("grad_h", "grad_W"))
    assert torch.equal(torch.autograd.grad(factor * only, W)[0], W.grad)


@pytest.mark.gpu
@pytest.mark.parametrize("factor", [0.3, 1 / 3])
@pytest.mark.parametrize("T", [70, 300])
def test_one_head_losses_on_the_gpu(factor, T):
    """A factor behind the loss against the stored gradients, and against the same factor in front of it (loss_scale, which the
    library multiplies in fp32 in front of its only rounding): each is one rounding away from the same numbers, to fp32."""
    h, W = _tensors("cuda", T=T)
    y = torch.arange(T, device="cuda") * 3
    ids, a = torch.arange(5, device="cuda").repeat(T, 1), torch.randn(T, 5, device="cuda")
    calls = [lambda s=1.0: A.cross_entropy(h, W, y, loss_scale=s), lambda s=1.0: A.topk_loss(h, W, a, ids, loss_scale=s)]
    raw = [K.kd_ce_fwd_bwd(h.detach(), W.detach(), y), K.kd_topk_fwd_bwd(a, ids, h.detach(), W.detach())]
    for call, out in zip(calls, raw):
        got = torch.autograd.grad(factor * call(), (h, W))
        front = torch.autograd.grad(call(factor), (h, W))
        for g, f, stored in zip(got, front, (out.get("grad_h", out.get("grad_h_s")), out.get("grad_W", out.get("grad_W_s")))):
            _check(g.cpu(), stored.cpu(), factor)
            g, f = g.double(), f.double()
            assert ((g - f).abs() <= 3 * 2.0 ** -8 * f.abs() * 1.01 + 1e-38).all()     # three roundings lie between them
            assert abs(float((g.abs().sum() - f.abs().sum()) / f.abs().sum())) < 2.0 ** -12


@pytest.mark.parametrize("factor", FACTORS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_two_model_loss_multiplies_once_rounded(factor, dtype, monkeypatch):
    h, W = _tensors(dtype=dtype)
    grads = dict(grad_h_s=h.detach() * 0.7, grad_W_s=W.detach() * 0.9, loss=torch.ones(1))
    monkeypatch.setattr(K, "kd_loss_fwd_bwd", lambda *a, **k: grads)
    (factor * A.kd_loss(h, W, h.detach(), W.detach())).backward()
    _check(h.grad, grads["grad_h_s"], factor)
    _check(W.grad, grads["grad_W_s"], factor)


@pytest.mark.gpu
def test_two_model_loss_on_the_gpu():
    h, W = _tensors("cuda")
    h_t, W_t = (x.detach() for x in _tensors("cuda", H=192))
    out = K.kd_loss_fwd_bwd(h_t, W_t, h.detach(), W.detach())
    for factor in (0.3, 1 / 3, 1.0):
        got = torch.autograd.grad(factor * A.kd_loss(h, W, h_t, W_t), (h, W))
        _check(got[0].cpu(), out["grad_h_s"].cpu(), factor)
        _check(got[1].cpu(), out["grad_W_s"].cpu(), factor)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_two_model_loss_gradients_know_the_factor_in_a_graph_of_the_backward_pass(dtype, monkeypatch):
    h, W = _tensors(dtype=dtype)
    grads = dict(grad_h_s=h.detach() * 0.7, grad_W_s=W.detach() * 0.9, loss=torch.ones(1))
    monkeypatch.setattr(K, "kd_loss_fwd_bwd", lambda *a, **k: grads)
    w = torch.tensor(0.3, requires_grad=True)
    got = torch.autograd.grad(w * A.kd_loss(h, W, h.detach(), W.detach()), (h, W), create_graph=True)
    _check(got[0].detach(), grads["grad_h_s"], 0.3)
    slope, = torch.autograd.grad(got[0].sum(), w)
    assert float(slope) == pytest.approx(float(grads["grad_h_s"].double().sum()), rel=1e-2, abs=1e-2)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [70, 300])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_type_that_gradients_are_computed_in(T, dtype):
    """grad_dtype=F32: a bf16 leaf gets the fp32 gradient (head_util's bounds for it), rounded once."""
    from oracle import head_oracle as O
    from tests import head_util as U
    h, W, y, rng = U.make(T, T, 64, 1000, dtype)
    a, ids = U.top_lists(rng, T, 1000, 6, y)
    n64, factor = (U.np64(h), U.np64(W)), float(np.float32(0.3))
    hd, Wd = (x.requires_grad_(True) for x in U.device(h, W))
    for loss, ref in ((A.cross_entropy(hd, Wd, y.cuda(), grad_dtype=K.F32), O.cross_entropy(*n64, y.numpy())),
                      (A.topk_loss(hd, Wd, a.cuda(), ids.cuda(), grad_dtype=K.F32), O.topk(U.np64(a), ids.numpy(), *n64))):
        b = U.bounds(*n64, ref, 1.0, dtype, "f32")
        for g, k in zip(torch.autograd.grad(factor * loss, (hd, Wd)), ("grad_h", "grad_W")):
            assert g.dtype == hd.dtype
            last = U.BF16 * 1.001 if dtype == "bf16" else U.F32
            want, bound = factor * ref[k], factor * b[k] * 1.01
            assert (np.abs(U.np64(g) - want) <= bound + last * (np.abs(want) + bound)).all()
    bf = torch.autograd.grad(A.cross_entropy(hd, Wd, y.cuda(), grad_dtype=K.BF16), Wd)[0]      # (of fp32 operands, too)
    raw = K.kd_ce_fwd_bwd(hd.detach(), Wd.detach(), y.cuda(), grad_dtype=K.BF16)["grad_W"]
    assert bf.dtype == Wd.dtype and torch.equal(bf, raw.to(Wd.dtype))

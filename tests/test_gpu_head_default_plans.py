"""The one-head losses as a large call plans them by itself: several vocabulary chunks of the width that the library chooses, logits made
twice, more than four token tiles and a number of them that is no multiple of four.  Against the definition in 64 bits on the device, element by
element, within the bounds of head_util.bounds."""
import numpy as np
import pytest
import torch

from paper_2603_01875_amd import kdloss as K
from tests import head_util as U

pytestmark = pytest.mark.gpu

# T, tokens that count, H, V, types, order: 17 tiles x 32768 columns; x 16384 (three parts of dL/dz); 7 tiles; fp32 operands; one chunk
# (still too many logits to keep them)
PLANS = [(4357, 4200, 72, 40008, "bf16", "bf16", "vh"), (4357, 4200, 64, 40000, "bf16", "bf16", "hv"),
         (4357, 4200, 64, 40008, "bf16", "f32", "vh"), (2000, 1700, 64, 100000, "bf16", "bf16", "vh"),
         (2000, 1700, 64, 100032, "bf16", "bf16", "hv"), (1500, 1290, 64, 40008, "f32", "f32", "vh"), (700, 600, 64, 100000, "bf16", "bf16", "vh")]


def _plan(p):
    """Whether the call takes several chunks: its workspace is below that of a single one."""
    one = type(p).from_buffer_copy(p)
    one.vocab_chunk = (p.V + 255) // 256 * 256
    return K.kd_loss_workspace_size(p) < K.kd_loss_workspace_size(one)


def _inputs(T, n, H, V, dtype):
    g = torch.Generator(device="cuda").manual_seed(T + V)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    W = (torch.randn(V, H, device="cuda", generator=g) * 0.1).to(dt)
    y = torch.randint(0, V, (T,), device="cuda", generator=g)
    h = torch.randn(T, H, device="cuda", generator=g)
    h = (h + 60 * torch.rand(T, 1, device="cuda", generator=g) * W[y].float()).to(dt)
    mask = torch.zeros(T, dtype=torch.uint8, device="cuda")
    mask[torch.randperm(T, device="cuda", generator=g)[:n]] = 1
    return g, h, W, y, mask


def _check(out, h, W, keep, dz, rows, e, p_err, grad, dtype, layout, factor=1.0):
    """dz: [T, V] without 1 / n; e: errors of the logits; p_err: those of dz in front of its rounding."""
    n = int(keep.sum())
    parts, sets = (6 if dtype == "f32" else 1), (1 if grad == "bf16" else 6)
    worst = e.amax(1)
    tol = factor * (2 * worst + 2.0 ** -19 + 8 * U.F32 * 40)
    got = out["per_token_loss"].double()
    assert bool((got[~keep] == 0).all()) and bool(((got - rows).abs() <= tol)[keep].all())
    assert abs(float(out["loss"].double()) - float(rows[keep].sum() / n)) <= float(tol.max())
    dz, p_err = dz * keep[:, None], p_err * keep[:, None]
    err = p_err + dz.abs() * ((U.BF16 if grad == "bf16" else 2.0 ** -22) + 2.0 ** -22) + 2.0 ** -40
    whole = dz.abs() + err
    op, last = (3 * U.F32 if dtype == "f32" else 0.0), (U.BF16 if grad == "bf16" else U.F32) + 4 * U.F32
    T, V = dz.shape
    for name, a, b, length in (("grad_h", lambda x: x @ W.double(), lambda x: x @ W.double().abs(), V),
                               ("grad_W", lambda x: x.t().contiguous() @ h.double(), lambda x: x.t().contiguous() @ h.double().abs(), T)):
        ref = a(dz) / n
        bound = (b(err) + (op + (length * sets + 64) * U.F32) * b(whole)) / n + last * ref.abs() + 1e-38
        g = out.get(name, out.get(name + "_s")).double()
        g = g.t() if name == "grad_W" and layout == "hv" else g
        off = (g - ref).abs() - bound
        assert float(off.max()) <= 0, (name, float(off.max()), int(off.argmax()), float(ref.abs().max()))
        if name == "grad_h":
            assert bool((g[~keep] == 0).all())


@pytest.mark.parametrize("T,n,H,V,dtype,grad,layout", PLANS)
def test_cross_entropy(T, n, H, V, dtype, grad, layout):
    g, h, W, y, mask = _inputs(T, n, H, V, dtype)
    smoothing, z_loss = 0.1, 1e-3
    p = K.make_ce_params(T, H, V, smoothing, z_loss, K.BF16 if dtype == "bf16" else K.F32, U.GRAD[grad], U.LAYOUT[layout])
    assert _plan(p) == (T > 700)
    out = K.kd_ce_fwd_bwd(h, W if layout == "vh" else W.t().contiguous(), y, mask, smoothing, z_loss, U.LAYOUT[layout], U.GRAD[grad])
    hd, Wd = h.double(), W.double().t().contiguous()
    z = hd @ Wd
    e = (H * (6 if dtype == "f32" else 1) + 11) * U.F32 * (hd.abs() @ Wd.abs())
    lse = torch.logsumexp(z, 1, keepdim=True)
    prob = (z - lse).exp()
    at = y[:, None]
    rows = (lse - (1 - smoothing) * z.gather(1, at) - smoothing * z.mean(1, keepdim=True) + z_loss * lse * lse)[:, 0]
    dz = prob * (1 + 2 * z_loss * lse) - smoothing / V
    dz.scatter_add_(1, at, torch.full_like(lse, smoothing - 1))
    factor = 1 + 64 * z_loss
    p_err = factor * prob * (e.amax(1, keepdim=True) + e + 2.0 ** -19)
    _check(out, h, W, mask != 0, dz, rows, e, p_err, grad, dtype, layout, factor)


@pytest.mark.parametrize("T,n,H,V,dtype,grad,layout", PLANS)
def test_top_logits_with_the_rest(T, n, H, V, dtype, grad, layout):
    g, h, W, y, mask = _inputs(T, n, H, V, dtype)
    k = 70
    p = K.make_topk_params(T, H, V, k, tail=K.TAIL_REST, in_dtype=K.BF16 if dtype == "bf16" else K.F32, grad_dtype=U.GRAD[grad],
                           w_layout=U.LAYOUT[layout])
    assert _plan(p) == (T > 700)
    # the token's row and others at equal steps over the vocabulary, all different; a fifth of them not there
    step = torch.randint(1, V // k, (T, 1), device="cuda", generator=g)
    ids = (y[:, None] + torch.arange(k, device="cuda") * step) % V
    a = torch.randn(T, k, device="cuda", generator=g) * 2
    ids[:, 1:][torch.rand(T, k - 1, device="cuda", generator=g) < 0.2] = -1
    there = ids >= 0
    lse_t = (torch.logsumexp(a.masked_fill(~there, -float("inf")), 1) + 0.3)
    out = K.kd_topk_fwd_bwd(a, ids, h, W if layout == "vh" else W.t().contiguous(), lse_t, mask, 1.0, K.TAIL_REST, U.LAYOUT[layout],
                            U.GRAD[grad])
    hd, Wd = h.double(), W.double().t().contiguous()
    z = hd @ Wd
    e = (H * (6 if dtype == "f32" else 1) + 11) * U.F32 * (hd.abs() @ Wd.abs())
    lse = torch.logsumexp(z, 1, keepdim=True)
    prob = (z - lse).exp()
    at = ids.clamp(min=0)
    q = torch.where(there, (a.double() - lse_t.double()[:, None]).exp(), 0.0)
    on = torch.zeros(T, V, device="cuda", dtype=torch.float64).scatter_add_(1, at, there.double()) > 0
    dense = torch.zeros(T, V, device="cuda", dtype=torch.float64).scatter_add_(1, at, q)
    rest = (1 - q.sum(1, keepdim=True)).clamp(min=0)
    assert float(rest.min()) > 0.2
    lse_out = torch.logsumexp(z.masked_fill(on, -float("inf")), 1, keepdim=True)
    out_p = (z - lse_out).exp().masked_fill(on, 0)
    rows = (torch.where(there, q * (torch.log(q) - (z.gather(1, at) - lse)), 0.0).sum(1) + (rest * (torch.log(rest) - (lse_out - lse)))[:, 0])
    dz = prob - dense - rest * out_p
    worst = e.amax(1, keepdim=True)
    p_err = (prob + rest * out_p) * (worst + e + 2.0 ** -19)
    _check(out, h, W, mask != 0, dz, rows, e, p_err, grad, dtype, layout)

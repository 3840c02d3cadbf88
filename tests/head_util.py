"""Helpers of the one-head losses' GPU tests: seeded inputs, calls, and comparison with the fp64 reference within bounds that
follow from the roundings."""
import numpy as np
import torch

from oracle import head_oracle as O
from paper_2603_01875_amd import kdloss as K

BF16, F32 = 2.0 ** -8, 2.0 ** -24          # half a step


def rounded(x, dtype):
    return torch.from_numpy(np.asarray(x, np.float32)).to(torch.bfloat16 if dtype == "bf16" else torch.float32)


def make(seed, T, H, V, dtype, lean=6.0, w_std=0.05):
    """Hidden states that lean towards a token's row, the head and the tokens, as torch CPU tensors in `dtype`."""
    rng = np.random.default_rng(seed)
    W = rng.standard_normal((V, H)) * w_std
    y = rng.integers(0, V, T)
    norm = np.linalg.norm(W[y], axis=1, keepdims=True)
    h = rng.standard_normal((T, H)) + rng.random((T, 1)) * lean * W[y] / norm ** 2
    return rounded(h, dtype), rounded(W, dtype), torch.from_numpy(y), rng


def top_lists(rng, T, V, k, y):
    ids = np.stack([rng.permutation(V)[:k] for _ in range(T)])
    ids[:, 0] = np.where((ids[:, 1:] == np.asarray(y)[:, None]).any(1), ids[:, 0], y)
    a = rng.standard_normal((T, k)) * 2
    return torch.from_numpy(a.astype(np.float32)), torch.from_numpy(ids)


def np64(t):
    return t.detach().cpu().double().numpy()


def bounds(h, W, ref, tau, in_dtype, grad_dtype, coefficient=1.0):
    """How far the outputs may be off, element by element.

    A logit is an fp32 sum of K products (K = H, or 6 H parts): K 2^-24 sum |h| |W| at most; fp32 operands in three parts miss
    less than 3 2^-24 of each product.  A log-sum-exp is off by as much as the logits, and by 2^-22 (exp2, log2 and its own
    rounding, in base 2, of size up to 32); p by the sum of both, times itself.  dL/dz then takes its roundings: 2^-8 for bf16
    gradients, 2^-23 in parts.  The products are fp32 sums of T or V terms; the result is rounded once."""
    absh, absW = np.abs(h), np.abs(W)
    parts = 6 if in_dtype == "f32" else 1
    dz_logit = ((h.shape[1] * parts + 8) * F32 * (absh @ absW.T) + 3 * F32 * (absh @ absW.T)) / tau
    worst = dz_logit.max(axis=1, keepdims=True)
    row = 2 * worst[:, 0] + 2.0 ** -19
    p_err = coefficient * (worst + dz_logit + 2.0 ** -19)
    z = h @ W.T / tau
    p = np.exp(O.log_softmax(z))
    dz_round = BF16 if grad_dtype == "bf16" else 2.0 ** -22
    dz_err = p * p_err + np.abs(ref["dz"]) * dz_round + 2.0 ** -22 * np.abs(ref["dz"]) + 2.0 ** -40
    dz_all = np.abs(ref["dz"]) + dz_err
    s = abs(ref["s"])
    T, V = ref["dz"].shape
    op = BF16 if in_dtype == "f32" and grad_dtype == "bf16" else 3 * F32 if in_dtype == "f32" else 0.0   # the other factor
    out = BF16 if grad_dtype == "bf16" else F32
    sets = 1 if grad_dtype == "bf16" else 6
    gh = s * ((dz_err + op * dz_all) @ absW + (V * sets + 64) * F32 * (dz_all @ absW))
    gW = s * ((dz_err + op * dz_all).T @ absh + (T * sets + 64) * F32 * (dz_all.T @ absh))
    return dict(rows=row, grad_h=gh + (out + 4 * F32) * np.abs(ref["grad_h"]) + 1e-38,
                grad_W=gW + (out + 4 * F32) * np.abs(ref["grad_W"]) + 1e-38)


def check(out, ref, h, W, tau=1.0, in_dtype="bf16", grad_dtype="bf16", layout="vh", factor=1.0, coefficient=1.0, magnitude=None):
    """`out`: dict of a *_fwd_bwd or *_fwd call.  `factor`: what losses are multiplied by; `magnitude`: size of the terms whose
    sum a token's loss is."""
    b = bounds(h, W, ref, tau, in_dtype, grad_dtype, coefficient)
    size = (40.0 if magnitude is None else magnitude)
    tol = abs(factor) * coefficient * (b["rows"] + 8 * F32 * size)
    rows = np64(out["per_token_loss"])
    assert np.isfinite(rows).all()
    assert (np.abs(rows - ref["per_token_loss"]) <= tol).all(), np.abs(rows - ref["per_token_loss"]).max()
    assert (rows[ref["per_token_loss"] == 0] == 0).all() or ref["n"] == len(rows)
    assert abs(float(out["loss"].item()) - ref["loss"]) <= tol.max()
    for k, alt in (("grad_h", "grad_h_s"), ("grad_W", "grad_W_s")):
        g = out.get(k, out.get(alt))
        if g is None:
            continue
        assert g.dtype == (torch.bfloat16 if grad_dtype == "bf16" else torch.float32)
        g = np64(g)
        g = g.T if k == "grad_W" and layout == "hv" else g
        off = np.abs(g - ref[k]) - b[k]
        assert (off <= 0).all(), (k, off.max(), np.unravel_index(off.argmax(), off.shape), np.abs(ref[k]).max())


def device(h, W, layout="vh"):
    return h.cuda(), (W if layout == "vh" else W.t().contiguous()).cuda()


LAYOUT = {"vh": K.W_VH, "hv": K.W_HV}
GRAD = {"bf16": K.BF16, "f32": K.F32}

"""What the one-head losses refuse, checked on the host: nothing is enqueued and no GPU is needed."""
import ctypes

import pytest
import torch

from paper_2603_01875_amd import autograd as A
from paper_2603_01875_amd import kdloss as K

NULL, SHAPE, ALIGN, PARAM, WORKSPACE = 1, 2, 3, 4, 5


def _ptrs(n):
    return [ctypes.c_void_p(0x100000 * (i + 1)) for i in range(n)]


def _ce(p, ptrs=None, nbytes=1 << 40, back=True):
    L = K.lib()
    a = _ptrs(8) if ptrs is None else ptrs          # h W labels mask loss ptl grad_h grad_W; workspace
    ws = ctypes.c_void_p(0x4000000) if len(a) == 8 else a[8]
    call = [a[0], a[1], a[2], a[3], a[4], a[5]] + (a[6:8] if back else [])
    return (L.kd_ce_fwd_bwd if back else L.kd_ce_fwd)(ctypes.byref(p) if p else None, *call, ws, ctypes.c_size_t(nbytes), None)


def _topk(p, ptrs=None, nbytes=1 << 40, back=True):
    L = K.lib()
    a = _ptrs(10) if ptrs is None else ptrs         # top index lse h W mask loss ptl grad_h grad_W
    ws = ctypes.c_void_p(0x4000000) if len(a) == 10 else a[10]
    call = a[:8] + (a[8:10] if back else [])
    return (L.kd_topk_fwd_bwd if back else L.kd_topk_fwd)(ctypes.byref(p) if p else None, *call, ws, ctypes.c_size_t(nbytes), None)


# (a workspace of 0 bytes is the last check: a call that gets that far passed the others)
@pytest.mark.parametrize("kw,status", [
    (dict(), WORKSPACE), (dict(T=0), SHAPE), (dict(T=(1 << 22) + 1), SHAPE), (dict(H=65544), SHAPE), (dict(V=(1 << 24) + 8), SHAPE),
    (dict(H=12), ALIGN), (dict(V=1004), ALIGN), (dict(in_dtype=2), PARAM), (dict(grad_dtype=-1), PARAM), (dict(w_layout=2), PARAM),
    (dict(index_dtype=2), PARAM), (dict(label_smoothing=1.0), PARAM), (dict(label_smoothing=-0.1), PARAM),
    (dict(label_smoothing=float("nan")), PARAM), (dict(z_loss=-1.0), PARAM), (dict(z_loss=float("inf")), PARAM),
    (dict(loss_scale=0.0), PARAM), (dict(loss_scale=float("nan")), PARAM), (dict(vocab_chunk=100), PARAM),
    (dict(label_smoothing=0.5, z_loss=1.0, vocab_chunk=256, loss_scale=-2.0, index_dtype=0, w_layout=0), WORKSPACE)])
@pytest.mark.parametrize("back", [True, False])
def test_ce_parameters(kw, status, back):
    kw = dict(dict(T=16, H=64, V=1000), **kw)
    p = K.make_ce_params(kw.pop("T"), kw.pop("H"), kw.pop("V"), **kw)
    assert _ce(p, nbytes=0, back=back) == status
    n = ctypes.c_size_t(0)
    assert K.lib().kd_ce_workspace_size(ctypes.byref(p), ctypes.byref(n)) == (0 if status == WORKSPACE else status)
    p.reserved = 1
    assert _ce(p, nbytes=0, back=back) == (PARAM if status == WORKSPACE else status)


@pytest.mark.parametrize("kw,status", [
    (dict(), WORKSPACE), (dict(K=0), SHAPE), (dict(K=K.TOPK_MAX + 1, V=8000), SHAPE), (dict(K=K.TOPK_MAX, V=8000), WORKSPACE),
    (dict(K=9, V=8), SHAPE), (dict(K=8, V=8), WORKSPACE), (dict(K=8, V=8, tail=K.TAIL_REST), SHAPE),
    (dict(K=7, V=8, tail=K.TAIL_REST), WORKSPACE), (dict(tail=3), PARAM), (dict(top_dtype=2), PARAM), (dict(tau=0.0), PARAM),
    (dict(tau=float("nan")), PARAM), (dict(tau=2e6), PARAM), (dict(flags=2), PARAM), (dict(flags=1), WORKSPACE), (dict(H=4), ALIGN),
    (dict(index_dtype=5), PARAM), (dict(loss_scale=0.0), PARAM), (dict(vocab_chunk=1 << 21), PARAM)])
@pytest.mark.parametrize("back", [True, False])
def test_topk_parameters(kw, status, back):
    kw = dict(dict(T=16, H=64, V=1000, K=4), **kw)
    p = K.make_topk_params(kw.pop("T"), kw.pop("H"), kw.pop("V"), kw.pop("K"), **kw)
    assert _topk(p, nbytes=0, back=back) == status
    n = ctypes.c_size_t(0)
    assert K.lib().kd_topk_workspace_size(ctypes.byref(p), ctypes.byref(n)) == (0 if status == WORKSPACE else status)
    p.reserved[1] = 1
    assert _topk(p, nbytes=0, back=back) == (PARAM if status == WORKSPACE else status)


def test_pointers():
    ce = K.make_ce_params(16, 64, 1000)
    for i in (0, 1, 2, 4):
        a = _ptrs(8)
        a[i] = None
        assert _ce(ce, a) == NULL and _ce(ce, a, back=False) == NULL, i
    a = _ptrs(8)
    a[3] = a[5] = a[6] = None                          # mask, per-token losses and one gradient may be missing
    assert _ce(ce, a, nbytes=0) == WORKSPACE
    a[7] = None                                        # ... not both
    assert _ce(ce, a, nbytes=0) == NULL
    assert _ce(ce, _ptrs(8) + [None]) == NULL
    for i, off, status in ((0, 8, ALIGN), (1, 8, ALIGN), (2, 4, ALIGN), (4, 2, ALIGN), (5, 1, ALIGN), (6, 8, ALIGN), (7, 4, ALIGN),
                           (3, 1, WORKSPACE)):
        a = _ptrs(8)
        a[i] = ctypes.c_void_p(a[i].value + off)
        assert _ce(ce, a, nbytes=0) == status, i
    assert _ce(K.make_ce_params(16, 64, 1000, index_dtype=K.I32), [x if i != 2 else ctypes.c_void_p(0x300004) for i, x in enumerate(_ptrs(8))],
               nbytes=0) == WORKSPACE
    for tail in (K.TAIL_RENORM, K.TAIL_REST, K.TAIL_DROP):
        tk = K.make_topk_params(16, 64, 1000, 4, tail=tail)
        for i in range(10):
            a = _ptrs(10)
            a[i] = None
            fine = i in (5, 7, 8, 9) or (i == 2 and tail == K.TAIL_RENORM)
            assert _topk(tk, a, nbytes=0) == (WORKSPACE if fine else NULL), (tail, i)
    assert _ce(None) == NULL and _topk(None) == NULL
    assert K.lib().kd_ce_workspace_size(ctypes.byref(ce), None) == NULL


def test_workspace_is_enough_for_either_direction_and_grows_slowly():
    for T, H, V in ((1, 8, 8), (100, 256, 5000), (4096, 1024, 151936), (8192, 4096, 128256)):
        p = K.make_ce_params(T, H, V)
        n = K.kd_loss_workspace_size(p)
        assert _ce(p, nbytes=n - 1) == WORKSPACE
        assert n < 64 << 20 or n < 2 * T * V * 2 // 3
    # (fp32 gradients hold dL/dz in several parts)
    assert K.kd_loss_workspace_size(K.make_ce_params(8192, 4096, 128256, grad_dtype=K.F32)) < 2 << 30


def test_binding_refuses_what_the_library_cannot_see():
    h, W, y = torch.zeros(4, 64), torch.zeros(16, 64), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError, match="CUDA"):
        K.kd_ce_fwd(h, W, y, workspace=torch.zeros(1))
    with pytest.raises(ValueError, match="2-dimensional"):
        K.kd_ce_fwd(h[0], W, y)
    with pytest.raises(ValueError, match="bfloat16 or float32"):
        K.kd_ce_fwd(h.half(), W.half(), y)
    with pytest.raises(ValueError, match="W is"):
        K.kd_ce_fwd(h, W.bfloat16(), y)
    with pytest.raises(ValueError, match="expected"):
        K.kd_ce_fwd(h, W, y, w_layout=K.W_HV)
    with pytest.raises(ValueError, match="int32 or int64"):
        K.kd_ce_fwd(h, W, y.float())
    with pytest.raises(ValueError, match="accumulate"):
        K.kd_ce_fwd_bwd(h, W, y, accumulate_grad_W=True)
    idx = torch.zeros(4, 3, dtype=torch.int64)
    with pytest.raises(ValueError, match=r"\[T, K\]"):
        K.kd_topk_fwd(torch.zeros(4, 2), idx, h, W)
    with pytest.raises(ValueError, match=r"\[T, K\]"):
        K.kd_topk_fwd(torch.zeros(3, 3), idx[:3], h, W)
    with pytest.raises(ValueError, match="top_logits must be"):
        K.kd_topk_fwd(torch.zeros(4, 3).half(), idx, h, W)
    with pytest.raises(ValueError, match="int32 or int64"):
        A.topk_loss(h, W, torch.zeros(4, 3), idx.short())
    p = K.make_ce_params(4, 64, 16, in_dtype=K.F32)
    with pytest.raises(ValueError, match="CUDA"):
        K.kd_ce_fwd_raw(p, h, W, y, None, torch.zeros(1), None, torch.zeros(16))

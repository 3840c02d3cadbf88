"""What the calls beside the losses refuse, checked on the host: nothing is enqueued and no GPU is needed."""
import ctypes

import pytest
import torch

from paper_2603_01875_amd import kdloss as K

NULL, SHAPE, ALIGN, PARAM, WORKSPACE = 1, 2, 3, 4, 5
BIG = ctypes.c_size_t(1 << 40)


def ptrs(n):
    return [ctypes.c_void_p(0x100000 * (i + 1)) for i in range(n)]


def size_of(name, p):
    n = ctypes.c_size_t(0)
    st = getattr(K.lib(), name)(ctypes.byref(p), ctypes.byref(n))
    assert getattr(K.lib(), name)(ctypes.byref(p), None) == NULL
    return st, n.value


@pytest.mark.parametrize("kw,status", [
    (dict(rows=0), SHAPE), (dict(cols=0), SHAPE), (dict(rows=(1 << 24) + 1), SHAPE), (dict(cols=(1 << 22) + 1), SHAPE), (dict(ld=99), SHAPE),
    (dict(src_dtype=2), PARAM), (dict(block=2), PARAM), (dict(block=-1), PARAM), (dict(rows=(1 << 22) + 1), SHAPE)])
def test_quantiser_parameters(kw, status):
    p = K.make_blocks_params(**dict(dict(rows=10, cols=100), **kw))
    assert K.lib().kd_quantize_e4m3_blocks(ctypes.byref(p), *ptrs(5), None) == status


def test_quantiser_pointers():
    L = K.lib()
    p = K.make_blocks_params(10, 100)
    assert L.kd_quantize_e4m3_blocks(None, *ptrs(5), None) == NULL
    for missing in ([0], [1], [2], [3], [4], [1, 2, 3, 4]):
        a = ptrs(5)
        for i in missing:
            a[i] = None
        assert L.kd_quantize_e4m3_blocks(ctypes.byref(p), *a, None) == NULL
    for i, off in ((0, 1), (1, 8), (2, 2), (3, 8), (4, 1)):
        a = ptrs(5)
        a[i] = ctypes.c_void_p(a[i].value + off)
        assert L.kd_quantize_e4m3_blocks(ctypes.byref(p), *a, None) == ALIGN
    p.reserved[1] = 1
    assert L.kd_quantize_e4m3_blocks(ctypes.byref(p), *ptrs(5), None) == PARAM


# (a workspace of 0 bytes is the last check: a call that gets that far passed the others)
@pytest.mark.parametrize("kw,status", [
    (dict(), WORKSPACE), (dict(M=0), SHAPE), (dict(N=0), SHAPE), (dict(K=0), SHAPE), (dict(M=(1 << 24) + 1), SHAPE),
    (dict(N=(1 << 24) + 1), SHAPE), (dict(K=(1 << 22) + 1), SHAPE), (dict(in_dtype=2), PARAM), (dict(out_dtype=-1), PARAM),
    (dict(b_block=2), PARAM)])
def test_product_parameters(kw, status):
    p = K.make_linear_params(**dict(dict(M=4, N=8, K=100), **kw))
    L = K.lib()
    a = ptrs(6)
    assert L.kd_matmul_e4m3(ctypes.byref(p), *a, ctypes.c_size_t(0), None) == status
    assert L.kd_linear_e4m3(ctypes.byref(p), *a[:5], ctypes.c_size_t(0), None) == status
    assert size_of("kd_linear_workspace_size", p)[0] == (0 if status == WORKSPACE else status)
    p.accumulate = 2
    assert L.kd_matmul_e4m3(ctypes.byref(p), *a, BIG, None) == (PARAM if status == WORKSPACE else status)


def test_product_pointers():
    L = K.lib()
    p = K.make_linear_params(4, 8, 100)
    assert L.kd_matmul_e4m3(None, *ptrs(6), BIG, None) == NULL
    for i in range(6):
        a = ptrs(6)
        a[i] = None
        assert L.kd_matmul_e4m3(ctypes.byref(p), *a, BIG, None) == NULL
    for i, off in ((0, 8), (1, 2), (2, 8), (3, 1), (4, 1), (5, 128)):
        a = ptrs(6)
        a[i] = ctypes.c_void_p(a[i].value + off)
        assert L.kd_matmul_e4m3(ctypes.byref(p), *a, BIG, None) == ALIGN
    for i, off in ((0, 1), (1, 8), (2, 1), (3, 1), (4, 16)):
        a = ptrs(5)
        a[i] = ctypes.c_void_p(a[i].value + off)
        assert L.kd_linear_e4m3(ctypes.byref(p), *a, BIG, None) == ALIGN
        a[i] = None
        assert L.kd_linear_e4m3(ctypes.byref(p), *a, BIG, None) == NULL
    p.b_block = K.BLOCK_ROW
    assert L.kd_linear_e4m3(ctypes.byref(p), *ptrs(5), BIG, None) == PARAM


@pytest.mark.parametrize("kw,status", [
    (dict(), WORKSPACE), (dict(T=0), SHAPE), (dict(T=(1 << 22) + 1), SHAPE), (dict(V=0), SHAPE), (dict(V=(1 << 24) + 1), SHAPE),
    (dict(ld=999), SHAPE), (dict(K=0), SHAPE), (dict(K=1001), SHAPE), (dict(K=1025, V=2000), SHAPE), (dict(K=1024, V=2000), WORKSPACE),
    (dict(in_dtype=2), PARAM), (dict(index_dtype=2), PARAM), (dict(tau=0.0), PARAM), (dict(tau=float("nan")), PARAM), (dict(tau=2e6), PARAM)])
def test_top_logits_parameters(kw, status):
    p = K.make_top_logits_params(**dict(dict(T=4, V=1000, K=10), **kw))
    assert K.lib().kd_top_logits(ctypes.byref(p), *ptrs(5), ctypes.c_size_t(0), None) == status
    st, n = size_of("kd_top_logits_workspace_size", p)
    assert st == (0 if status == WORKSPACE else status)
    if st == 0:
        assert K.lib().kd_top_logits(ctypes.byref(p), *ptrs(5), ctypes.c_size_t(n - 1), None) == WORKSPACE
    p.reserved[0] = 1
    assert K.lib().kd_top_logits(ctypes.byref(p), *ptrs(5), BIG, None) == (PARAM if status == WORKSPACE else status)


@pytest.mark.parametrize("kw,status", [
    (dict(), WORKSPACE), (dict(T=0), SHAPE), (dict(V=0), SHAPE), (dict(ld=10), SHAPE), (dict(in_dtype=3), PARAM), (dict(index_dtype=-1), PARAM),
    (dict(temperature=-1.0), PARAM), (dict(temperature=1e-7), PARAM), (dict(temperature=float("nan")), PARAM), (dict(temperature=0.0), WORKSPACE),
    (dict(top_k=-1), PARAM), (dict(top_k=5000), WORKSPACE), (dict(top_p=0.0), PARAM), (dict(top_p=1.1), PARAM), (dict(top_p=float("nan")), PARAM),
    (dict(min_p=-0.1), PARAM), (dict(min_p=1.1), PARAM), (dict(min_p=1.0), WORKSPACE)])
def test_sampling_parameters(kw, status):
    p = K.make_sample_params(**dict(dict(T=4, V=1000), **kw))
    assert K.lib().kd_sample(ctypes.byref(p), *ptrs(9), ctypes.c_size_t(0), None) == status
    st, n = size_of("kd_sample_workspace_size", p)
    assert st == (0 if status == WORKSPACE else status)
    if st == 0:
        assert K.lib().kd_sample(ctypes.byref(p), *ptrs(9), ctypes.c_size_t(n - 1), None) == WORKSPACE
    p.reserved[1] = 1
    assert K.lib().kd_sample(ctypes.byref(p), *ptrs(9), BIG, None) == (PARAM if status == WORKSPACE else status)


def test_rows_pointers():
    L = K.lib()
    t, s = K.make_top_logits_params(4, 1000, 10), K.make_sample_params(4, 1000)
    for i, off, needed in ((0, 1, True), (1, 1, True), (2, 4, True), (3, 2, False), (4, 64, True)):
        a = ptrs(5)
        a[i] = ctypes.c_void_p(a[i].value + off)
        assert L.kd_top_logits(ctypes.byref(t), *a, BIG, None) == ALIGN
        if needed:
            a[i] = None
            assert L.kd_top_logits(ctypes.byref(t), *a, BIG, None) == NULL
    # logits u temperature top_k top_p min_p token logp workspace
    for i, off, needed in ((0, 1, True), (1, 2, True), (2, 1, False), (3, 1, False), (4, 2, False), (5, 3, False), (6, 4, True), (7, 1, False),
                           (8, 16, True)):
        a = ptrs(9)
        a[i] = ctypes.c_void_p(a[i].value + off)
        assert L.kd_sample(ctypes.byref(s), *a, BIG, None) == ALIGN
        if needed:
            a[i] = None
            assert L.kd_sample(ctypes.byref(s), *a, BIG, None) == NULL


def test_gradient_lists():
    L = K.lib()

    def lists(n=2, counts=(10, 20), dtypes=(0, 1), at=(0x1000, 0x2000)):
        return [n, (ctypes.c_void_p * 2)(*at), (ctypes.c_int64 * 2)(*counts), (ctypes.c_int32 * 2)(*dtypes)]
    total, ws = ctypes.c_void_p(0x5000), ctypes.c_void_p(0x10000)

    def norm(a, kind=0, total=total, ws=ws, nbytes=1 << 30):
        return L.kd_grad_norm(*a, kind, total, ws, ctypes.c_size_t(nbytes), None)

    def clip(a, kind=0, total=total, limit=1.0, out=None, out_dtypes=None, to=None):
        return L.kd_grad_clip(*a, kind, total, limit, out, out_dtypes, to, None)
    for call in (norm, clip):
        assert call(lists(n=0)) == SHAPE and call(lists(n=K.GRADS_MAX + 1)) == SHAPE and call(lists(counts=(1, -1))) == SHAPE
        assert call(lists(counts=(1, (1 << 40) + 1))) == SHAPE and call(lists(counts=(1 << 40, 1 << 40))) == SHAPE
        assert call(lists(dtypes=(0, 2))) == PARAM and call(lists(at=(0x1000, None))) == NULL and call(lists(at=(0x1001, 0x2000))) == ALIGN
        assert call(lists(at=(0x1000, 0x2002))) == ALIGN and call(lists(), kind=2) == PARAM and call(lists(), total=None) == NULL
        assert call(lists(), total=ctypes.c_void_p(0x5004)) == ALIGN
        for i in (1, 2, 3):
            a = lists()
            a[i] = None
            assert call(a) == NULL
    assert norm(lists(), ws=None) == NULL and norm(lists(), ws=ctypes.c_void_p(0x10080)) == ALIGN and norm(lists(), nbytes=8) == WORKSPACE
    assert clip(lists(), limit=-1.0) == PARAM and clip(lists(), limit=float("nan")) == PARAM and clip(lists(), limit=float("inf")) == PARAM
    assert clip(lists(), to=ctypes.c_void_p(0x6002)) == ALIGN
    out, types = (ctypes.c_void_p * 2)(0x8000, 0x9000), (ctypes.c_int32 * 2)(1, 0)
    assert clip(lists(), out=out) == NULL and clip(lists(), out=out, out_dtypes=(ctypes.c_int32 * 2)(1, 7)) == PARAM
    assert clip(lists(), out=(ctypes.c_void_p * 2)(0x8000, None), out_dtypes=types) == NULL
    assert clip(lists(), out=(ctypes.c_void_p * 2)(0x8002, 0x9000), out_dtypes=types) == ALIGN
    assert clip(lists(), out=(ctypes.c_void_p * 2)(0x1000, 0x9000), out_dtypes=types) == PARAM       # in place, in another type
    n = ctypes.c_size_t(0)
    assert L.kd_grad_norm_workspace_size(2, (ctypes.c_int64 * 2)(1, 2), ctypes.byref(n)) == 0 and n.value > 0
    assert L.kd_grad_norm_workspace_size(0, (ctypes.c_int64 * 2)(1, 2), ctypes.byref(n)) == SHAPE
    assert L.kd_grad_norm_workspace_size(2, None, ctypes.byref(n)) == NULL and L.kd_grad_norm_workspace_size(2, (ctypes.c_int64 * 2)(1, 2), None) == NULL


def test_wrappers_refuse_what_the_library_cannot_see():
    z = torch.zeros(4, 100)
    for call in (lambda: K.quantize_e4m3_blocks(z), lambda: K.kd_top_logits(z, 5), lambda: K.kd_sample(z, torch.rand(4)),
                 lambda: K.kd_linear_e4m3(z, K.E4m3Blocks(z, z, K.BLOCK_TILE)), lambda: K.kd_clip_grad_norm([z], 1.0),
                 lambda: K.kd_clip_grad_norm([], 1.0), lambda: K.kd_clip_grad_norm([None], 1.0), lambda: K.GradList([z], [z, z]),
                 lambda: K.kd_matmul_e4m3(z, z), lambda: K.quantize_e4m3_blocks(torch.zeros(4)), lambda: K.GradList([3.0])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(TypeError):
        K.kd_loss_workspace_size(K.make_blocks_params(1, 1))

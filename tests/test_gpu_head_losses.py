"""The one-head losses on the GPU against the fp64 reference: sizes, types, orders, masks, lists, what a call may leave out, what
it must not read, captured and concurrent calls."""
import numpy as np
import pytest
import torch

from oracle import head_oracle as O
from paper_2603_01875_amd import autograd as A
from paper_2603_01875_amd import kdloss as K
from tests import head_util as U

pytestmark = pytest.mark.gpu

SIZES = [(1, 8, 8), (1, 64, 16), (2, 128, 1000), (3, 72, 264), (17, 192, 520), (63, 64, 4096), (64, 256, 2056), (65, 128, 1000),
         (128, 320, 1544), (129, 64, 776), (200, 520, 5000), (256, 128, 2048), (257, 192, 2056), (300, 136, 776), (520, 64, 4104),
         (1000, 128, 1288)]
TYPES = [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")]


def _labels(y, rng, T, share=0.2):
    y = y.clone()
    y[torch.from_numpy(rng.random(T) < share)] = -100
    if T > 1:
        y[T - 1] = -1
    return y


def _ce(case, seed, dtype="bf16", grad="bf16", layout="vh", smoothing=0.0, z_loss=0.0, chunk=0, scale=1.0, i32=False, masked=True):
    T, H, V = case
    h, W, y, rng = U.make(seed, T, H, V, dtype)
    if masked:
        y = _labels(y, rng, T)
    mask = (rng.random(T) < 0.8).astype(np.uint8) if masked and T > 8 else None
    ref = O.cross_entropy(U.np64(h), U.np64(W), y.numpy(), mask, smoothing, z_loss, scale)
    hd, Wd = U.device(h, W, layout)
    yd = (y.int() if i32 else y).cuda()
    md = None if mask is None else torch.from_numpy(mask).cuda()
    out = K.kd_ce_fwd_bwd(hd, Wd, yd, md, smoothing, z_loss, U.LAYOUT[layout], U.GRAD[grad], vocab_chunk=chunk, loss_scale=scale)
    fwd = K.kd_ce_fwd(hd, Wd, yd, md, smoothing, z_loss, U.LAYOUT[layout], loss_scale=scale)
    torch.cuda.synchronize()
    more = dict(tau=1.0, in_dtype=dtype, grad_dtype=grad, layout=layout, factor=scale, coefficient=1 + 64 * z_loss)
    U.check(out, ref, U.np64(h), U.np64(W), **more)
    U.check(fwd, ref, U.np64(h), U.np64(W), **more)
    return out


@pytest.mark.parametrize("case", SIZES)
@pytest.mark.parametrize("dtype,grad", TYPES)
def test_ce_sizes_and_types(case, dtype, grad):
    _ce(case, sum(case), dtype, grad)


@pytest.mark.parametrize("case", [(1, 64, 64), (70, 128, 1024), (300, 64, 2112), (130, 72, 264), (600, 192, 1000)])
@pytest.mark.parametrize("dtype,grad", TYPES)
def test_ce_heads_stored_hidden_major(case, dtype, grad):
    _ce(case, 7, dtype, grad, layout="hv")


@pytest.mark.parametrize("case", [(2, 64, 72), (100, 128, 1000), (300, 136, 2056)])
@pytest.mark.parametrize("layout", ["vh", "hv"])
@pytest.mark.parametrize("grad", ["bf16", "f32"])
@pytest.mark.parametrize("smoothing,z_loss", [(0.1, 0.0), (0.0, 0.01), (0.3, 0.001)])
def test_ce_smoothing_and_z_loss(case, layout, grad, smoothing, z_loss):
    _ce(case, 11, "bf16", grad, layout, smoothing, z_loss, scale=-1.5, i32=True)


@pytest.mark.parametrize("chunk", [256, 512, 1280])
@pytest.mark.parametrize("grad", ["bf16", "f32"])
def test_ce_chunks(chunk, grad):
    _ce((300, 128, 3000), 13, "bf16", grad, chunk=chunk, smoothing=0.1)
    _ce((70, 128, 3000), 14, "f32", grad, chunk=chunk)


def test_ce_every_token_counts():
    _ce((333, 64, 1000), 15, masked=False)


def _topk(case, k, tail, seed, dtype="bf16", grad="bf16", layout="vh", tau=1.0, chunk=0, flags=0, scale=1.0, ragged=True, top="f32",
          i32=False):
    T, H, V = case
    h, W, y, rng = U.make(seed, T, H, V, dtype)
    a, ids = U.top_lists(rng, T, V, k, y)
    if top == "bf16":
        a = a.bfloat16()
    lse = torch.from_numpy((np.log(np.exp(U.np64(a) / tau).sum(1)) - np.log(0.6 + 0.39 * rng.random(T))).astype(np.float32))
    mask = None
    if ragged and T > 4:
        mask = (rng.random(T) < 0.8).astype(np.uint8)
        gone = rng.random((T, k)) < 0.3
        ids[torch.from_numpy(gone)] = -1
        ids[1] = -7                                        # a token without entries
        a = a.float()
        a[2, 0] = -np.inf
        if k > 2:
            ids[3, 1] = ids[3, 0] if int(ids[3, 0]) >= 0 else 5
        a = a.bfloat16() if top == "bf16" else a
    ref = O.topk(U.np64(a), ids.numpy(), U.np64(h), U.np64(W), U.np64(lse), mask, tau, tail, scale, bool(flags & K.FLAG_TAU2))
    hd, Wd = U.device(h, W, layout)
    md = None if mask is None else torch.from_numpy(mask).cuda()
    args = (a.cuda(), (ids.int() if i32 else ids).cuda(), hd, Wd, None if tail == O.RENORM else lse.cuda(), md, tau, tail)
    out = K.kd_topk_fwd_bwd(*args, U.LAYOUT[layout], U.GRAD[grad], vocab_chunk=chunk, flags=flags, loss_scale=scale)
    fwd = K.kd_topk_fwd(*args, U.LAYOUT[layout], flags=flags, loss_scale=scale)
    torch.cuda.synchronize()
    # with the rest, what lies beside the list is scaled by r / (1 - P) in the gradient
    big = 1.0
    if tail == O.REST:
        p = np.exp(O.log_softmax(U.np64(h) @ U.np64(W).T / tau))
        on = np.zeros(p.shape, bool)
        for t in range(T):
            i = ids[t].numpy()
            on[t][i[(i >= 0) & np.isfinite(U.np64(a[t]))]] = True
        big = 2 + 1.0 / np.where(on, 0, p).sum(1).min()
    factor = scale * (tau * tau if flags & K.FLAG_TAU2 else 1.0)
    more = dict(tau=tau, in_dtype=dtype, grad_dtype=grad, layout=layout, factor=factor, coefficient=big)
    U.check(out, ref, U.np64(h), U.np64(W), **more)
    U.check(fwd, ref, U.np64(h), U.np64(W), **more)
    return out


@pytest.mark.parametrize("case,k", [((1, 64, 16), 1), ((5, 8, 8), 7), ((3, 72, 264), 40), ((64, 128, 2056), 8), ((100, 256, 1000), 64),
                                    ((257, 64, 4104), 33), ((300, 136, 776), 200), ((520, 192, 1544), 3), ((40, 64, 8000), 1024),
                                    ((260, 64, 1088), 1024)])
@pytest.mark.parametrize("tail", [O.RENORM, O.REST, O.DROP])
@pytest.mark.parametrize("dtype,grad", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
def test_topk_sizes_types_and_tails(case, k, tail, dtype, grad):
    _topk(case, k, tail, sum(case) + k, dtype, grad)


@pytest.mark.parametrize("case", [(70, 128, 1024), (300, 64, 2112), (130, 72, 264)])
@pytest.mark.parametrize("tail", [O.RENORM, O.REST])
def test_topk_heads_stored_hidden_major(case, tail):
    _topk(case, 16, tail, 3, layout="hv", tau=2.0, i32=True)


@pytest.mark.parametrize("tail", [O.RENORM, O.REST, O.DROP])
def test_topk_temperature_scale_chunks_and_types(tail):
    _topk((300, 128, 3000), 20, tail, 5, tau=0.7, chunk=512, flags=K.FLAG_TAU2, scale=0.25, top="bf16")
    _topk((90, 128, 3000), 20, tail, 6, tau=3.0, chunk=256, grad="f32", ragged=False)


def test_topk_whole_vocabulary_listed():
    _topk((20, 64, 264), 264, O.RENORM, 9, ragged=False)
    _topk((300, 64, 264), 263, O.REST, 10, ragged=False)


def test_topk_rest_where_the_student_is_sure():
    """The student's mass beside the list is 1e-8 and less: as a difference from 1 it would be gone."""
    T, H, V = 130, 64, 1000
    h, W, y, rng = U.make(21, T, H, V, "f32")
    W[:] = 0
    W[:, 0] = torch.linspace(-1, 1, V) * 0.1
    W[7, 1] = 1.0
    h[:] = 0
    h[:, 0] = torch.randn(T)
    h[:, 1] = torch.linspace(20, 40, T)
    a, ids = torch.zeros(T, 2), torch.tensor([[7, 3]]).repeat(T, 1)
    lse = torch.full((T,), float(np.log(2.0 / 0.9)))
    ref = O.topk(a.numpy(), ids.numpy(), U.np64(h), U.np64(W), U.np64(lse), tail=O.REST)
    out = K.kd_topk_fwd_bwd(a.cuda(), ids.cuda(), h.cuda(), W.cuda(), lse.cuda(), tail=K.TAIL_REST)
    np.testing.assert_allclose(U.np64(out["per_token_loss"]), ref["per_token_loss"], rtol=1e-5)
    np.testing.assert_allclose(U.np64(out["grad_h_s"]), ref["grad_h"], rtol=1e-4, atol=1e-9)
    np.testing.assert_allclose(U.np64(out["grad_W_s"]), ref["grad_W"], rtol=1e-4, atol=1e-7 * np.abs(ref["grad_W"]).max())


@pytest.mark.parametrize("T", [1, 5, 300])
def test_nothing_counts(T):
    h, W, y, _ = U.make(2, T, 64, 1000, "bf16")
    hd, Wd = U.device(h, W)
    gW = torch.full((1000, 64), 3.0, device="cuda", dtype=torch.bfloat16)
    none = torch.full((T,), -100, device="cuda")
    for out in (K.kd_ce_fwd_bwd(hd, Wd, none), K.kd_ce_fwd_bwd(hd, Wd, y.cuda(), torch.zeros(T, device="cuda", dtype=torch.uint8)),
                K.kd_topk_fwd_bwd(torch.zeros(T, 3, device="cuda"), none[:, None].repeat(1, 3), hd, Wd),
                K.kd_topk_fwd_bwd(torch.full((T, 3), -np.inf, device="cuda"), none[:, None].repeat(1, 3).abs(), hd, Wd)):
        assert float(out["loss"].item()) == 0
        for k, v in out.items():
            if k != "workspace":
                assert not v.any(), k
    out = K.kd_ce_fwd_bwd(hd, Wd, none, grad_W=gW, accumulate_grad_W=True)
    assert (gW == 3).all()


@pytest.mark.parametrize("T", [4, 70, 400])
def test_tokens_that_do_not_count_may_hold_anything(T):
    h, W, y, rng = U.make(3, T, 128, 1000, "bf16")
    y[1::3] = -100
    hd, Wd = U.device(h, W)
    clean = K.kd_ce_fwd_bwd(hd, Wd, y.cuda())
    hd[1::3] = float("nan")
    dirty = K.kd_ce_fwd_bwd(hd, Wd, y.cuda(), workspace=torch.full_like(clean["workspace"], 0xff))
    for k in ("loss", "per_token_loss", "grad_h", "grad_W"):
        assert torch.equal(clean[k], dirty[k]), k
    assert (dirty["grad_h"][1::3] == 0).all()


@pytest.mark.parametrize("T", [4, 300])
def test_rows_past_the_vocabulary_are_not_read_and_make_their_token_nan(T):
    h, W, y, _ = U.make(4, T, 64, 1000, "bf16")
    hd, Wd = U.device(h, W)
    for bad in (1000, 1 << 40):
        y[2] = bad
        out = K.kd_ce_fwd_bwd(hd, Wd, y.cuda())
        rows = out["per_token_loss"].isnan()
        assert rows[2] and int(rows.sum()) == 1 and out["loss"].isnan().all()
        assert out["grad_h"][2].isnan().all() and not out["grad_h"][[0, 1, 3]].isnan().any()
    ids = torch.arange(3).repeat(T, 1)
    ids[1, 1] = 1000
    a = torch.zeros(T, 3)
    a[3, 0] = float("nan")
    for tail in (K.TAIL_RENORM, K.TAIL_REST, K.TAIL_DROP):
        out = K.kd_topk_fwd_bwd(a.cuda(), ids.cuda(), hd, Wd, torch.full((T,), 2.0, device="cuda"), tail=tail)
        rows = out["per_token_loss"].isnan()
        assert rows[1] and rows[3] and int(rows.sum()) == 2
        assert out["grad_h_s"][1].isnan().all() and not out["grad_h_s"][[0, 2]].isnan().any()


def test_weights_of_infinity_in_rows_of_their_own():
    """-inf in a column of the head where every hidden state is positive: that row's probability is 0."""
    T, H, V = 300, 128, 1000
    h, W, y, _ = U.make(5, T, H, V, "bf16")
    h[:, 5] = h[:, 5].abs() + 1
    y[y == 9] = 10
    W2 = W.clone()
    W2[9, 5] = -float("inf")
    out = K.kd_ce_fwd_bwd(*U.device(h, W2), y.cuda())
    lp = U.np64(h) @ U.np64(W).T
    lp[:, 9] = -np.inf
    lp = lp - np.log(np.exp(lp - lp.max(1, keepdims=True)).sum(1, keepdims=True)) - lp.max(1, keepdims=True)
    np.testing.assert_allclose(U.np64(out["per_token_loss"]), -lp[np.arange(T), y.numpy()], rtol=1e-5)
    assert (out["grad_W"][9] == 0).all() and not out["grad_W"].isnan().any()


@pytest.mark.parametrize("T,chunk,layout", [(50, 0, "vh"), (50, 0, "hv"), (300, 0, "vh"), (300, 256, "vh"), (300, 256, "hv")])
@pytest.mark.parametrize("smoothing", [0.0, 0.1])
def test_probabilities_of_zero_where_the_target_is_not(T, chunk, layout, smoothing):
    """A logit of minus infinity that the target gives a probability: the loss is infinite, and dL/dz = p - q still holds."""
    H, V = 128, 1024
    h, W, y, _ = U.make(55, T, H, V, "bf16")
    h[:, 5] = h[:, 5].abs() + 1
    y[y == 9] = 10
    y[::4] = 9
    W_inf, W_low = W.clone(), W.clone()
    W_inf[9, 5], W_low[9, 5] = -float("inf"), -1e6
    out = K.kd_ce_fwd_bwd(*U.device(h, W_inf, layout), y.cuda(), None, smoothing, 0.0, U.LAYOUT[layout], K.F32, vocab_chunk=chunk,
                          want_grad_h=False)
    low = O.cross_entropy(U.np64(h), U.np64(W_low), y.numpy(), None, smoothing)
    rows = U.np64(out["per_token_loss"])
    infinite = np.ones(T, bool) if smoothing else y.numpy() == 9
    assert np.isposinf(rows[infinite]).all() and np.isposinf(out["loss"].item())
    W[9] = 0                                               # (the row is no logit's error; its share of p, below 1 %, is the 1.01)
    b = U.bounds(U.np64(h), U.np64(W), low, 1.0, "bf16", "f32")
    assert (np.abs(rows - low["per_token_loss"])[~infinite] <= 1.01 * b["rows"][~infinite] + 8 * U.F32 * 40).all()
    gW = U.np64(out["grad_W"] if layout == "vh" else out["grad_W"].T)
    assert (np.abs(gW - low["grad_W"]) <= 1.01 * b["grad_W"]).all()


@pytest.mark.parametrize("T", [50, 300])
@pytest.mark.parametrize("tail", [O.RENORM, O.DROP])
def test_entries_of_no_weight_add_nothing(T, tail):
    """Top logits of the type's lowest value: their probability is 0, also where the student's is."""
    H, V, k = 128, 1024, 6
    h, W, y, rng = U.make(56, T, H, V, "bf16")
    h[:, 5] = h[:, 5].abs() + 1
    W[9, 5] = -float("inf")
    a, ids = U.top_lists(rng, T, V, k, y)
    ids[ids == 9] = 11
    ids[:, 0], a[:, 0] = 9, torch.finfo(torch.float32).min
    lse = torch.zeros(T) + 3.0
    out = K.kd_topk_fwd_bwd(a.cuda(), ids.cuda(), *U.device(h, W), lse=None if tail == O.RENORM else lse.cuda(), tail=tail)
    W[9, 5] = -1e6
    ref = O.topk(U.np64(a), ids.numpy(), U.np64(h), U.np64(W), U.np64(lse), tail=tail)
    W[9] = 0
    b = U.bounds(U.np64(h), U.np64(W), ref, 1.0, "bf16", "bf16")
    assert (np.abs(U.np64(out["per_token_loss"]) - ref["per_token_loss"]) <= 1.01 * b["rows"] + 8 * U.F32 * 40).all()
    assert not out["grad_W_s"].isnan().any() and (out["grad_W_s"][9] == 0).all()


@pytest.mark.parametrize("T", [50, 300])
@pytest.mark.parametrize("grad", ["bf16", "f32"])
def test_gradients_one_at_a_time_and_added_up(T, grad):
    h, W, y, rng = U.make(6, T, 192, 2056, "bf16")
    y = _labels(y, rng, T)
    hd, Wd = U.device(h, W)
    kw = dict(grad_dtype=U.GRAD[grad])
    both = K.kd_ce_fwd_bwd(hd, Wd, y.cuda(), **kw)
    only_h = K.kd_ce_fwd_bwd(hd, Wd, y.cuda(), want_grad_W=False, **kw)
    only_W = K.kd_ce_fwd_bwd(hd, Wd, y.cuda(), want_grad_h=False, **kw)
    assert only_h["grad_W"] is None and only_W["grad_h"] is None
    assert torch.equal(only_h["grad_h"], both["grad_h"]) and torch.equal(only_W["grad_W"], both["grad_W"])
    assert torch.equal(only_h["loss"], both["loss"])
    there = torch.randn(2056, 192, device="cuda").to(both["grad_W"].dtype)
    added = there.clone()
    K.kd_ce_fwd_bwd(hd, Wd, y.cuda(), grad_W=added, accumulate_grad_W=True, **kw)
    # the product in fp32 is what the written one was rounded from
    half = U.BF16 if grad == "bf16" else U.F32
    want = there.double() + both["grad_W"].double()
    assert ((added.double() - want).abs() <= half * (want.abs() + both["grad_W"].double().abs()) * 1.01 + 1e-12).all()


def test_captured_calls_replay_bit_exactly():
    T, H, V = 300, 128, 2056
    h, W, y, rng = U.make(8, T, H, V, "bf16")
    a, ids = U.top_lists(rng, T, V, 12, y)
    hd, Wd = U.device(h, W)
    for T_ in (40, 300):
        x, yd, ad, idd = hd[:T_].contiguous(), _labels(y, rng, T)[:T_].cuda(), a[:T_].cuda(), ids[:T_].cuda()
        lse = torch.full((T_,), 6.0, device="cuda")
        p = K.make_ce_params(T_, H, V, 0.1, 1e-3, vocab_chunk=512)
        p2 = K.make_topk_params(T_, H, V, 12, tail=K.TAIL_REST, accumulate_grad_W=True)
        ws, ws2 = K.alloc_workspace(p), K.alloc_workspace(p2)
        o = dict(loss=torch.zeros(1, device="cuda"), ptl=torch.zeros(T_, device="cuda"), gh=torch.zeros_like(x), gW=torch.zeros_like(Wd),
                 loss2=torch.zeros(1, device="cuda"), ptl2=torch.zeros(T_, device="cuda"), gh2=torch.zeros_like(x))

        def call():
            K.kd_ce_fwd_bwd_raw(p, x, Wd, yd, None, o["loss"], o["ptl"], o["gh"], o["gW"], ws)
            K.kd_topk_fwd_bwd_raw(p2, ad, idd, lse, x, Wd, None, o["loss2"], o["ptl2"], o["gh2"], o["gW"], ws2)
        call()
        torch.cuda.synchronize()
        ref = {k: v.clone() for k, v in o.items()}
        assert all(v.any() for v in ref.values())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        for rep in range(3):
            for v in o.values():
                v.fill_(7)
            ws.fill_(0x5a)
            ws2.fill_(0xff)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            for k in ref:
                assert torch.equal(o[k], ref[k]), (rep, k)


def test_two_streams():
    probs = []
    for i, (T, H, V) in enumerate(((300, 128, 4104), (50, 256, 3000))):
        h, W, y, rng = U.make(30 + i, T, H, V, "bf16")
        a, ids = U.top_lists(rng, T, V, 9, y)
        probs.append((*U.device(h, W), y.cuda(), a.cuda(), ids.cuda()))

    def run(i):
        h, W, y, a, ids = probs[i]
        one, two = K.kd_ce_fwd_bwd(h, W, y), K.kd_topk_fwd_bwd(a, ids, h, W)
        return [one["loss"], one["grad_h"], one["grad_W"], two["per_token_loss"], two["grad_h_s"], two["grad_W_s"]]
    want = [run(i) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        got = []
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got.append(run(i))
        torch.cuda.synchronize()
        for a, b in zip(want, got):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_with_the_divergence_of_two_models_as_a_training_step_has_them():
    """The KD loss, the labels and the stored top logits of one student head: summed as torch scalars, and by adding to one
    gradient of the head; both are the sum of the references."""
    from oracle import kd_oracle as KD
    T, H, V = 300, 128, 2056
    h, W, y, rng = U.make(40, T, H, V, "f32")
    h_t, W_t, _, _ = U.make(41, T, 192, V, "f32")
    y = _labels(y, rng, T)
    a, ids = U.top_lists(rng, T, V, 16, y)
    n64 = [U.np64(x) for x in (h, W, h_t, W_t)]
    kd = KD.kd_loss_fwd_bwd(n64[2], n64[3], n64[0], n64[1], None, 1.0, 0, 0.5, KD.W_VH)
    ce = O.cross_entropy(n64[0], n64[1], y.numpy(), scale=0.3)
    tk = O.topk(U.np64(a), ids.numpy(), n64[0], n64[1], scale=0.2)
    want = {"loss": kd["loss"] + ce["loss"] + tk["loss"], "h": kd["grad_h_s"] + ce["grad_h"] + tk["grad_h"],
            "W": kd["grad_W_s"] + ce["grad_W"] + tk["grad_W"]}
    hd, Wd = U.device(h, W)
    hd.requires_grad_(True)
    Wd.requires_grad_(True)
    loss = (A.kd_loss(hd, Wd, h_t.cuda(), W_t.cuda()) + 0.3 * A.cross_entropy(hd, Wd, y.cuda())
            + A.topk_loss(hd, Wd, a.cuda(), ids.cuda(), loss_scale=0.2))
    loss.backward()
    assert abs(loss.item() - want["loss"]) < 1e-5 * want["loss"]
    # the two-model loss rounds dL/dz to bf16: 2^-8 of its own gradients' terms, here of its largest gradient
    for g, k in ((hd.grad, "h"), (Wd.grad, "W")):
        kd_g = kd["grad_h_s" if k == "h" else "grad_W_s"]
        assert np.abs(U.np64(g) - want[k]).max() <= 2e-2 * np.abs(kd_g).max() + 1e-5 * np.abs(want[k]).max()
    d = (hd.detach(), Wd.detach())
    gW = K.kd_loss_fwd_bwd(h_t.cuda(), W_t.cuda(), *d)["grad_W_s"]
    K.kd_ce_fwd_bwd(*d, y.cuda(), grad_W=gW, accumulate_grad_W=True, loss_scale=0.3)
    K.kd_topk_fwd_bwd(a.cuda(), ids.cuda(), *d, grad_W_s=gW, accumulate_grad_W=True, loss_scale=0.2)
    assert np.abs(U.np64(gW) - want["W"]).max() <= 2e-2 * np.abs(kd["grad_W_s"]).max() + 1e-5 * np.abs(want["W"]).max()


def test_autograd_asks_only_for_what_is_needed_and_its_slopes_are_the_losses():
    T, H, V = 90, 64, 1000
    h, W, y, rng = U.make(50, T, H, V, "f32", lean=2.0)
    a, ids = U.top_lists(rng, T, V, 8, y)
    lse = torch.logsumexp(a, 1) + 0.2
    hd, Wd, yd = *U.device(h, W), y.cuda()
    fns = {"ce": lambda h, W: A.cross_entropy(h, W, yd, label_smoothing=0.1, z_loss=1e-3),
           "topk": lambda h, W: A.topk_loss(h, W, a.cuda(), ids.cuda(), lse.cuda(), tau=2.0, tail=K.TAIL_REST, flags=K.FLAG_TAU2)}
    for f in fns.values():
        with torch.no_grad():
            plain = f(hd.requires_grad_(True), Wd)
        assert not plain.requires_grad
        x, w = hd.detach().requires_grad_(True), Wd.detach().requires_grad_(True)
        both = torch.autograd.grad(f(x, w), (x, w))
        assert torch.equal(torch.autograd.grad(f(x, w.detach()), x)[0], both[0])
        assert torch.equal(torch.autograd.grad(f(x.detach(), w), w)[0], both[1])
        assert f(x, w).item() == plain.item()
        # a central difference: the loss, of size 10, is good to 1e-6 and its third derivative along d small
        for base, g, along in ((x, both[0], lambda d: f(x.detach() + d, w.detach())), (w, both[1], lambda d: f(x.detach(), w.detach() + d))):
            d = g / g.norm()
            eps = 2e-2 * float(base.detach().norm()) / base.numel() ** 0.5
            slope = float(along(eps * d).double() - along(-eps * d).double()) / (2 * eps)
            assert slope == pytest.approx(float(g.norm()), rel=1e-2, abs=2e-6 / eps)


def test_a_head_whose_offsets_pass_32_bits():
    """V H elements past 2^31, and lists at its end."""
    T, H, V = 40, 8192, 270000
    g = torch.Generator(device="cuda").manual_seed(1)
    W = torch.empty(V, H, device="cuda", dtype=torch.bfloat16)
    for v0 in range(0, V, 32768):
        W[v0:v0 + 32768] = (torch.randn(min(32768, V - v0), H, device="cuda", generator=g) * 0.02).bfloat16()
    h = torch.randn(T, H, device="cuda", generator=g).bfloat16()
    y = torch.randint(V - 2000, V, (T,), device="cuda", generator=g)
    out = K.kd_ce_fwd_bwd(h, W, y)
    z = torch.cat([h.double() @ W[v0:v0 + 8192].double().t() for v0 in range(0, V, 8192)], 1)
    lp = torch.log_softmax(z, 1)
    want = -lp.gather(1, y[:, None])[:, 0]
    # an fp32 sum of 8192 products of size 0.02: 8192 2^-24 2^-6 8192^0.5 at most, twice
    assert ((out["per_token_loss"].double() - want).abs() <= 1e-3).all()
    dz = lp.exp()
    dz[torch.arange(T), y] -= 1
    for rows in (slice(0, 64), slice(V - 2000, V)):
        gW = dz[:, rows].t() @ h.double() / T
        bound = dz[:, rows].abs().t() @ h.double().abs() / T * (U.BF16 + 2e-3) + U.BF16 * gW.abs()
        assert ((out["grad_W"][rows].double() - gW).abs() <= bound).all()


@pytest.mark.parametrize("T", [31, 32, 33])
@pytest.mark.parametrize("layout", ["vh", "hv"])
def test_around_the_tokens_that_one_workgroup_merges(T, layout):
    _ce((T, 128, 1024), 60 + T, layout=layout, smoothing=0.05)
    _topk((T, 128, 1024), 70, O.REST, 60 + T, layout=layout)


def test_fp32_products_whose_partial_sums_would_be_too_many():
    """fp32 operands and gradients: six products of 2304 x 2560 sums are more than 128 MiB, so each adds to those in front of it."""
    T, H, V = 2304, 2560, 520
    h, W, y, rng = U.make(80, T, H, V, "f32", w_std=0.02)
    y = _labels(y, rng, T)
    ref = O.cross_entropy(U.np64(h), U.np64(W), y.numpy())
    out = K.kd_ce_fwd_bwd(*U.device(h, W), y.cuda())
    torch.cuda.synchronize()
    U.check(out, ref, U.np64(h), U.np64(W), in_dtype="f32", grad_dtype="f32")


@pytest.mark.parametrize("T,k", [(40, 7), (300, 70), (300, 300)])
@pytest.mark.parametrize("tail", [O.RENORM, O.REST, O.DROP])
def test_the_same_row_in_many_entries(T, k, tail):
    """Lists of three rows, and of one, each many times over; importance weights that do not add up to one."""
    H, V = 64, 520
    h, W, y, rng = U.make(90, T, H, V, "f32")
    a = torch.from_numpy(rng.standard_normal((T, k)).astype(np.float32))
    ids = torch.from_numpy(np.asarray([0, 255, V - 1])[rng.integers(0, 3, (T, k))])
    ids[::3] = 256
    lse = torch.from_numpy((np.log(np.exp(U.np64(a)).sum(1)) + (0.5 if tail == O.REST else -0.7)).astype(np.float32))
    ref = O.topk(U.np64(a), ids.numpy(), U.np64(h), U.np64(W), U.np64(lse), None, 1.0, tail)
    out = K.kd_topk_fwd_bwd(a.cuda(), ids.cuda(), *U.device(h, W), lse=None if tail == O.RENORM else lse.cuda(), tail=tail)
    torch.cuda.synchronize()
    p = np.exp(O.log_softmax(U.np64(h) @ U.np64(W).T))
    on = np.zeros((T, V), bool)
    np.put_along_axis(on, ids.numpy(), True, 1)
    # (DROP: the weights add up to 2; REST: beside the list, r / (1 - P))
    big = 2 + 1.0 / np.where(on, 0, p).sum(1).min() if tail == O.REST else 2.1
    U.check(out, ref, U.np64(h), U.np64(W), in_dtype="f32", grad_dtype="f32", coefficient=big)


@pytest.mark.parametrize("T", [20, 300])
def test_arrays_aligned_to_their_elements_only(T):
    """Labels, lists, masks (bool), and the losses' places need no more; what lies beside them stays."""
    H, V, k = 128, 1000, 9
    h, W, y, rng = U.make(91, T, H, V, "bf16")
    y = _labels(y, rng, T)
    a, ids = U.top_lists(rng, T, V, k, y.abs() % V)
    hd, Wd = U.device(h, W)
    mask = torch.from_numpy(rng.random(T) < 0.7)

    def odd(t, fill):
        whole = torch.full((t.numel() + 2,), fill, dtype=t.dtype, device="cuda")
        whole[1:-1] = t.flatten().cuda()
        return whole[1:-1].view(t.shape)
    for itype, ttype in ((torch.int32, torch.bfloat16), (torch.int64, torch.float32)):
        want = K.kd_ce_fwd_bwd(hd, Wd, y.to(itype).cuda(), mask.cuda().to(torch.uint8))
        ytop = (a.to(ttype), ids.to(itype))
        want2 = K.kd_topk_fwd_bwd(*(t.cuda() for t in ytop), hd, Wd, mask=mask.cuda())
        got = K.kd_ce_fwd_bwd(hd, Wd, odd(y.to(itype), 3), odd(mask, True))
        got2 = K.kd_topk_fwd_bwd(odd(ytop[0], 99.0), odd(ytop[1], 3), hd, Wd, mask=odd(mask, True))
        for w, g in ((want, got), (want2, got2)):
            for n in w:
                assert n == "workspace" or torch.equal(w[n], g[n]), n
        p = K.make_ce_params(T, H, V, index_dtype=K.I32 if itype == torch.int32 else K.I64)
        places = torch.full((T + 4,), 5.0, device="cuda")
        K.kd_ce_fwd_raw(p, hd, Wd, y.to(itype).cuda(), mask.cuda(), places[1:2], places[3:3 + T], K.alloc_workspace(p))
        assert torch.equal(places[1:2], want["loss"]) and torch.equal(places[3:3 + T], want["per_token_loss"])
        assert (places[[0, 2, T + 3]] == 5).all()


def test_two_graphs_that_share_a_workspace():
    """Captured one after the other on one workspace and replayed in turn, in both orders, with eager calls between."""
    H, V = 128, 2056
    h, W, y, rng = U.make(92, 300, H, V, "bf16")
    a, ids = U.top_lists(rng, 300, V, 12, y)
    hd, Wd = U.device(h, W)
    ws = torch.empty(max(K.kd_loss_workspace_size(K.make_ce_params(300, H, V)), K.kd_loss_workspace_size(K.make_topk_params(50, H, V, 12))),
                     dtype=torch.uint8, device="cuda")
    calls = [lambda: K.kd_ce_fwd_bwd(hd, Wd, yd, workspace=ws),
             lambda: K.kd_topk_fwd_bwd(ad, idd, xd, Wd, workspace=ws)]
    yd, ad, idd, xd = y.cuda(), a[:50].cuda(), ids[:50].cuda(), hd[:50].contiguous()
    want, graphs, outs = [], [], []
    for call in calls:
        want.append({k: v.clone() for k, v in call().items() if k != "workspace"})
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(call())
        graphs.append(g)
    for order in ((0, 1), (1, 0), (0, 0, 1, 1)):
        for i in order:
            graphs[i].replay()
        calls[order[0]]()
        torch.cuda.synchronize()
        for i in (0, 1):
            assert all(torch.equal(outs[i][k], want[i][k]) for k in want[i]), (order, i)
            for k in want[i]:
                outs[i][k].fill_(3)


@pytest.mark.parametrize("T,H,V,k", [(1, 64, 264, 3), (64, 64, 1000, 5), (65, 72, 1000, 70), (128, 128, 2056, 9), (129, 128, 776, 9),
                                     (300, 136, 1544, 33)])
@pytest.mark.parametrize("dtype,layout", [("bf16", "vh"), ("f32", "vh"), ("bf16", "hv")])
def test_nothing_beside_the_buffers_is_written(T, H, V, k, dtype, layout):
    h, W, y, rng = U.make(93, T, H, V, dtype)
    a, ids = U.top_lists(rng, T, V, k, y)
    hd, Wd = U.device(h, W, layout)
    ids, a, y = ids.cuda(), a.cuda(), y.cuda()
    kw = dict(in_dtype=K.BF16 if dtype == "bf16" else K.F32, w_layout=U.LAYOUT[layout])
    for chunk in (0, 256):
        calls = [(K.make_ce_params(T, H, V, 0.1, vocab_chunk=chunk, **kw),
                  lambda p, o: K.kd_ce_fwd_bwd_raw(p, hd, Wd, y, None, *o)),
                 (K.make_topk_params(T, H, V, k, vocab_chunk=chunk, **kw),
                  lambda p, o: K.kd_topk_fwd_bwd_raw(p, a, ids, None, hd, Wd, None, *o))]
        for p, call in calls:
            es = hd.element_size()
            sizes = [4, 4 * T, es * T * H, es * V * H, K.kd_loss_workspace_size(p)]
            at = [4096]
            for n in sizes:
                at.append((at[-1] + n + 4096 + 255) // 256 * 256)
            whole = torch.full((at[-1],), 0x5a, dtype=torch.uint8, device="cuda")
            part = [whole[b:b + n] for b, n in zip(at, sizes)]
            types = [torch.float32, torch.float32, hd.dtype, hd.dtype, torch.uint8]
            call(p, [x.view(t) for x, t in zip(part, types)])
            torch.cuda.synchronize()
            for x in part[:4]:
                assert not (x == 0x5a).all()
            for x in part:
                x.fill_(0x5a)
            assert (whole == 0x5a).all()

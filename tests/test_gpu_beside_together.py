"""The calls beside the losses as a program uses them: one after the other up to a loss and clipped gradients, from a captured graph, on two streams
at once, and on arrays of more than 2^31 elements."""
import numpy as np
import pytest
import torch

from oracle import head_oracle
from paper_2603_01875_amd import autograd as A
from paper_2603_01875_amd import kdloss as K
from tests import head_util as HU
from tests.test_gpu_blocks import check_product, reference
from tests.test_gpu_rows import check_tokens, check_top

pytestmark = pytest.mark.gpu


def np64(t):
    return t.detach().cpu().double().numpy()


def randn(seed, *shape, scale=1.0, dtype=torch.bfloat16):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(*shape, generator=g) * scale).to(dtype).cuda()


def test_a_step_of_distillation():
    """Teacher's layer and logits in e4m3, its top logits as targets, the student's layer in e4m3, the loss, then all gradients clipped:
    each stage against what its inputs, as they are on the device, say in 64 bits."""
    T, H, V, k, tau = 70, 256, 1504, 24, 2.0
    teacher, head = randn(1, T, H), K.quantize_e4m3_blocks(randn(2, V, H, scale=0.06), K.BLOCK_TILE)
    logits = K.kd_linear_e4m3(teacher, head)
    a = K.quantize_e4m3_blocks(teacher)
    assert torch.equal(logits, K.kd_matmul_e4m3(a, head))
    top = K.kd_top_logits(logits, k, tau)
    check_top(logits, k, tau, top)

    x, W1 = randn(3, T, H).requires_grad_(), randn(4, H, H, scale=0.06).requires_grad_()
    W2 = randn(5, V, H, scale=0.06).requires_grad_()
    h = A.linear_e4m3(x, W1)
    loss = A.topk_loss(h, W2, **top, tau=tau, tail=K.TAIL_REST)
    gh, gW2 = torch.autograd.grad(loss, (h, W2), retain_graph=True)
    ref = head_oracle.topk(np64(top["top_logits"]), top["top_index"].cpu().numpy(), np64(h), np64(W2), np64(top["lse"]), tau=tau, tail=K.TAIL_REST)
    out = K.kd_topk_fwd_bwd(**{n: top[n] for n in ("top_logits", "top_index")}, h_s=h.detach(), W_s=W2.detach(), lse=top["lse"], tau=tau,
                            tail=K.TAIL_REST)
    HU.check(out, ref, np64(h), np64(W2), tau)
    assert torch.equal(gh, out["grad_h_s"]) and torch.equal(gW2, out["grad_W_s"]) and loss.item() == out["loss"].item()
    grads = torch.autograd.grad(loss, (x, W1, W2))
    q, qt = K.quantize_e4m3_blocks(gh, both=True)
    assert torch.equal(grads[0], K.kd_matmul_e4m3(q, K.quantize_e4m3_blocks(W1.detach(), K.BLOCK_TILE, transpose=True)))
    assert torch.equal(grads[1], K.kd_matmul_e4m3(qt, K.quantize_e4m3_blocks(x.detach(), transpose=True)))
    assert torch.equal(grads[2], gW2)

    before = [g.clone() for g in grads]
    norm = np.sqrt(sum((np64(g) ** 2).sum() for g in grads))
    limit = float(np.float32(0.37 * norm))
    got = K.kd_clip_grad_norm(list(grads), limit)
    assert abs(got.item() - norm) <= 2.0 ** -23 * norm
    for g, b in zip(grads, before):                         # the factor is rounded to fp32, the product to fp32 and to bf16
        want = np64(b) * (limit / norm)
        assert (np.abs(np64(g) - want) <= (2.0 ** -8 + 3 * 2.0 ** -24) * np.abs(want) + 1e-40).all()


def test_tokens_of_a_student_and_their_cross_entropy():
    """Logits of a layer in e4m3, tokens drawn from them, the cross entropy of these tokens and its gradients, clipped."""
    T, H, V = 40, 128, 3000
    h, W = randn(11, T, H, dtype=torch.float32), randn(12, V, H, scale=0.3, dtype=torch.float32)
    logits = K.kd_linear_e4m3(h, K.quantize_e4m3_blocks(W, K.BLOCK_TILE))
    u = torch.rand(T, generator=torch.Generator().manual_seed(13)).cuda()
    settings = dict(temperature=0.8, top_k=50, top_p=0.9)
    got = K.kd_sample(logits, u, **settings)
    check_tokens(logits, u, settings, got, T - 1)
    out = K.kd_ce_fwd_bwd(h, W, got["token"], grad_dtype=K.F32)
    ref = head_oracle.cross_entropy(np64(h), np64(W), got["token"].cpu().numpy())
    HU.check(out, ref, np64(h), np64(W), in_dtype="f32", grad_dtype="f32")
    norm = np.sqrt((np64(out["grad_h"]) ** 2).sum() + (np64(out["grad_W"]) ** 2).sum())
    assert abs(K.kd_clip_grad_norm([out["grad_h"], out["grad_W"]], 1e9).item() - norm) <= 2.0 ** -23 * norm


SHAPES = [(3, 200, 1000, 8), (70, 2100, 5000, 64), (300, 520, 33_000, 200)]


def everything(T, H, V, k, x, W, u, max_norm=0.5):
    """All calls in a row; what they give, in one list."""
    w = K.quantize_e4m3_blocks(W, K.BLOCK_TILE)
    z = K.kd_linear_e4m3(x, w, out_dtype=K.F32)
    top = K.kd_top_logits(z, k, 2.0)
    draws = [K.kd_sample(z, u), K.kd_sample(z, u, 0.7, top_k=k), K.kd_sample(z, u, 1.3, top_p=0.8), K.kd_sample(z, u, 1.0, min_p=0.01)]
    xg, Wg = x.detach().requires_grad_(), W.detach().requires_grad_()
    gx, gW = torch.autograd.grad(A.linear_e4m3(xg, Wg), (xg, Wg), z.to(x.dtype))
    norm = K.kd_clip_grad_norm([gx, gW], max_norm)
    return [z, *top.values(), *(v for d in draws for v in d.values()), gx, gW, norm]


@pytest.mark.parametrize("T,H,V,k", SHAPES)
def test_captured_and_replayed(T, H, V, k):
    x, W, u = randn(21, T, H), randn(22, V, H, scale=0.1), torch.rand(T, generator=torch.Generator().manual_seed(23)).cuda()
    inputs = [(randn(30 + i, T, H), torch.rand(T, generator=torch.Generator().manual_seed(40 + i)).cuda()) for i in range(3)]
    want = [[t.clone() for t in everything(T, H, V, k, xi, W, ui)] for xi, ui in inputs]
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = everything(T, H, V, k, x, W, u)
    for i in (0, 1, 2, 1):
        x.copy_(inputs[i][0])
        u.copy_(inputs[i][1])
        torch.cuda.synchronize()
        everything(T, H, V, k, x, W, u)              # eager work between the replays
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want[i]))


def test_two_graphs_share_their_workspaces():
    """Each graph writes what it reads of a workspace: what the other one, or anyone, left there does not matter."""
    T, H, V, k = 70, 2100, 5000, 64
    W = K.quantize_e4m3_blocks(randn(52, V, H, scale=0.1), K.BLOCK_TILE)
    lp, tp, sp = K.make_linear_params(T, V, H, K.BF16, K.F32), K.make_top_logits_params(T, V, k, in_dtype=K.F32), \
        K.make_sample_params(T, V, top_p=0.8, in_dtype=K.F32)
    ws = torch.empty(max(K.alloc_workspace(p).numel() for p in (lp, tp, sp)) + 256, dtype=torch.uint8, device="cuda")

    def calls(x, u):
        z = K.kd_linear_e4m3(x, W, out_dtype=K.F32, workspace=ws)
        top, draw = K.kd_top_logits(z, k, workspace=ws), K.kd_sample(z, u, top_p=0.8, workspace=ws)
        norm = K.kd_clip_grad_norm(K.GradList([z], [torch.empty_like(z)]), 1.0, workspace=ws) if ws.numel() >= K.GradList([z]).workspace_bytes else z
        return [z, *top.values(), *draw.values(), norm]
    xs = [randn(53 + i, T, H) for i in range(2)]
    us = [torch.rand(T, generator=torch.Generator().manual_seed(55 + i)).cuda() for i in range(2)]
    want = [[t.clone() for t in calls(x, u)] for x, u in zip(xs, us)]
    torch.cuda.synchronize()
    graphs, got = [], []
    for x, u in zip(xs, us):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            got.append(calls(x, u))
        graphs.append(g)
    for i in (0, 1, 1, 0, 1, 0):
        ws.fill_(0xff if i else 0x3c)
        graphs[i].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got[i], want[i]))


def test_two_streams_at_once():
    T, H, V, k = 70, 2100, 5000, 64
    sets = [(randn(61 + i, T, H), randn(63 + i, V, H, scale=0.1), torch.rand(T, generator=torch.Generator().manual_seed(65 + i)).cuda())
            for i in range(2)]
    want = [[t.clone() for t in everything(T, H, V, k, *s)] for s in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    for _ in range(3):
        got = []
        for s, st in zip(sets, streams):
            with torch.cuda.stream(st):
                got.append(everything(T, H, V, k, *s))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for x, y in zip(got, want) for a, b in zip(x, y))


def test_raw_calls_take_the_stream_that_they_are_given():
    T, H, V = 33, 256, 700
    x, w = randn(71, T, H), K.quantize_e4m3_blocks(randn(72, V, H), K.BLOCK_TILE)
    p = K.make_linear_params(T, V, H)
    out, ws = torch.zeros(T, V, dtype=torch.bfloat16, device="cuda"), K.alloc_workspace(p)
    want = K.kd_linear_e4m3(x, w)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    K.kd_linear_e4m3_raw(p, x, w, out, ws, stream=s.cuda_stream)
    s.synchronize()
    assert torch.equal(out, want)


# ---- more than 2^31 elements ----
def test_a_store_of_logits_behind_two_to_the_31():
    T, V = 14_500, 151_936
    z = torch.empty(T, V, dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(3))
    u = torch.rand(T, generator=torch.Generator().manual_seed(4)).cuda()
    last = slice(T - 5, T)
    for settings in (dict(), dict(top_k=40), dict(top_p=0.7)):
        whole, part = K.kd_sample(z, u, **settings), K.kd_sample(z[last].clone(), u[last].clone(), **settings)
        assert all(torch.equal(whole[n][last], part[n]) for n in part)
    whole, part = K.kd_top_logits(z, 16), K.kd_top_logits(z[last].clone(), 16)
    assert torch.equal(whole["top_index"][last], part["top_index"]) and torch.equal(whole["top_logits"][last], part["top_logits"])
    check_top(z[last], 16, 1.0, {n: whole[n][last] for n in whole})


def test_matrices_behind_two_to_the_31():
    M, H = 530_000, 4096
    x = torch.empty(M, H, dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(5))
    q, qt = K.quantize_e4m3_blocks(x, both=True)
    last = slice(M // 128 * 128 - 128, M)
    r, rt = K.quantize_e4m3_blocks(x[last].clone(), both=True)
    assert torch.equal(q.codes[last], r.codes) and torch.equal(q.scales[last], r.scales)
    assert torch.equal(qt.codes[:, last], rt.codes[:, :M - last.start]) and torch.equal(qt.scales[:, last.start // 128:], rt.scales)
    w = K.quantize_e4m3_blocks(randn(6, 4100, H), K.BLOCK_TILE)
    y = K.kd_matmul_e4m3(q, w)                          # 2.2e9 results
    check_product(y[last], *reference(r, w, H, True), H, "bf16")
    # the long axis contracted: 64 rows of x^T against themselves
    few = K.E4m3Blocks(qt.codes[:64].contiguous(), qt.scales[:64].contiguous(), K.BLOCK_ROW)
    g = np64(K.kd_matmul_e4m3(few, qt, out_dtype=K.F32))
    part = x[:, :64].double()
    ref = np64(part.t().contiguous() @ part)
    # each code is off by up to 2^-4 of its value: a sum of M products of normal numbers, at random, by 6 standard deviations of 2^-4 sqrt(2 M)
    assert (np.abs(g[:, :64] - ref) <= 2.0 ** -4 * np.abs(ref) * np.eye(64) + 6 * 2.0 ** -4 * np.sqrt(2 * M)).all()


def test_a_gradient_of_more_than_two_to_the_31_elements():
    n = (1 << 31) + 4097
    g = torch.full((n,), 2.0 ** -10, dtype=torch.bfloat16, device="cuda")
    g[n - 1] = 64.0
    norm = np.sqrt((n - 1) * 2.0 ** -20 + 4096.0)
    got = K.kd_clip_grad_norm([g], float(np.float32(norm / 2)))
    assert abs(got.item() - norm) <= 2.0 ** -23 * norm
    f = np.float32(norm / 2) / norm
    assert abs(g[n - 1].item() - 64 * f) <= 2.0 ** -7 * 64 and bool((g[:-1] == g[0]).all()) and abs(g[0].item() - 2.0 ** -10 * f) <= 2.0 ** -18


def test_most_rows_that_a_matrix_may_have():
    rows, cols = 1 << 24, 1040
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator("cuda").manual_seed(7))
    q, r = K.quantize_e4m3_blocks(x), K.quantize_e4m3_blocks(x[-300:].clone())
    assert torch.equal(q.codes[-300:], r.codes) and torch.equal(q.scales[-300:], r.scales)

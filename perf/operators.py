"""The losses over one output head: softmax cross entropy with labels, and distillation from a teacher's top
logits.  Both take the student's hidden states and its head and never hold a [T, V] array of logits that a
caller would see; a pass is one call of a training step (loss and both gradients), of an evaluation (loss and
per-token losses alone), or two micro-batches whose head gradients add up.

Fields of a case
  op        "ce"       K.kd_ce_*: labels, label smoothing, a penalty on the log-sum-exp
            "topk"     K.kd_topk_*: the teacher's K largest logits and their vocabulary entries per token
  entry     "step"     loss, per-token losses, both gradients
            "eval"     loss and per-token losses
            "micro"    (ce) two micro-batches, the second adding to the head's gradient, each weighted by one half
  T, H, V   tokens, hidden size, vocabulary;  K: top logits per token (topk)
  dtype, grad          "bf16" / "f32" operands, gradients
  layout               "vh" / "hv" storage order of the head
  smoothing, z_loss    (ce)
  tau, tail            (topk) temperature; "renorm": the top logits are the whole distribution, "rest": what the
                       teacher has beside them is one more category, "drop": it is left out
  count                which tokens count: "all", "tail25" (padded ends of four sequences), "prompt" (the first part
                       of each sequence is not learned from), "random10"
"""
import math

import numpy as np
import torch

own = False

V_QWEN, V_LLAMA = 151936, 128256
SHARE = {"all": 1.0, "tail25": 0.875, "prompt": 0.75, "random10": 0.9}      # of the tokens, in the mean


def _case(name, op, entry, T, H, V, K=0, dtype="bf16", grad="bf16", layout="vh", smoothing=0.0, z_loss=0.0, tau=1.0,
          tail="renorm", count="all"):
    return dict(name=name, op=op, entry=entry, T=T, H=H, V=V, K=K, dtype=dtype, grad=grad, layout=layout,
                smoothing=smoothing, z_loss=z_loss, tau=tau, tail=tail, count=count)


def listed():
    return [
        # what a user tries first, in fp32: launches and latency decide
        _case("ce_tiny_f32", "ce", "step", 128, 128, 4096, dtype="f32", grad="f32"),
        # the log-probability of one sampled token, as generation reports it: the head is read once
        _case("ce_one_token", "ce", "eval", 1, 1024, V_QWEN),
        # scoring a short answer
        _case("ce_short_answer", "ce", "eval", 48, 2048, V_LLAMA, count="random10"),
        # a micro-batch of one short sequence
        _case("ce_short_sequence", "ce", "step", 200, 2048, V_QWEN, count="prompt"),
        # supervised step of 4 x 1024 tokens, padded ends
        _case("ce_step", "ce", "step", 4096, 1024, V_QWEN, count="tail25"),
        # a head kept as [H, V], smoothed labels, the log-sum-exp held down
        _case("ce_smooth_hv", "ce", "step", 2048, 1024, V_QWEN, layout="hv", smoothing=0.1, z_loss=1e-4, count="prompt"),
        # two odd micro-batches, fp32 gradients that add up
        _case("ce_micro_odd", "ce", "micro", 777, 1000, 50264, grad="f32", smoothing=0.05, count="random10"),
        # a wide student on a long batch
        _case("ce_wide", "ce", "step", 8192, 4096, V_LLAMA, count="tail25"),
        # a small fp32 student on eight logits per token
        _case("topk_small_f32", "topk", "step", 250, 256, 8000, K=8, dtype="f32", grad="f32", tau=2.0, tail="rest"),
        # one short sequence per step
        _case("topk_short_sequence", "topk", "step", 100, 1024, V_QWEN, K=32, tau=2.0, tail="renorm"),
        # the distillation step from 64 stored logits per token, the teacher's rest as one category
        _case("topk_step", "topk", "step", 4096, 1024, V_QWEN, K=64, tail="rest", count="tail25"),
        # evaluation of a ragged batch
        _case("topk_eval", "topk", "eval", 1003, 2048, V_LLAMA, K=20, tail="rest", count="random10"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: sizes spread over their logarithm and mostly odd, every entry point, order and type, no costlier
    than the largest listed one."""
    most = work(_case("", "ce", "step", 8192, 4096, V_LLAMA))["flops"]
    while True:
        op = rng.choice(["ce", "topk"])
        entry = rng.choice(["step", "step", "eval", "micro"] if op == "ce" else ["step", "step", "eval"])
        T = _log_int(rng, 1, 8192)
        V = rng.choice([V_QWEN, V_LLAMA, 8 * _log_int(rng, 500, 19000)])
        H = 64 * _log_int(rng, 2, 64)
        dtype, grad, layout = "bf16", rng.choice(["bf16", "bf16", "bf16", "f32"]), "vh"
        r = rng.random()
        if r < 0.2:
            layout = "hv"
        elif r < 0.45:      # hidden sizes off the 64-element grid, or fp32 operands: small problems
            H, T, V = 8 * _log_int(rng, 8, 200), min(T, 2048), min(V, 50264)
            if rng.random() < 0.5:
                dtype, grad, T, V = "f32", "f32", min(T, 1024), min(V, 32000)
        c = _case("", op, entry, T, H, V, dtype=dtype, grad=grad, layout=layout, count=rng.choice(list(SHARE)))
        del c["name"]
        if op == "ce":
            c["smoothing"], c["z_loss"] = rng.choice([0.0, 0.0, 0.1]), rng.choice([0.0, 0.0, 1e-4])
        else:
            c["K"] = _log_int(rng, 1, 256)
            c["tau"], c["tail"] = rng.choice([1.0, 1.0, 2.0]), rng.choice(["renorm", "rest", "rest", "drop"])
        if work(c)["flops"] <= most:
            return c


def _counts(case, g):
    """Which tokens count, on the device; the first always does."""
    T, kind = case["T"], case["count"]
    if kind == "all":
        return torch.ones(T, dtype=torch.bool, device="cuda")
    if kind == "random10":
        m = torch.rand(T, device="cuda", generator=g) >= 0.1
    else:
        n = max(T // 4, 1)
        where = torch.arange(T, device="cuda")
        cut = torch.rand((T + n - 1) // n, device="cuda", generator=g)[where // n]
        m = where % n < n * (1 - cut / 4) if kind == "tail25" else where % n >= n * cut / 2
    m[0] = True
    return m


def prepare(case, seed):
    """Operands on the device: RMS-normalised hidden states (bf16) that lean towards their token's row of the head, so
    that its logit stands up to 16 above the others', as a partly trained student's does; Gaussian heads."""
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    T, H, V, K = case["T"], case["H"], case["V"], case["K"]
    dt = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    W = torch.empty(V, H, device="cuda", dtype=dt)
    for v0 in range(0, V, 32768):
        n = min(32768, V - v0)
        W[v0:v0 + n] = (torch.randn(n, H, device="cuda", generator=g) * 0.02).to(dt)
    parts = []
    for _ in range(2 if case["entry"] == "micro" else 1):
        keep = _counts(case, g)
        token = (V * torch.rand(T, device="cuda", generator=g).pow(3)).long().clamp(0, V - 1)      # frequent ones are frequent
        lean = (torch.rand(T, 1, device="cuda", generator=g) * 16 / (0.02 * H)).clamp(max=0.9)
        row = torch.nn.functional.normalize(W[token].float(), dim=1) * math.sqrt(H)
        h = torch.randn(T, H, device="cuda", generator=g) * (1 - lean * lean).sqrt() + lean * row
        if case["dtype"] == "bf16":
            h = h / h.pow(2).mean(1, keepdim=True).sqrt()
        p = dict(h=h.to(dt))
        if case["op"] == "ce":
            p["labels"] = torch.where(keep, token, torch.full_like(token, -100))
        else:
            # the token itself and others spread over the vocabulary, all different; logits that fall off with the rank
            step = 1 + 2 * (torch.rand(T, 1, device="cuda", generator=g) * ((V // K - 1) // 2)).long()
            rank = torch.arange(K, device="cuda")
            p["index"] = (token[:, None] + rank * step) % V
            z = 14 + 2 * torch.randn(T, 1, device="cuda", generator=g) - 2 * torch.log1p(rank.float())
            z = z + 0.3 * torch.randn(T, K, device="cuda", generator=g)
            p["logits"] = torch.sort(z, 1, descending=True).values.contiguous()
            held = 0.7 + 0.29 * torch.rand(T, device="cuda", generator=g)            # what the top logits hold of the whole
            p["lse"] = torch.logsumexp(p["logits"] / case["tau"], 1) - torch.log(held)
            short = torch.rand(T, 1, device="cuda", generator=g) < 0.2               # some lists are shorter than K
            p["index"] = torch.where(short & (rank >= max(K // 2, 1)), torch.full_like(p["index"], -1), p["index"])
            p["mask"] = keep.to(torch.uint8)
        parts.append(p)
    return dict(case=case, W=W if case["layout"] == "vh" else W.t().contiguous(), parts=parts)


# ------------------------------------------------------------------------------------------------
# the plain form, in 32 bits
# ------------------------------------------------------------------------------------------------
def _logits(c, h, W):
    return h.float() @ (W.float().t() if c["layout"] == "vh" else W.float())


def _gradients(c, dz, h, W):
    gh = dz @ (W.float() if c["layout"] == "vh" else W.float().t())
    gW = dz.t() @ h.float() if c["layout"] == "vh" else h.float().t() @ dz
    return gh, gW


def _plain_ce(c, p, W, scale):
    """(loss, per-token losses, both gradients in 32 bits, or None)."""
    keep = p["labels"] >= 0
    n = keep.sum().clamp(min=1)
    y = p["labels"].clamp(min=0)[:, None]
    z = _logits(c, p["h"], W)
    top = z.max(1, keepdim=True).values
    lse = top + torch.log((z - top).exp().sum(1, keepdim=True))
    eps = c["smoothing"]
    rows = lse - (1 - eps) * z.gather(1, y) - eps * z.mean(1, keepdim=True) + c["z_loss"] * lse * lse
    rows = torch.where(keep, scale * rows[:, 0], torch.zeros_like(rows[:, 0]))
    loss = (rows.sum() / n).reshape(1)
    if c["entry"] == "eval":
        return loss, rows, None, None
    dz = (z - lse).exp_() * (1 + 2 * c["z_loss"] * lse) - eps / c["V"]
    dz.scatter_add_(1, y, torch.full_like(lse, eps - 1))
    dz *= torch.where(keep, scale / n, torch.zeros_like(rows))[:, None]
    return (loss, rows) + _gradients(c, dz, p["h"], W)


def _plain_topk(c, p, W, scale):
    tau, there = c["tau"], p["index"] >= 0
    keep = (p["mask"] != 0) & there.any(1)
    n = keep.sum().clamp(min=1)
    at = p["index"].clamp(min=0)
    a = (p["logits"] / tau).masked_fill(~there, -math.inf)
    lse_t = torch.logsumexp(a, 1, keepdim=True) if c["tail"] == "renorm" else p["lse"][:, None]
    q = (a - lse_t).exp()
    held = q.sum(1, keepdim=True)
    z = _logits(c, p["h"], W) / tau
    top = z.max(1, keepdim=True).values
    lse = top + torch.log((z - top).exp().sum(1, keepdim=True))
    rows = torch.where(there, q * ((a - lse_t) - (z.gather(1, at) - lse)), torch.zeros_like(q)).sum(1, keepdim=True)
    listed_ = torch.zeros_like(z).scatter_add_(1, at, there.float()) > 0
    inside, outside = held, held
    if c["tail"] == "rest":
        rest = (1 - held).clamp(min=0)
        lse_out = top + torch.log((z - top).exp().masked_fill(listed_, 0).sum(1, keepdim=True))
        rows = rows + torch.where(rest > 0, rest * (torch.log(rest) - (lse_out - lse)), torch.zeros_like(rest))
        inside = held + rest
        outside = inside - rest * (lse - lse_out).exp()
    rows = torch.where(keep, scale * rows[:, 0], torch.zeros_like(rows[:, 0]))
    loss = (rows.sum() / n).reshape(1)
    if c["entry"] == "eval":
        return loss, rows, None, None
    dz = (z - lse).exp_() * torch.where(listed_, inside, outside)
    dz.scatter_add_(1, at, -q)
    dz *= torch.where(keep, scale / (n * tau), torch.zeros_like(rows))[:, None]
    return (loss, rows) + _gradients(c, dz, p["h"], W)


def _plain(st):
    c, W = st["case"], st["W"]
    plain = _plain_ce if c["op"] == "ce" else _plain_topk
    to = torch.float32 if c["grad"] == "f32" else torch.bfloat16
    loss, rows, gh, gW = plain(c, st["parts"][0], W, 0.5 if c["entry"] == "micro" else 1.0)
    if c["entry"] == "eval":
        return dict(loss=loss, ptl=rows)
    out = dict(loss=loss, ptl=rows, grad_h=gh.to(to))
    if c["entry"] == "micro":
        loss2, rows2, gh2, gW2 = plain(c, st["parts"][1], W, 0.5)
        if to is torch.float32:
            gW = gW + gW2
        else:
            gW = gW.to(to).float() + gW2                   # what a bf16 gradient holds between two micro-batches
        out.update(loss2=loss2, ptl2=rows2, grad_h2=gh2.to(to))
    out["grad_W"] = gW.to(to)
    return out


# ------------------------------------------------------------------------------------------------
# the framework's calls
# ------------------------------------------------------------------------------------------------
def _kept(st):
    """Parameters, outputs and workspace that a training program makes once and keeps."""
    if "params" in st:
        return
    from paper_2603_01875_amd import kdloss as K
    c = st["case"]
    T, H, V = c["T"], c["H"], c["V"]
    kw = dict(in_dtype=K.F32 if c["dtype"] == "f32" else K.BF16, grad_dtype=K.F32 if c["grad"] == "f32" else K.BF16,
              w_layout=K.W_VH if c["layout"] == "vh" else K.W_HV)
    if c["op"] == "ce":
        kw.update(label_smoothing=c["smoothing"], z_loss=c["z_loss"], loss_scale=0.5 if c["entry"] == "micro" else 1.0)
        st["params"] = K.make_ce_params(T, H, V, **kw)
        st["params2"] = K.make_ce_params(T, H, V, accumulate_grad_W=True, **kw)
    else:
        tail = {"renorm": K.TAIL_RENORM, "rest": K.TAIL_REST, "drop": K.TAIL_DROP}[c["tail"]]
        st["params"] = K.make_topk_params(T, H, V, c["K"], tau=c["tau"], tail=tail, **kw)
    st["ws"] = K.alloc_workspace(st["params"])
    to = torch.float32 if c["grad"] == "f32" else torch.bfloat16
    for k in ("", "2")[:len(st["parts"])]:
        st["loss" + k] = torch.empty(1, device="cuda")
        st["ptl" + k] = torch.empty(T, device="cuda")
        st["grad_h" + k] = torch.empty(T, H, device="cuda", dtype=to)
    st["grad_W"] = torch.empty_like(st["W"], dtype=to)


def _own(st):
    from paper_2603_01875_amd import kdloss as K
    _kept(st)
    c, p, W, ws = st["case"], st["parts"][0], st["W"], st["ws"]
    loss, ptl, gh, gW = st["loss"], st["ptl"], st["grad_h"], st["grad_W"]
    if c["op"] == "topk":
        lse = None if c["tail"] == "renorm" else p["lse"]
        if c["entry"] == "eval":
            K.kd_topk_fwd_raw(st["params"], p["logits"], p["index"], lse, p["h"], W, p["mask"], loss, ptl, ws)
            return dict(loss=loss, ptl=ptl)
        K.kd_topk_fwd_bwd_raw(st["params"], p["logits"], p["index"], lse, p["h"], W, p["mask"], loss, ptl, gh, gW, ws)
        return dict(loss=loss, ptl=ptl, grad_h=gh, grad_W=gW)
    if c["entry"] == "eval":
        K.kd_ce_fwd_raw(st["params"], p["h"], W, p["labels"], None, loss, ptl, ws)
        return dict(loss=loss, ptl=ptl)
    K.kd_ce_fwd_bwd_raw(st["params"], p["h"], W, p["labels"], None, loss, ptl, gh, gW, ws)
    out = dict(loss=loss, ptl=ptl, grad_h=gh, grad_W=gW)
    if c["entry"] == "micro":
        p2 = st["parts"][1]
        K.kd_ce_fwd_bwd_raw(st["params2"], p2["h"], W, p2["labels"], None, st["loss2"], st["ptl2"], st["grad_h2"], gW, ws)
        out.update(loss2=st["loss2"], ptl2=st["ptl2"], grad_h2=st["grad_h2"])
    return out


def run(st):
    return _own(st) if own else _plain(st)


def work(case):
    """Each operand read once and each result written once; 2 flop per multiply-add of the logits and of the two
    backward products, on the tokens that count (in the mean over the masks)."""
    T, H, V, K = case["T"], case["H"], case["V"], case["K"]
    n = max(T * SHARE[case["count"]], 1.0)
    es, gs = (4 if case["dtype"] == "f32" else 2), (4 if case["grad"] == "f32" else 2)
    passes = 2 if case["entry"] == "micro" else 1
    target = T * 8 if case["op"] == "ce" else n * (K * 12 + 4) + T
    nbytes = V * H * es + passes * (n * H * es + target + T * 4)
    flops = 2.0 * passes * n * V * H
    if case["entry"] != "eval":
        nbytes += V * H * gs + passes * T * H * gs
        flops *= 3.0
    return {"bytes": float(nbytes), "flops": float(flops)}


# ------------------------------------------------------------------------------------------------
# the definition in 64 bits, a block of tokens at a time
# ------------------------------------------------------------------------------------------------
def _target(case, p, s, V):
    """Teacher probabilities of a block as a dense array, and what lies beside the listed entries (None: nothing)."""
    ids = p["index"][s].cpu().numpy()
    a = p["logits"][s].double().cpu().numpy() / case["tau"]
    a[ids < 0] = -np.inf
    full = a.max(1, keepdims=True)
    full = np.where(np.isfinite(full), full, 0.0)
    norm = full + np.log(np.exp(a - full).sum(1, keepdims=True)) if case["tail"] == "renorm" else p["lse"][s].double().cpu().numpy()[:, None]
    q = torch.from_numpy(np.exp(a - norm)).cuda()
    at = torch.from_numpy(np.maximum(ids, 0)).cuda()
    dense = torch.zeros(q.shape[0], V, device="cuda", dtype=torch.float64).scatter_add_(1, at, q)
    member = torch.zeros(q.shape[0], V, device="cuda", dtype=torch.float64).scatter_add_(1, at, (q > 0).double()) > 0
    rest = (1 - q.sum(1)).clamp(min=0) if case["tail"] == "rest" else None
    return dense, member, rest


def _exact_part(case, p, W, scale):
    T, V = case["T"], W.shape[0]
    if case["op"] == "ce":
        keep, div = p["labels"] >= 0, 1.0
    else:
        keep, div = (p["mask"] != 0) & (p["index"] >= 0).any(1), case["tau"]
    n = max(int(keep.sum()), 1)
    rows = torch.zeros(T, device="cuda", dtype=torch.float64)
    back = case["entry"] != "eval"
    gh = torch.zeros(T, W.shape[1], device="cuda", dtype=torch.float64) if back else None
    gW = torch.zeros_like(W) if back else None
    for t0 in range(0, T, 1024):
        s = slice(t0, min(t0 + 1024, T))
        h = p["h"][s].double()
        lp = torch.log_softmax(h @ W.t() / div, 1)
        prob = lp.exp()
        if case["op"] == "ce":
            q = torch.full_like(lp, case["smoothing"] / V)
            q[torch.arange(q.shape[0], device="cuda"), p["labels"][s].clamp(min=0)] += 1 - case["smoothing"]
            lse = (h * W[0]).sum(1) - lp[:, 0]
            rows[s] = -(q * lp).sum(1) + case["z_loss"] * lse ** 2
            dz = prob - q + 2 * case["z_loss"] * lse[:, None] * prob
        else:
            q, member, rest = _target(case, p, s, V)
            rows[s] = torch.special.xlogy(q, q).sum(1) - (q * lp).sum(1)
            dz = prob * q.sum(1, keepdim=True) - q
            if rest is not None:
                out = prob.masked_fill(member, 0)
                log_out = torch.log(out.sum(1))
                rows[s] += torch.special.xlogy(rest, rest) - rest * log_out
                dz += rest[:, None] * (prob - out / out.sum(1, keepdim=True))
        rows[s] = torch.where(keep[s], scale * rows[s], torch.zeros_like(rows[s]))
        if back:
            dz = torch.where(keep[s][:, None], dz * (scale / (n * div)), torch.zeros_like(dz))
            gh[s] = dz @ W
            gW += dz.t() @ h
    return (rows.sum() / n).reshape(1), rows, gh, gW


def exact(case, seed):
    st = prepare(case, seed)
    hv = case["layout"] == "hv"
    W = (st["W"].t() if hv else st["W"]).double().contiguous()
    scale = 0.5 if case["entry"] == "micro" else 1.0
    got = [_exact_part(case, p, W, scale) for p in st["parts"]]
    out = dict(loss=got[0][0], ptl=got[0][1])
    if case["entry"] == "eval":
        return out
    gW = got[0][3] if len(got) == 1 else got[0][3] + got[1][3]
    out.update(grad_h=got[0][2], grad_W=gW.t().contiguous() if hv else gW)
    if case["entry"] == "micro":
        out.update(loss2=got[1][0], ptl2=got[1][1], grad_h2=got[1][2])
    return out

"""What a distillation program calls before and behind the losses: the linear layer in e4m3 with a scale per block of
128, the top logits of a teacher and tokens sampled from a student, and the norm of all gradients with clipping.  A pass is
one call as such a program makes it.

Fields of a case, by `op`
  "linear"  y = x W^T, both in e4m3.  entry "fwd": K.kd_linear_e4m3, x in bf16 or fp32, quantised in the call (a scale per token
            and 128 hidden columns), W quantised before (a scale per 128 x 128).  "step": autograd.linear_e4m3, forward and both
            gradients, W quantised in the call, gradients of the result in blocks of 128 outputs, and for grad_W both factors in
            blocks of 128 tokens.  T, H, V: tokens, inputs, outputs;  dtype: of x (and W, "step");  out: of y and the gradients
  "sample"  K.kd_sample: one token per row of logits, by the first of temperature, top-k, top-p, min-p that a program sets, from
            one given uniform number.  T, V, dtype;  filters "none", "top_k", "top_p", "min_p", "all" (one setting for the
            batch) or "rows" (each row its own, some greedy);  layout "plain", "padded" (rows longer than V), "masked" (a part
            of the vocabulary is at minus infinity)
  "top"     K.kd_top_logits: the K largest logits of a row, their places, the row's log-sum-exp.  T, V, K, tau, dtype, layout
  "clip"    K.kd_clip_grad_norm over n tensors of N elements in all, dtype "bf16", "f32" or "mixed".  entry "copy": the clipped
            gradients go to arrays of their own (type out);  "in_place": the norm is below its limit, as it is in most steps
"""
import math

import numpy as np
import torch

own = False

V_QWEN, V_LLAMA = 151936, 128256
MAX_E4M3 = 448.0
LEAST = 448 * 2.0 ** -126      # of a block's largest magnitude


def listed():
    return [
        # a projection of eight tokens: launches and latency decide
        dict(name="linear_small", op="linear", entry="fwd", T=8, H=1024, V=1024, dtype="bf16", out="bf16"),
        # the teacher's head for one generated token: the head is read once
        dict(name="linear_one_token_head", op="linear", entry="fwd", T=1, H=4096, V=V_QWEN, dtype="bf16", out="f32"),
        # a ragged batch through an odd layer
        dict(name="linear_ragged", op="linear", entry="fwd", T=777, H=1000, V=5003, dtype="f32", out="f32"),
        # a training step of a square projection
        dict(name="linear_step", op="linear", entry="step", T=4096, H=4096, V=4096, dtype="bf16", out="bf16"),
        # a micro-batch of teacher logits
        dict(name="linear_logits", op="linear", entry="fwd", T=4096, H=4096, V=V_QWEN, dtype="bf16", out="bf16"),
        # the next token of one sequence
        dict(name="sample_one", op="sample", T=1, V=V_QWEN, dtype="bf16", filters="all", layout="plain"),
        # a serving batch, each request with its own settings
        dict(name="sample_batch", op="sample", T=64, V=V_LLAMA, dtype="f32", filters="rows", layout="masked"),
        # on-policy rollouts: the student's own distribution
        dict(name="sample_rollouts", op="sample", T=512, V=V_QWEN, dtype="bf16", filters="none", layout="plain"),
        # a short answer scored by a small teacher
        dict(name="top_short", op="top", T=7, V=32003, K=20, tau=1.0, dtype="f32", layout="plain"),
        # what a step's distillation targets are stored from
        dict(name="top_store", op="top", T=4096, V=V_QWEN, K=64, tau=2.0, dtype="bf16", layout="plain"),
        # a small fp32 student: launches and latency
        dict(name="clip_small", op="clip", entry="copy", n=24, N=3_200_000, dtype="f32", out="f32"),
        # all gradients of a student of 1.7 billion weights
        dict(name="clip_model", op="clip", entry="copy", n=311, N=1_700_000_000, dtype="bf16", out="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: sizes spread over their logarithm and mostly odd, every entry, type and setting, no costlier than the
    largest listed one of its operator."""
    most = {c["op"]: work(c) for c in listed()}
    for c in listed():
        most[c["op"]] = {k: max(v, work(c)[k]) for k, v in most[c["op"]].items()}
    while True:
        op = rng.choice(["linear", "linear", "sample", "sample", "top", "clip"])
        V = rng.choice([V_QWEN, V_LLAMA, _log_int(rng, 1000, 200000)])
        dtype = rng.choice(["bf16", "f32"])
        layout = rng.choice(["plain", "plain", "padded", "masked"])
        if op == "linear":
            entry = rng.choice(["fwd", "fwd", "step"])
            T, H = _log_int(rng, 1, 8192), 8 * _log_int(rng, 16, 1024)
            V = rng.choice([V, 8 * _log_int(rng, 16, 2048), _log_int(rng, 128, 16384)])
            if entry == "step":
                V = min(V, 16384)
            c = dict(op=op, entry=entry, T=T, H=H, V=V, dtype=dtype, out=dtype if entry == "step" else rng.choice(["bf16", "f32"]))
        elif op == "sample":
            c = dict(op=op, T=_log_int(rng, 1, 512), V=V, dtype=dtype,
                     filters=rng.choice(["none", "top_k", "top_p", "min_p", "all", "rows", "rows"]), layout=layout)
        elif op == "top":
            c = dict(op=op, T=_log_int(rng, 1, 4096), V=V, K=_log_int(rng, 1, 256), tau=rng.choice([1.0, 2.0]), dtype=dtype,
                     layout=layout)
        else:
            c = dict(op=op, entry=rng.choice(["copy", "copy", "in_place"]), n=_log_int(rng, 1, 400),
                     N=_log_int(rng, 20000, 1_700_000_000), dtype=rng.choice(["bf16", "f32", "mixed"]), out="bf16")
            c["out"] = c["dtype"] if c["entry"] == "in_place" else rng.choice(["bf16", "f32"])
        w = work(c)
        if all(w[k] <= most[op][k] for k in w):
            return c


def _type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------
def _prepare_linear(c, g):
    T, H, V = c["T"], c["H"], c["V"]
    # hidden states as they leave a norm: some columns many times as large as the others
    big = 1 + 15 * (torch.rand(H, device="cuda", generator=g) < 0.01)
    x = (torch.randn(T, H, device="cuda", generator=g) * big).to(_type(c["dtype"]))
    W = torch.randn(V, H, device="cuda", generator=g) * 0.02
    if c["entry"] == "step":
        dy = torch.randn(T, V, device="cuda", generator=g) * (1e-3 * torch.rand(T, 1, device="cuda", generator=g))
        return dict(x=x, W=W.to(_type(c["dtype"])), dy=dy.to(_type(c["dtype"])))
    codes, scales = _blocks_of_weights(W)                    # the quantised layer that such a program loads and keeps
    room = -H % 16
    codes = torch.nn.functional.pad(codes, (0, room)) if room else codes
    return dict(x=x, codes=codes.contiguous(), scales=scales.contiguous())


def _blocks_of_weights(W):
    """e4m3 codes (bytes) of [V, H] weights and the scale of each 128 x 128."""
    V, H = W.shape
    full = torch.nn.functional.pad(W, (0, -H % 128, 0, -V % 128))
    tiles = full.view(full.shape[0] // 128, 128, full.shape[1] // 128, 128)
    top = tiles.abs().amax((1, 3), keepdim=True).clamp(min=LEAST)
    codes = _codes(tiles, top).view(torch.uint8)
    return codes.view(full.shape)[:V, :H], (top / torch.full_like(top, MAX_E4M3))[:, 0, :, 0]


def _codes(x, top):
    """e4m3 of 448 x / top, from 32 bits: one rounding in front of e4m3's (7 x has three bits more than x)."""
    return (x * 0.4375 / top * 1024).to(torch.float8_e4m3fn)


def _prepare_logits(c, g):
    """Logits of a language model: some thousands of entries stand out, falling off with their rank, over a wide rest."""
    T, V = c["T"], c["V"]
    ld = (V + 63) // 64 * 64 + 64 if c["layout"] == "padded" else V
    z = torch.empty(T, ld, device="cuda", dtype=_type(c["dtype"]))
    rank = torch.arange(min(V // 2, 2000), device="cuda")
    for t0 in range(0, T, 512):
        n = min(512, T - t0)
        y = torch.randn(n, ld, device="cuda", generator=g) * (1 + 2 * torch.rand(n, 1, device="cuda", generator=g))
        at = (torch.rand(n, 1, device="cuda", generator=g) * V).long()
        step = 1 + 2 * (torch.rand(n, 1, device="cuda", generator=g) * (V // (2 * rank.numel()) - 1)).long().clamp(min=0)
        peak = 6 + 12 * torch.rand(n, 1, device="cuda", generator=g) - 2 * torch.log1p(rank.float())
        y.scatter_add_(1, (at + rank * step) % V, peak.clamp(min=0))
        if c["layout"] == "masked":
            y = y.masked_fill(torch.rand(1, ld, device="cuda", generator=g) < 0.3, -math.inf)
        z[t0:t0 + n] = y.to(z.dtype)
    return z[:, :V]


def _pick(values, T, g, dtype):
    v = torch.tensor(values, device="cuda", dtype=dtype)
    return v[torch.randint(0, len(values), (T,), device="cuda", generator=g)]


def _prepare_sample(c, g):
    T = c["T"]
    st = dict(z=_prepare_logits(c, g), u=torch.rand(T, device="cuda", generator=g))
    one = dict(none=(1.0, 0, 1.0, 0.0), top_k=(0.8, 50, 1.0, 0.0), top_p=(1.0, 0, 0.95, 0.0), min_p=(1.2, 0, 1.0, 0.05),
               all=(0.7, 40, 0.9, 0.02)).get(c["filters"])
    if one is None:
        st["settings"] = dict(temperature=_pick([0.0, 0.6, 0.7, 1.0, 1.0, 1.5], T, g, torch.float32),
                              top_k=_pick([0, 0, 1, 20, 50, 1000], T, g, torch.int32),
                              top_p=_pick([1.0, 1.0, 0.8, 0.9, 0.95, 0.99], T, g, torch.float32),
                              min_p=_pick([0.0, 0.0, 0.0, 0.02, 0.1], T, g, torch.float32))
    else:
        st["settings"] = dict(zip(("temperature", "top_k", "top_p", "min_p"), one))
    return st


def _sizes(n, N):
    """Elements of n tensors, N together: a few large ones, many of the middle, some short."""
    share = np.array([(i * 7919 % 97 + 1) ** 2 for i in range(n)], float)
    size = np.maximum(1, (share / share.sum() * N).astype(np.int64))
    size[0] += N - size.sum()
    return size.tolist()


def _prepare_clip(c, g):
    """Gradients as views of one array per type, as a program keeps them that reduces them over ranks in large pieces."""
    sizes = _sizes(c["n"], c["N"])
    types = [torch.float32 if c["dtype"] == "f32" or (c["dtype"] == "mixed" and i % 4 == 3) else torch.bfloat16 for i in range(len(sizes))]
    flat, parts = {}, []
    for t in (torch.bfloat16, torch.float32):
        total = sum(s for s, x in zip(sizes, types) if x is t)
        if total:
            flat[str(t)] = torch.empty(total, device="cuda", dtype=t)
            for i in range(0, total, 1 << 28):
                n = min(1 << 28, total - i)
                flat[str(t)][i:i + n] = (torch.randn(n, device="cuda", generator=g) * 1e-3).to(t)
    at = dict.fromkeys(flat, 0)
    for s, t in zip(sizes, types):
        parts.append(flat[str(t)][at[str(t)]:at[str(t)] + s])
        at[str(t)] += s
    st = dict(flat=flat, parts=parts, max_norm=1.0 if c["entry"] == "copy" else 1e6)
    if c["entry"] == "copy":
        st["max_norm"] = 0.37e-3 * math.sqrt(c["N"])         # a third of the norm or so
        to = _type(c["out"])
        st["copy"] = {k: torch.zeros_like(v, dtype=to) for k, v in flat.items()}
        at, st["copies"] = dict.fromkeys(flat, 0), []
        for s, t in zip(sizes, types):
            st["copies"].append(st["copy"][str(t)][at[str(t)]:at[str(t)] + s])
            at[str(t)] += s
    return st


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    if case["op"] == "linear":
        st = _prepare_linear(case, g)
    elif case["op"] == "clip":
        st = _prepare_clip(case, g)
    elif case["op"] == "sample":
        st = _prepare_sample(case, g)
    else:
        st = dict(z=_prepare_logits(case, g))
    st["case"] = case
    return st


# ------------------------------------------------------------------------------------------------
# the plain form
# ------------------------------------------------------------------------------------------------
def _rows_quantised(x):
    """[R, C] in 32 bits -> what its e4m3 codes stand for, a scale per row and 128 columns."""
    R, C = x.shape
    full = torch.nn.functional.pad(x, (0, -C % 128)) if C % 128 else x
    b = full.reshape(R, -1, 128)
    top = b.abs().amax(2, keepdim=True).clamp(min=LEAST)
    return (_codes(b, top).float() * (top / torch.full_like(top, MAX_E4M3))).reshape(R, -1)[:, :C]


def _tiles_value(codes, scales):
    V, H = codes.shape
    s = scales.repeat_interleave(128, 0)[:V].repeat_interleave(128, 1)[:, :H]
    return codes.view(torch.float8_e4m3fn).float() * s


def _plain_linear(st):
    c, to = st["case"], _type(st["case"]["out"])
    x = st["x"].float()
    if c["entry"] == "fwd":
        return dict(y=(_rows_quantised(x) @ _tiles_value(st["codes"][:, :c["H"]], st["scales"]).t()).to(to))
    W = _tiles_value(*_blocks_of_weights(st["W"].float()))
    dy = st["dy"].float()
    y = _rows_quantised(x) @ W.t()
    gx = _rows_quantised(dy) @ W
    gW = _rows_quantised(dy.t().contiguous()) @ _rows_quantised(x.t().contiguous()).t()
    return dict(y=y.to(to), grad_x=gx.to(to), grad_W=gW.to(to))


def _column(v, like):
    return v.to(like.dtype)[:, None] if isinstance(v, torch.Tensor) else torch.full_like(like[:, :1], v)


def _plain_sample(st):
    """In 64 bits: a token's place in the running sum is what a uniform number is compared with."""
    z, s = st["z"].double(), st["settings"]
    temperature, top_k, top_p, min_p = (_column(s[k], z) for k in ("temperature", "top_k", "top_p", "min_p"))
    if not isinstance(s["temperature"], torch.Tensor):       # (the settings are 32-bit numbers)
        temperature, top_p, min_p = temperature.float().double(), top_p.float().double(), min_p.float().double()
    greedy = temperature == 0
    top_k = torch.where(top_k == 0, torch.full_like(top_k, z.shape[1]), top_k)
    top_k = torch.where(greedy, torch.ones_like(top_k), top_k)
    z = z / torch.where(greedy, torch.ones_like(temperature), temperature)
    w = (z - z.amax(1, keepdim=True)).exp()
    if st["case"]["filters"] != "none":
        sorted_, order = torch.sort(z, dim=1, descending=True, stable=True)
        ws = w.gather(1, order)
        inside = torch.arange(z.shape[1], device=z.device) < top_k
        ws = torch.where(inside, ws, torch.zeros_like(ws))
        run_ = ws.cumsum(1)
        keep = inside & (run_ - ws < top_p * run_[:, -1:]) & (ws >= min_p)
        w = torch.zeros_like(w).scatter_(1, order, torch.where(keep, ws, torch.zeros_like(ws)))
    cdf = w.cumsum(1)
    total = cdf[:, -1:]
    token = (cdf <= st["u"].double()[:, None] * total).sum(1, keepdim=True)
    return dict(token=token[:, 0], logp=(w.gather(1, token) / total).log()[:, 0].float())


def _plain_top(st):
    c = st["case"]
    top, at = torch.sort(st["z"], dim=1, descending=True, stable=True)
    y = st["z"].float() / c["tau"]
    m = y.amax(1, keepdim=True)
    lse = m + (y - m).exp().sum(1, keepdim=True).log()
    there = top[:, :c["K"]] > -math.inf
    return dict(logits=top[:, :c["K"]], index=torch.where(there, at[:, :c["K"]], -1), lse=lse[:, 0])


def _plain_clip(st):
    norm = sum(x.float().square().sum(dtype=torch.float64) for x in st["flat"].values()).sqrt()
    factor = (st["max_norm"] / norm).clamp(max=1.0).float()
    to = st.get("copy", st["flat"])
    return dict(norm=norm.float(), grads={k: (x.float() * factor).to(to[k].dtype) for k, x in st["flat"].items()})


# ------------------------------------------------------------------------------------------------
# the framework's calls
# ------------------------------------------------------------------------------------------------
def _own_linear(st):
    from paper_2603_01875_amd import autograd as A
    from paper_2603_01875_amd import kdloss as K
    c = st["case"]
    if c["entry"] == "step":
        x, W = st["x"].requires_grad_(), st["W"].requires_grad_()
        y = A.linear_e4m3(x, W)
        gx, gW = torch.autograd.grad(y, (x, W), st["dy"])
        return dict(y=y.detach(), grad_x=gx, grad_W=gW)
    if "weights" not in st:                                  # what the program keeps beside the layer
        st["weights"] = K.E4m3Blocks(st["codes"], st["scales"], K.BLOCK_TILE)
        st["params"] = K.make_linear_params(c["T"], c["V"], c["H"], in_dtype=K.F32 if c["dtype"] == "f32" else K.BF16,
                                            out_dtype=K.F32 if c["out"] == "f32" else K.BF16)
        st["ws"] = K.alloc_workspace(st["params"])
        st["y"] = torch.empty(c["T"], c["V"], device="cuda", dtype=_type(c["out"]))
    K.kd_linear_e4m3_raw(st["params"], st["x"], st["weights"], st["y"], st["ws"])
    return dict(y=st["y"])


def _own_sample(st):
    from paper_2603_01875_amd import kdloss as K
    c, s = st["case"], st["settings"]
    if "params" not in st:
        rows = isinstance(s["temperature"], torch.Tensor)
        one = {} if rows else s
        st["params"] = K.make_sample_params(c["T"], c["V"], ld=st["z"].stride(0), in_dtype=K.F32 if c["dtype"] == "f32" else K.BF16, **one)
        st["rows"] = s if rows else {}
        st["ws"] = K.alloc_workspace(st["params"])
        st["token"] = torch.empty(c["T"], device="cuda", dtype=torch.int64)
        st["logp"] = torch.empty(c["T"], device="cuda")
    K.kd_sample_raw(st["params"], st["z"], st["u"], st["token"], st["logp"], st["ws"], **st["rows"])
    return dict(token=st["token"], logp=st["logp"])


def _own_top(st):
    from paper_2603_01875_amd import kdloss as K
    c = st["case"]
    if "params" not in st:
        st["params"] = K.make_top_logits_params(c["T"], c["V"], c["K"], ld=st["z"].stride(0), tau=c["tau"],
                                                in_dtype=K.F32 if c["dtype"] == "f32" else K.BF16)
        st["ws"] = K.alloc_workspace(st["params"])
        st["top"] = torch.empty(c["T"], c["K"], device="cuda", dtype=st["z"].dtype)
        st["index"] = torch.empty(c["T"], c["K"], device="cuda", dtype=torch.int64)
        st["lse"] = torch.empty(c["T"], device="cuda")
    K.kd_top_logits_raw(st["params"], st["z"], st["top"], st["index"], st["lse"], st["ws"])
    return dict(logits=st["top"], index=st["index"], lse=st["lse"])


def _own_clip(st):
    from paper_2603_01875_amd import kdloss as K
    if "list" not in st:
        st["list"] = K.GradList(st["parts"], out=st.get("copies"))
    norm = K.kd_clip_grad_norm(st["list"], st["max_norm"])
    return dict(norm=norm, grads=st.get("copy", st["flat"]))


def run(st):
    op = st["case"]["op"]
    if own:
        return dict(linear=_own_linear, sample=_own_sample, top=_own_top, clip=_own_clip)[op](st)
    return dict(linear=_plain_linear, sample=_plain_sample, top=_plain_top, clip=_plain_clip)[op](st)


def work(case):
    """Each input read once and each output written once; 2 flop per multiply-add of the products, a handful per logit."""
    size = dict(bf16=2.0, f32=4.0)
    if case["op"] == "linear":
        T, H, V, es, os_ = case["T"], case["H"], case["V"], size[case["dtype"]], size[case["out"]]
        if case["entry"] == "step":
            return {"bytes": (T * H + V * H + T * V) * (es + os_), "flops": 6.0 * T * H * V}
        return {"bytes": T * H * es + V * H * (1 + 4 / 16384) + T * V * os_, "flops": 2.0 * T * H * V}
    if case["op"] == "clip":
        es = dict(size, mixed=2.5)[case["dtype"]]
        return {"bytes": case["N"] * (es + (size[case["out"]] if case["entry"] == "copy" else 0.0)), "flops": 3.0 * case["N"]}
    T, V, es = case["T"], case["V"], size[case["dtype"]]
    if case["op"] == "sample":
        return {"bytes": T * (V * es + 4.0 + 12.0), "flops": 4.0 * T * V}
    return {"bytes": T * (V * es + case["K"] * (es + 8.0) + 4.0), "flops": 4.0 * T * V}


# ------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ------------------------------------------------------------------------------------------------
def _e4m3(v):
    """Nearest number with four significant bits, exponent -6 or more; ties to even, at most 448."""
    a = v.abs()
    unit = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -6))) - 3)
    unit = torch.where(a >= 16 * unit, 2 * unit, torch.where(a < 8 * unit, unit / 2, unit)).clamp(min=2.0 ** -9)    # (log2's last bit)
    return torch.sign(v) * (torch.round(a / unit) * unit).clamp(max=MAX_E4M3)


def _exact_blocks(x, rows):
    """x (64 bits) through e4m3, a scale per block of `rows` x 128."""
    R, C = x.shape
    out = torch.empty_like(x)
    for j in range(0, C, 128):
        b = x[:, j:j + 128]
        top = b.abs().amax(1)
        if rows > 1:
            top = torch.cat([t.amax().expand(t.numel()) for t in top.split(rows)])
        top = top.clamp(min=LEAST)[:, None]
        out[:, j:j + 128] = _e4m3(b * MAX_E4M3 / top) * (top / MAX_E4M3)
    return out


def _exact_linear(case, st):
    H = case["H"]
    x = st["x"].double()
    if case["entry"] == "fwd":
        xq = _exact_blocks(x, 1)
        y = torch.empty(case["T"], case["V"], device="cuda", dtype=torch.float64)
        for v0 in range(0, case["V"], 16384):
            codes = st["codes"][v0:v0 + 16384, :H].view(torch.float8_e4m3fn).double()
            for i in range(0, codes.shape[0], 128):
                codes[i:i + 128] *= st["scales"][(v0 + i) // 128].double().repeat_interleave(128)[:H]
            y[:, v0:v0 + 16384] = xq @ codes.t().contiguous()
        return dict(y=y)
    W, dy = _exact_blocks(st["W"].double(), 128), st["dy"].double()
    gW = _exact_blocks(dy.t().contiguous(), 1) @ _exact_blocks(x.t().contiguous(), 1).t().contiguous()
    return dict(y=_exact_blocks(x, 1) @ W.t().contiguous(), grad_x=_exact_blocks(dy, 1) @ W, grad_W=gW)


def _exact_sample(case, st):
    T = case["T"]
    z, u = st["z"].double().cpu().numpy(), st["u"].double().cpu().numpy()
    s = {k: v.double().cpu().numpy() if isinstance(v, torch.Tensor) else np.full(T, float(np.float32(v))) for k, v in st["settings"].items()}
    token, logp = np.zeros(T, np.int64), np.zeros(T)
    for t in range(T):
        if s["temperature"][t] == 0:
            token[t] = int(np.argmax(z[t]))
            continue
        y = z[t] / s["temperature"][t]
        p = np.exp(y - y.max())
        kept = np.arange(y.size)
        if case["filters"] != "none":
            down = np.argsort(-z[t], kind="stable")
            down = down[:int(s["top_k"][t]) or y.size]
            mass = np.cumsum(p[down])
            n = 1 + int((mass[:-1] < s["top_p"][t] * mass[-1]).sum())
            down = down[:n]
            kept = np.sort(down[p[down] >= s["min_p"][t]])
        run_ = np.cumsum(p[kept])
        at = int(np.searchsorted(run_, u[t] * run_[-1], side="right"))
        token[t] = kept[at]
        logp[t] = math.log(p[kept[at]] / run_[-1])
    return dict(token=torch.from_numpy(token), logp=torch.from_numpy(logp))


def _exact_top(case, st):
    T, K = case["T"], case["K"]
    top = torch.empty(T, K, device="cuda", dtype=torch.float64)
    lse = torch.empty(T, device="cuda", dtype=torch.float64)
    for t0 in range(0, T, 256):
        z = st["z"][t0:t0 + 256].double()
        top[t0:t0 + 256] = torch.topk(z, K, dim=1).values
        lse[t0:t0 + 256] = torch.logsumexp(z / case["tau"], 1)
    return dict(logits=top, index=None, lse=lse)


def _exact_clip(case, st):
    total = torch.zeros((), device="cuda", dtype=torch.float64)
    for x in st["parts"]:
        total += x.double().square().sum()
    norm = total.sqrt()
    factor = min(1.0, st["max_norm"] / float(norm))
    return dict(norm=norm, grads={k: x.double() * factor for k, x in st["flat"].items()})


def exact(case, seed):
    st = prepare(case, seed)
    return dict(linear=_exact_linear, sample=_exact_sample, top=_exact_top, clip=_exact_clip)[case["op"]](case, st)

"""Top logits and sampled tokens on the GPU against the fp64 reference."""
import numpy as np
import pytest
import torch

from oracle import beside_oracle as O
from paper_2603_01875_amd import kdloss as K

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
VS = [1, 2, 7, 8, 9, 63, 500, 2047, 2048, 2049, 4100, 8192, 8200, 20011, 50257, 151936]


def np64(t):
    return t.detach().cpu().double().numpy()


def rows(seed, T, V, kind, dtype):
    rng = np.random.default_rng(seed)
    z = rng.standard_normal((T, V)) * 2
    if kind == "model":                                  # some entries stand out
        n = min(V, 300)
        for t in range(T):
            z[t, rng.permutation(V)[:n]] += 9 - 2 * np.log1p(np.arange(n))
    elif kind == "equal":
        z[:] = -1.5
    elif kind == "steps":                                # few values, many equal ones
        z = np.rint(z)
    elif kind == "masked":
        z[rng.random((T, V)) < 0.9] = -np.inf
        z[:, V // 2] = 0.25
    elif kind == "one":
        z[:] = -np.inf
        z[np.arange(T), rng.integers(0, V, T)] = -3.0
    elif kind == "lowest":                               # a mask of the type's lowest value
        z[rng.random((T, V)) < 0.9] = float(torch.finfo(DT[dtype]).min)
    elif kind == "zeros":
        z = np.where(rng.random((T, V)) < 0.5, 0.0, -0.0)
    elif kind == "wide":
        z = z * 40
    return torch.from_numpy(z.astype(np.float32)).to(DT[dtype])


KINDS = ["normal", "model", "equal", "steps", "masked", "one", "lowest", "zeros", "wide"]


def check_top(z, K_, tau, out):
    top, index, lse = O.top_logits(np64(z), K_, tau)
    assert (out["top_index"].cpu().numpy() == index).all()
    got = np64(out["top_logits"])
    assert ((got == top) | (np.isnan(got) & np.isnan(top))).all()
    # an fp32 sum of powers of two: its terms' exponents are off by three half steps of at most 32 before the term is below 2^-32 of the
    # whole, a sum of 64 and then nine and ten additions; the result is rounded once
    got = np64(out["lse"])
    same = (got == lse) | (np.isnan(got) & np.isnan(lse))
    with np.errstate(invalid="ignore"):
        assert (same | (np.abs(got - lse) <= (3 * 32 + 85) * 2.0 ** -24 + 2.0 ** -23 * np.abs(lse))).all()


@pytest.mark.parametrize("V", VS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["normal", "model", "steps", "equal"])
def test_top_logits_sizes(V, dtype, kind):
    z = rows(V, 3, V, kind, dtype)
    for K_ in sorted({1, min(V, 5), min(V, 64), min(V, K.TOPK_MAX)}):
        check_top(z, K_, 1.0, K.kd_top_logits(z.cuda(), K_))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,K_,tau", [(5, 777, 20, 2.0), (2, 33000, 100, 0.5), (130, 3000, 8, 1.0)])
def test_top_logits_kinds(kind, dtype, T, V, K_, tau):
    z = rows(T + V, T, V, kind, dtype)
    check_top(z, K_, tau, K.kd_top_logits(z.cuda(), K_, tau))


def test_top_logits_of_rows_that_have_none_or_no_numbers():
    z = torch.randn(6, 5000)
    z[0] = -float("inf")
    z[1, 77] = float("nan")
    z[2, 4999], z[2, 3] = float("inf"), float("inf")
    z[3] = float("nan")
    z[4, 1:] = -float("inf")
    z[5, 7] = -float("nan")
    for dtype in (torch.float32, torch.bfloat16):
        out = K.kd_top_logits(z.to(dtype).cuda(), 9, index_dtype=K.I32)
        assert out["top_index"].dtype == torch.int32
        check_top(z.to(dtype), 9, 1.0, out)


def test_top_logits_of_rows_with_more_equal_ones_than_a_list_holds():
    z = torch.randn(6, 20_000)
    z[0, 5000:] = float("nan")
    z[1, ::2] = 9.0
    z[2, 3000:] = float("inf")
    z[3, ::3], z[3, 1::3] = 0.0, -0.0
    z[4] = float(torch.finfo(torch.float32).min)
    z[5, 100:] = -float("inf")
    for dtype in (torch.float32, torch.bfloat16):
        for K_ in (1, 700, 1024):
            check_top(z.to(dtype), K_, 1.0, K.kd_top_logits(z.to(dtype).cuda(), K_))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("offset,ld", [(1, 2100), (3, 2051), (8, 4096)])
def test_rows_of_a_wider_array_at_an_odd_offset(dtype, offset, ld):
    wide = torch.randn(7 * ld + 64).to(DT[dtype])
    z = wide[offset:offset + 7 * ld].view(7, ld)[:, :2049]
    dev = wide.cuda()[offset:offset + 7 * ld].view(7, ld)[:, :2049]
    check_top(z, 33, 1.0, K.kd_top_logits(dev, 33))
    u = torch.rand(7)
    check_tokens(z, u, dict(top_p=0.9), K.kd_sample(dev, u.cuda(), top_p=0.9))
    check_tokens(z, u, {}, K.kd_sample(dev, u.cuda()))


def check_tokens(z, u, settings, out, least=0):
    """Tokens are equal wherever the sums' error (exp to 2^-39, and as much again for the total that u or top_p multiplies) cannot
    reach the next border: 2^-36 of the whole.  At least `least` of the rows have to be such."""
    z, u = np64(z), np64(u)
    token, logp = out["token"].cpu().numpy(), np64(out["logp"])
    pinned = 0
    for t in range(z.shape[0]):
        s = {k: (v[t].item() if isinstance(v, torch.Tensor) else v) for k, v in settings.items()}
        want, lp = O.sample(z[t], u[t], **s)
        if want >= 0 and O.distance(z[t], u[t], **s) < 2.0 ** -36:
            assert 0 <= token[t] < z.shape[1] and z[t][token[t]] > -np.inf
            continue
        pinned += 1
        assert token[t] == want, (t, s, token[t], want, u[t])
        if want < 0:
            assert np.isnan(logp[t])
        else:
            # the logit's distance from the largest and the sum's logarithm in 64 bits, one rounding
            assert abs(logp[t] - lp) <= 2.0 ** -24 * abs(lp) + 2.0 ** -34
    assert pinned >= least


SETTINGS = [dict(), dict(temperature=0.0), dict(temperature=0.7), dict(temperature=3.0), dict(top_k=1), dict(top_k=40), dict(top_k=700),
            dict(top_k=2000), dict(top_p=0.9), dict(top_p=0.999), dict(top_p=0.01), dict(min_p=0.05), dict(min_p=1.0), dict(min_p=1e-4),
            dict(temperature=0.8, top_k=50, top_p=0.9, min_p=0.02), dict(temperature=1.5, top_k=3000, top_p=0.95, min_p=0.001),
            dict(top_p=0.9, min_p=0.01), dict(top_k=100, top_p=0.5), dict(temperature=1e-6), dict(temperature=1e6)]
US = [0.0, 2.0 ** -30, 0.3, 0.5, 0.99, 1 - 2.0 ** -24]


@pytest.mark.parametrize("V", VS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", ["normal", "model"])
def test_tokens_sizes(V, dtype, kind):
    z = rows(V + 1, 6, V, kind, dtype)
    u = torch.tensor(US)
    for s in (SETTINGS[0], SETTINGS[5], SETTINGS[8], SETTINGS[11], SETTINGS[14]):
        check_tokens(z, u, s, K.kd_sample(z.cuda(), u.cuda(), **s), 4)


@pytest.mark.parametrize("settings", SETTINGS, ids=lambda s: ",".join(f"{k}={v}" for k, v in s.items()) or "all")
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tokens_kinds(kind, settings, dtype):
    z = rows(11, 6, 12345, kind, dtype)
    u = torch.tensor(US)
    check_tokens(z, u, settings, K.kd_sample(z.cuda(), u.cuda(), **settings))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,V", [(40, 1000), (300, 20000), (3, 151936)])
def test_tokens_with_settings_of_each_row(dtype, T, V):
    rng = np.random.default_rng(T)
    z = rows(T, T, V, "model", dtype)
    z[rng.random(T) < 0.3] = rows(T + 1, T, V, "steps", dtype)[0]
    u = torch.from_numpy(rng.random(T).astype(np.float32))
    s = dict(temperature=torch.from_numpy(rng.choice([0, 0.5, 1, 1.3], T).astype(np.float32)),
             top_k=torch.from_numpy(rng.choice([0, 0, 1, 40, 1000, V + 5], T).astype(np.int32)),
             top_p=torch.from_numpy(rng.choice([1, 0.9, 0.5], T).astype(np.float32)),
             min_p=torch.from_numpy(rng.choice([0, 0, 0.05], T).astype(np.float32)))
    check_tokens(z, u, s, K.kd_sample(z.cuda(), u.cuda(), **{k: v.cuda() for k, v in s.items()}), T // 2)


@pytest.mark.parametrize("settings", [dict(top_p=0.9), dict(min_p=0.01), dict(top_p=0.7, min_p=0.002)])
def test_tokens_of_more_rows_than_share_their_sums(settings):
    T, V = 2100, 4500
    z = rows(5, T, V, "normal", "bf16")
    z[::7] = rows(6, 1, V, "equal", "bf16")
    u = torch.from_numpy(np.random.default_rng(1).random(T).astype(np.float32))
    check_tokens(z, u, settings, K.kd_sample(z.cuda(), u.cuda(), **settings), T - 400)


def test_every_token_of_a_row_is_drawn_where_the_uniform_numbers_say():
    """A sweep of u over one row: the borders lie where the reference has them."""
    V, T = 700, 4000
    row = rows(3, 1, V, "model", "f32")
    z = row.expand(T, V)
    u = torch.from_numpy(((np.arange(T) + 0.5) / T).astype(np.float32))
    for s in (dict(), dict(top_k=30), dict(top_p=0.8), dict(min_p=0.01)):
        out = K.kd_sample(z.cuda().contiguous(), u.cuda(), **s)
        check_tokens(z, u, s, out, T - 5)
        assert (np.diff(out["token"].cpu().numpy()) >= 0).all()


def test_rows_that_cannot_be_drawn_from():
    z = torch.randn(9, 3000)
    z[0] = -float("inf")
    z[1, 5], z[2, 5], z[3, 5] = float("nan"), float("inf"), -float("nan")
    u = torch.tensor([0.5, 0.5, 0.5, 0.5, 1.0, -0.1, float("nan"), 0.5, 0.5])
    for s in (dict(), dict(top_k=5), dict(top_p=0.5), dict(temperature=0.0)):
        out = K.kd_sample(z.cuda(), u.cuda(), index_dtype=K.I32, **s)
        assert out["token"].dtype == torch.int32
        assert (out["token"][:7] == -1).all() and torch.isnan(out["logp"][:7]).all() and (out["token"][7:] >= 0).all()
    f = torch.full((9,), 0.5)
    bad = dict(temperature=torch.tensor([1, 1, 1, 1, -1.0, float("nan"), 1e-7, 2e6, float("inf")]),
               top_k=torch.tensor([1, 1, 1, 1, -1, -5, 1, 1, 1], dtype=torch.int32),
               top_p=torch.tensor([1, 1, 1, 1, 0.0, 1.5, float("nan"), -1.0, 0.5]),
               min_p=torch.tensor([0, 0, 0, 0, -0.1, 1.5, float("nan"), 0.5, 0.0]))
    for k, v in bad.items():
        out = K.kd_sample(z.cuda(), f.cuda(), **{k: v.cuda()})
        assert (out["token"][4:6] == -1).all()
        ok = dict(temperature=[], top_k=[6, 7, 8], top_p=[8], min_p=[7, 8])[k]
        assert [t for t in range(4, 9) if out["token"][t] >= 0] == ok


def test_a_longer_row_than_any_vocabulary():
    V = (1 << 24) - 3
    z = torch.randn(1, V, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    u = torch.tensor([0.7])
    for s in (dict(), dict(top_k=50), dict(top_p=0.5)):
        check_tokens(z, u, s, K.kd_sample(z.cuda(), u.cuda(), **s))
    check_top(z, 1024, 1.0, K.kd_top_logits(z.cuda(), 1024))


def test_results_are_the_same_bits_every_time():
    z = rows(9, 30, 30000, "steps", "bf16").cuda()
    u = torch.rand(30, device="cuda")
    first = K.kd_sample(z, u, top_p=0.9), K.kd_top_logits(z, 100)
    for _ in range(5):
        again = K.kd_sample(z, u, top_p=0.9), K.kd_top_logits(z, 100)
        for x, y in zip(first, again):
            assert all(torch.equal(x[k], y[k]) for k in x)

"""Tokens of rows whose largest logit is far from zero, up to the ends of the type, on the GPU against the fp64 reference."""
import numpy as np
import pytest
import torch

from paper_2603_01875_amd import kdloss as K
from tests.test_gpu_rows import DT, check_tokens

pytestmark = pytest.mark.gpu
SETTINGS = [dict(), dict(top_k=40), dict(top_k=1500), dict(top_p=0.9), dict(min_p=0.05), dict(temperature=0.0), dict(temperature=1e-6), dict(temperature=1e6),
            dict(temperature=0.7, top_k=50, top_p=0.9, min_p=0.02)]
US = [0.0, 0.1234567, 0.3, 0.5, 0.877, 1 - 2.0 ** -24]


def check(z, settings, least):
    u = torch.tensor((US * z.shape[0])[:z.shape[0]])
    print(tuple(z.shape), z.dtype, settings, flush=True)
    check_tokens(z, u, settings, K.kd_sample(z.cuda(), u.cuda(), **settings), least)


def name(s):
    return ",".join(f"{k}={v}" for k, v in s.items()) or "all"


@pytest.mark.parametrize("settings", SETTINGS, ids=name)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 33, 5001, 151_935])
def test_rows_of_one_value_however_large(V, dtype, settings):
    """A row that is masked throughout with the type's lowest value is a uniform draw, as any row of equal logits."""
    most = float(torch.finfo(DT[dtype]).max)
    z = torch.tensor([-most, most, -1e18, 1e18, -1e20, 1e20, -1e30, 1e30, 3e15, -500.0, 255.0, 257.0]).to(DT[dtype]).view(-1, 1).expand(-1, V).contiguous()
    # (with top-p, u times the kept ones may be a whole number: those rows are not pinned)
    check(z, settings, 6 if "top_p" in settings or "top_k" in settings else 10)


@pytest.mark.parametrize("settings", SETTINGS, ids=name)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [5001, 151_936])
def test_rows_around_a_far_value(V, dtype, settings):
    """Numbers around -3e7 to 1e10, with what the type resolves there, and a part of the vocabulary at the lowest value."""
    rng = np.random.default_rng(V)
    z = rng.standard_normal((12, V)) * 2
    z += np.array([0, 200, 300, -300, 1000, -1e4, 1e5, -1e6, 1e7, -3e7, 1e9, 1e10])[:, None]
    z = torch.from_numpy(z.astype(np.float32)).to(DT[dtype])
    z[::2, ::3] = float(torch.finfo(DT[dtype]).min)
    check(z, settings, 6)


@pytest.mark.parametrize("settings", SETTINGS, ids=name)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_few_entries_at_the_ends_of_the_type(dtype, settings):
    rng = np.random.default_rng(1)
    most = torch.finfo(DT[dtype]).max
    z = torch.from_numpy((rng.standard_normal((6, 20_011)) * 3).astype(np.float32)).to(DT[dtype])
    z[0, 5::4000] = most
    z[1, 7000:] = -most
    z[2, :] = -most
    z[2, 19_000] = 0.0
    z[3, ::2], z[3, 1::2] = most, -most
    z[4, :] = -most
    z[4, 17::5000] = -most * 0.75
    z[5, 100:] = -float("inf")
    z[5, :100] = -most
    check(z, settings, 3)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_batch_with_a_row_that_is_masked_throughout(dtype):
    """Each row's own temperature, one row all lowest values: its token is as likely anywhere."""
    T, V = 64, 20_011
    rng = np.random.default_rng(2)
    z = torch.from_numpy((rng.standard_normal((T, V)) * 3).astype(np.float32)).to(DT[dtype])
    z[::9] = torch.finfo(DT[dtype]).min
    u = torch.from_numpy(rng.random(T).astype(np.float32))
    s = dict(temperature=torch.from_numpy(rng.choice([0.3, 1.0, 1.7], T).astype(np.float32)))
    out = K.kd_sample(z.cuda(), u.cuda(), **{k: v.cuda() for k, v in s.items()})
    check_tokens(z, u, s, out, T - 2)
    same = out["token"][::9].cpu()
    assert (same == (u[::9].double() * V).long()).all()

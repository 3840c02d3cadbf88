"""Top logits of a student whose logits share a large part: the loss knows differences of them only, so the part must not leave a
rounding behind.  All logits are sums of few bits, exact in fp32."""
import numpy as np
import pytest
import torch

from oracle import head_oracle as O
from paper_2603_01875_amd import kdloss as K
from tests import head_util as U

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [20, 100, 300])
@pytest.mark.parametrize("k", [5, 64, 100])
@pytest.mark.parametrize("tail", [O.RENORM, O.REST, O.DROP])
@pytest.mark.parametrize("dtype,tau", [("bf16", 1.0), ("bf16", 2.0 ** -6), ("f32", 1.0)])
def test_a_large_common_part_cancels(T, k, tail, dtype, tau):
    H, V = 64, 1024
    rng = np.random.default_rng(T + k)
    W, h = np.zeros((V, H)), np.zeros((T, H))
    W[:, 0], h[:, 0] = 1.0, 65536.0 * tau
    W[:, 1:9] = rng.integers(-8, 9, (V, 8)) / 8
    h[:, 1:9] = rng.integers(-4, 5, (T, 8)) / 4 * tau      # (logits over tau: 65536 and sixteen bits behind it, multiples of 2^-5)
    h, W = U.rounded(h, dtype), U.rounded(W, dtype)
    ids = torch.from_numpy(np.stack([rng.permutation(V)[:k] for _ in range(T)]))
    a = torch.from_numpy((rng.standard_normal((T, k)) * tau).astype(np.float32))
    lse = torch.from_numpy((np.log(np.exp(U.np64(a) / tau).sum(1)) + (0.5 if tail == O.REST else -0.7)).astype(np.float32))
    ref = O.topk(U.np64(a), ids.numpy(), U.np64(h), U.np64(W), U.np64(lse), tau=tau, tail=tail)
    out = K.kd_topk_fwd(a.cuda(), ids.cuda(), *U.device(h, W), lse=None if tail == O.RENORM else lse.cuda(), tau=tau, tail=tail)
    rows = U.np64(out["per_token_loss"])
    # exp2, log2 and what is a difference of logits, of size 40 at most, as in head_util.bounds with exact logits
    tol = 2.0 ** -19 + 8 * U.F32 * 40
    assert (np.abs(rows - ref["per_token_loss"]) <= tol).all(), np.abs(rows - ref["per_token_loss"]).max()
    assert abs(float(out["loss"].item()) - ref["loss"]) <= tol

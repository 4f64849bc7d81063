"""Finite logits of any size: a log-sum-exp, a log-probability and gradients that are finite, within the bounds that the sums'
arithmetic gives (test_gpu_logprob has them; of logits of 10^10 they leave only the leading digits)."""
import numpy as np
import pytest
import torch

from oracle.logprob import oracle_logprob

from test_gpu_logprob import bounds, make
from util import to_np

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,dtype", [(3, torch.bfloat16), (40, torch.bfloat16), (300, torch.bfloat16), (40, torch.float32)])
@pytest.mark.parametrize("size", [1e4, 1e7, 1e10, 1e20])
@pytest.mark.parametrize("scale", [1.0, -1.0])
def test_finite_logits_of_any_size(lib, n, dtype, size, scale):
    hidden, weight, targets, g = make(n, 512, 700, n, dtype=dtype)
    hidden = (hidden.float() * size).to(dtype)
    hn, wn = to_np(hidden), to_np(weight)
    z = scale * (hn @ wn.T)
    if n > 4:
        targets[::2] = torch.as_tensor(z.argmax(1)[::2].astype(np.int32), device="cuda")   # rows that are certain
    want = oracle_logprob(hn, wn, targets.cpu().numpy(), None, scale)
    lp, lse = lib.psrl_token_logprob_fwd(hidden, weight, targets, scale=scale)
    zerr, lerr = bounds(hn, wn, scale, want, dtype)
    assert (np.abs(to_np(lse) - want["lse"]) <= lerr).all()
    assert (np.abs(to_np(lp) - want["logprob"]) <= lerr + zerr + 2.0 ** -22 * (np.abs(want["logprob"]) + 2 * np.abs(want["lse"]))).all()
    dh, dw = lib.psrl_token_logprob_bwd(hidden, weight, targets, lp, lse, g, scale=scale)
    # |dz| <= 2 |G| whatever the logits' error
    top_w, top_h = np.abs(wn).max(0), np.abs(hn)
    g_abs = np.abs(to_np(g))
    assert torch.isfinite(dh).all() and torch.isfinite(dw).all()
    # dz has at most the target and entries whose probabilities the logits' error can make one: every entry, in the worst case
    assert (np.abs(to_np(dh)) <= 1.01 * g_abs[:, None] * (top_w + np.abs(wn).sum(0))[None, :] + 1e-30).all()
    assert (np.abs(to_np(dw)) <= 1.01 * 2 * (g_abs[:, None] * top_h).sum(0)[None, :]).all()


@pytest.mark.parametrize("n,dtype", [(3, torch.bfloat16), (40, torch.bfloat16), (300, torch.bfloat16), (40, torch.float32)])
@pytest.mark.parametrize("size", [1.0, 1e10])
def test_huge_logits_beside_one_that_is_no_number(lib, n, dtype, size):
    hidden, weight, targets, g = make(n, 512, 700, n, dtype=dtype)
    hidden = (hidden.float() * size).to(dtype)
    weight[650, 3] = float("nan")
    lp, lse = lib.psrl_token_logprob_fwd(hidden, weight, targets)
    assert torch.isnan(lse).all() and torch.isnan(lp).all()

"""Rows whose logits are not numbers, on every path of the token log-probabilities: what the model lost may not come back as
a probability of one.  The other rows' results are the same bits as without them."""
import pytest
import torch

from test_gpu_logprob import make

pytestmark = pytest.mark.gpu
PATHS = [(3, torch.bfloat16), (4, torch.bfloat16), (40, torch.bfloat16), (300, torch.bfloat16), (5000, torch.bfloat16), (40, torch.float32),
         (300, torch.float32)]


@pytest.mark.parametrize("n,dtype", PATHS)
@pytest.mark.parametrize("what", ["nan", "inf", "overflow", "all minus inf"])
def test_rows_without_a_distribution(lib, n, dtype, what):
    hidden, weight, targets, g = make(n, 64, 300, n, dtype=dtype)
    weight[:, 5] = weight[:, 5].abs() + 1          # the logits of a row with an infinity there are all infinite, none NaN
    g = g.abs() + 0.5
    clean = lib.psrl_token_logprob_fwd(hidden, weight, targets)
    dh_clean, _ = lib.psrl_token_logprob_bwd(hidden, weight, targets, *clean, g)
    bad = torch.zeros(n, dtype=torch.bool, device="cuda")
    bad[1::max(2, n // 7)] = True
    dirty, scale = hidden.clone(), 1.0
    if what == "overflow":
        dirty[bad] = 3e38
        dirty[bad, 6:] = 0
        weight[:, :6] = weight[:, :6].abs() + 2    # products beyond fp32's range
        clean = lib.psrl_token_logprob_fwd(hidden, weight, targets)
        dh_clean, _ = lib.psrl_token_logprob_bwd(hidden, weight, targets, *clean, g)
    else:
        dirty[bad, 5] = {"nan": float("nan"), "inf": float("inf"), "all minus inf": -float("inf")}[what]
    lp, lse = lib.psrl_token_logprob_fwd(dirty, weight, targets)
    assert torch.isnan(lp[bad]).all() and not torch.isfinite(lse[bad]).any()
    assert torch.equal(lp[~bad], clean[0][~bad]) and torch.equal(lse[~bad], clean[1][~bad])
    dh, dw = lib.psrl_token_logprob_bwd(dirty, weight, targets, lp, lse, g)
    assert not torch.isfinite(dh[bad]).all(1).any()
    assert torch.equal(dh[~bad], dh_clean[~bad])


@pytest.mark.parametrize("n,dtype", PATHS)
def test_an_entry_of_the_vocabulary_without_a_number(lib, n, dtype):
    """NaN in one row of the weights reaches every distribution; an entry that can never be drawn has log-probability -inf."""
    hidden, weight, targets, g = make(n, 64, 300, n + 1, dtype=dtype)
    hidden[:, 5] = hidden[:, 5].abs() + 1
    impossible = weight.clone()
    impossible[123, 5] = -float("inf")
    targets[1] = 123
    targets[0] = 122
    lp, lse = lib.psrl_token_logprob_fwd(hidden, impossible, targets)
    assert lp[1] == -float("inf") and torch.isfinite(lp[0]) and torch.isfinite(lse).all()
    weight[299, 7] = float("nan")
    lp, lse = lib.psrl_token_logprob_fwd(hidden, weight, targets)
    assert torch.isnan(lp).all() and torch.isnan(lse).all()
    targets[2] = -1                                  # ignored, whatever its row holds
    lp, _ = lib.psrl_token_logprob_fwd(hidden, weight, targets)
    assert lp[2] == 0 and torch.isnan(lp[:2]).all()

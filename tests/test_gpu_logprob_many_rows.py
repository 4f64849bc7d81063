"""More rows than one dimension of a launch counts blocks (65,535 of 64 rows), fp32."""
import pytest
import torch

from test_gpu_logprob import sum_error

pytestmark = pytest.mark.gpu


def test_fp32_beyond_four_million_rows(lib):
    n, h, v = 65535 * 64 + 71, 8, 5
    g0 = torch.Generator(device="cuda").manual_seed(1)
    hidden = torch.randn(n, h, generator=g0, device="cuda")
    weight = torch.randn(v, h, generator=g0, device="cuda") / 3
    targets = torch.randint(0, v, (n,), generator=g0, device="cuda").to(torch.int32)
    g = torch.randn(n, generator=g0, device="cuda")
    lp, lse = lib.psrl_token_logprob_fwd(hidden, weight, targets)
    dh, dw = lib.psrl_token_logprob_bwd(hidden, weight, targets, lp, lse, g)
    at = torch.arange(n, device="cuda")
    hd, wd = hidden.double(), weight.double()
    z = hd @ wd.T
    ref = torch.logsumexp(z, 1)
    a = (hd.abs() @ wd.abs().T).amax(1)
    err = sum_error(h, torch.float32) * a + 2.0 ** -20 + 2.0 ** -22 * ref.abs()
    assert ((lse.double() - ref).abs() <= err).all()
    want = z[at, targets.long()] - ref
    assert ((lp.double() - want).abs() <= 2 * err + 2.0 ** -22 * (want.abs() + 2 * ref.abs())).all()
    dz = -g.double()[:, None] * torch.exp(z - ref[:, None])
    dz[at, targets.long()] += g.double()
    # an error of the logits or of lp moves dz by |g| p times as much; 2^-18 for the exponential and the products
    pe = (4 * err + 2.0 ** -18)[:, None] * g.double().abs()[:, None]
    one = torch.ones_like(wd)
    bound_h = pe * wd.abs().sum(0) + sum_error(v, torch.float32) * (dz.abs() @ wd.abs())
    assert ((dh.double() - dz @ wd).abs() <= bound_h + 2.0 ** -23).all()
    bound_w = (one[:, :1] * (pe * hd.abs()).sum(0)) + sum_error(n, torch.float32) * (dz.abs().T @ hd.abs())
    assert ((dw.double() - dz.T @ hd).abs() <= bound_w).all()

"""Gradients of norms whose products with the rows pass fp32's range although the gradients do not: d_x is finite wherever the formula's is.

Tolerance as for ordinary rows (tests/test_gpu_rms_norm.py): 2^-17 r (|g| + |u| mean |g u|) and a half step of the result, 2^-8 of it in bf16; with
rows scaled by 2^-110 the roundings are the same."""
import numpy as np
import pytest
import torch

from oracle.layer import oracle_rms_bwd

from util import to_np

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dim", [8, 64, 264, 512, 1024, 4096, 5120, 12288, 32768])
@pytest.mark.parametrize("rows", [7, 700])
def test_large_gradients(lib, dtype, dim, rows):
    g = torch.Generator(device="cuda").manual_seed(dim)
    x, w, dy = (torch.randn(*s, device="cuda", generator=g) for s in ((rows, dim), (dim,), (rows, dim)))
    w = w.clamp(-2, 2)
    dy = dy.clamp(-3, 3)
    plain = x.to(dtype).clone(), dy.to(dtype).clone()
    # rows of their own size times gradients of their own: each sum of g h is beyond 2^128 but no term of d_x is
    size = {0: (2.0 ** 40, 2.0 ** 100), 1: (2.0 ** 7, 2.0 ** 123), 2: (2.0 ** 55, 2.0 ** 90), 3: (-(2.0 ** 20), 2.0 ** 118), 4: (2.0 ** 100, 2.0 ** 60),
            5: (2.0 ** 120, 2.0 ** 90)}
    for i, (a, b) in size.items():
        x[i], dy[i] = x[i].abs() * a, dy[i].abs() * b      # of one sign, so that nothing cancels
    x, w, dy = x.to(dtype), w.abs().to(dtype), dy.to(dtype)
    d_x = lib.psrl_rms_norm_bwd(x, w, dy)[0]
    torch.cuda.synchronize()
    want, _ = oracle_rms_bwd(to_np(x), to_np(w), to_np(dy), 1e-6)
    h, gg = to_np(x), to_np(dy) * to_np(w)
    r = 1.0 / np.sqrt((h * h).mean(-1, keepdims=True) + 1e-6)
    u = h * r
    tol = 2.0 ** -17 * r * (np.abs(gg) + np.abs(u) * np.abs(gg * u).mean(-1, keepdims=True)) + 2.0 ** -148
    assert np.isfinite(want).all() and np.abs(gg * h).sum(-1)[:6].min() > 2.0 ** 128
    if dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (np.abs(want) + tol) + 2.0 ** -134
    got = to_np(d_x)
    assert np.isfinite(got).all() and (np.abs(got - want) <= tol).all()
    # the rows beside them have the bits that they have without them
    rest = lib.psrl_rms_norm_bwd(plain[0], w, plain[1])[0]
    assert torch.equal(d_x[6:], rest[6:])
    again = lib.psrl_rms_norm_bwd(x, w, dy, want_weight=False)[0]
    assert torch.equal(again, d_x)

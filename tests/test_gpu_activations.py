"""The products' activations and their slopes relative to the value, far out on the negative side too, by every kernel that has them.

z comes through a product with one factor of 1, exactly.  With e = 2^-24 (half a step of fp32), from the documented bounds of the functions
(expf 1 step, erfcf 4; the hardware's 2^x 2 steps, its reciprocal 1; a step is 2 e):
  silu       fp32: exponential 2 e, sum 1, quotient 1, products 2: 16 e with room.  bf16: the exponent z log2(e) + 24 is rounded once, by a half step of at
             most 128, and its factor log2(e) by e: (16 + 2 |z|) e of 2^x, 2^x 4 e, reciprocal 2 e, sum and products 3 e: (32 + 5 |z|) e
  gelu       fp32: the argument's two roundings change erfc by 2 (z^2 + 1) e, erfcf 8 e, products 2 e: (2 z^2 + 16) e.  bf16: the exponent as above with
             z^2 / 2 for |z| and its own two roundings, 3 z^2 e + 25 e; the polynomial 2^-18.8 = 37 e, reciprocal, sums and products 16 e: (3 z^2 + 80) e
  gelu_tanh  u = 2 sqrt(2 / pi) (z + 0.044715 z^3) within 5 e, 5 |u| e in the exponential: that more than silu of u
and a slope the same of the sum of its terms' sizes, 8 e more (and z^2 e for the density's exponent, counted by the gelu's).  A result in bf16 is half a
step off, 2^-8 of the value; below the normal numbers 2^-149 a step, with a factor |z| < 128 behind it: 2^-140, and 2^-134 in bf16."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
ACTS = ["relu", "silu", "gelu", "gelu_tanh"]
E = 2.0 ** -24


def exact(z, act, bf16):
    """value, slope, the terms of the slope by size, e's of the value"""
    z = torch.as_tensor(z, dtype=torch.float64)
    if act == "relu":
        return z.clamp(min=0), (z > 0).double(), (z > 0).double(), 0 * z
    if act == "gelu":
        c, d = 0.5 * torch.special.erfc(-z / 2 ** 0.5), torch.exp(-z * z / 2) / (2 * np.pi) ** 0.5
        return z * c, c + z * d, c + z.abs() * d, 3 * z * z + 80 if bf16 else 2 * z * z + 16
    u = z if act == "silu" else 2 * (2 / np.pi) ** 0.5 * (z + 0.044715 * z ** 3)
    du = 1 if act == "silu" else 2 * (2 / np.pi) ** 0.5 * (1 + 3 * 0.044715 * z * z)
    s, q = torch.special.expit(u), torch.special.expit(-u)
    return z * s, s + z * s * q * du, s + z.abs() * s * q * du, (32 if bf16 else 16) + (10 if act == "gelu_tanh" else 5) * u.abs().clamp(max=200)


def check(got, want, size, steps, name):
    tol = steps * E * size + 2.0 ** -140
    if got.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (want.abs() + tol) + 2.0 ** -134
    err = (got.double().cpu() - want).abs() - tol
    at = int(err.argmax())
    assert torch.isfinite(got).all() and float(err.max()) <= 0, (name, at, float(got[at]), float(want[at]))


def arguments(n, dtype):
    z = torch.cat([torch.linspace(-100, 30, n // 2, dtype=torch.float64), torch.linspace(-15, 15, n - n // 2, dtype=torch.float64)])
    return z.to(dtype).cuda()


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("rows,dtype", [(100, torch.bfloat16), (5000, torch.bfloat16), (5000, torch.float32)])
def test_value(lib, act, rows, dtype):
    """Few rows, pairs of CTAs, fp32."""
    z = arguments(rows, dtype)
    x, w = torch.zeros(rows, 8, device="cuda", dtype=dtype), torch.zeros(24, 8, device="cuda", dtype=dtype)
    x[:, 0], w[:, 0] = z, 1.0
    want, _, _, steps = exact(z.cpu().double(), act, dtype == torch.bfloat16)
    y, stored = lib.psrl_linear_fwd(x, w, activation=act, want_z=True)
    plain = lib.psrl_linear_fwd(x, w, activation=act)[0]
    torch.cuda.synchronize()
    assert torch.equal(stored, z[:, None].expand(-1, 24)) and torch.equal(plain, y)
    for c in (0, 23):
        check(y[:, c], want, want.abs(), steps, act)


@pytest.mark.parametrize("act", ACTS)
def test_value_8_bit(lib, act):
    """Codes of 1 with z for the row's scale: z in fp32 whatever its size."""
    for rows in (100, 5000):
        z = arguments(rows, torch.float32)
        x, w = (torch.ones(n, 16, device="cuda").to(torch.float8_e4m3fn) for n in (rows, 24))
        y = lib.psrl_linear_fwd(x, w, activation=act, x_scale=z / 16, weight_scale=torch.ones(24, device="cuda"))[0]
        want, _, _, steps = exact(z.cpu().double(), act, True)
        check(y[:, 5], want, want.abs(), steps, act)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_slope(lib, act, dtype):
    rows = 5000
    z = arguments(rows, dtype)[:, None].expand(-1, 8).contiguous()
    x, one = torch.zeros(rows, 8, device="cuda", dtype=dtype), torch.ones(rows, 8, device="cuda", dtype=dtype)
    d_x, _, _, d_mul = lib.psrl_linear_bwd(x, torch.eye(8, device="cuda", dtype=dtype), one, z=z, activation=act, mul=one, want_weight=False)
    value, slope, size, steps = exact(z[:, 0].cpu().double(), act, dtype == torch.bfloat16)
    check(d_mul[:, 3], value, value.abs(), steps, "d_mul")
    check(d_x[:, 3], slope, size, steps + 8, "dz")

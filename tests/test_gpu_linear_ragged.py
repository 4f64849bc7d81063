"""Results whose rows end inside 16 bytes, in slices of a larger matrix: nothing beside or behind them is written, by any of the products' kernels,
and they have the bits of the same call with outputs of its own."""
import pytest
import torch

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.bfloat16}


def around(rows, cols, first, pitch, dtype):
    whole = torch.full((rows + 2, pitch), 7.0, device="cuda", dtype=dtype)
    return whole[1:rows + 1, first:first + cols], whole


def untouched(whole, rows, cols, first):
    rest = torch.ones_like(whole, dtype=torch.bool)
    rest[1:rows + 1, first:first + cols] = False
    return bool((whole[rest] == 7.0).all())


# few rows, pairs with a tile each, pairs with several, a pair whose groups share a tile
@pytest.mark.parametrize("m,k", [(5, 64), (100, 4096), (200, 64), (397, 208), (1000, 72), (5000, 64), (8200, 16)])
@pytest.mark.parametrize("n", [1, 2, 7, 8, 9, 63, 65, 127, 130, 255, 257, 513, 701, 1111])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3", "f32"])
def test_only_the_results_are_written(lib, dtype, m, k, n):
    t = TYPES[dtype]
    g = torch.Generator(device="cuda").manual_seed(m + n)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)
    x, w, bias = rnd(m, k), rnd(n, k), rnd(n).to(t)
    kw = {}
    if dtype == "e4m3":
        (x, sx), (w, sw) = lib.psrl_quantize_rows(x), lib.psrl_quantize_rows(w)
        kw = dict(x_scale=sx, weight_scale=sw)
    else:
        x, w = x.to(t), w.to(t)
    pitch = -(-n // 8) * 8 + 24
    beside = [around(m, n, 8, pitch, t)[0].copy_(rnd(m, n)) for _ in range(2)]
    mul, res = beside
    # bias alone leaves by two buffers, the rest by three
    want = lib.psrl_linear_fwd(x, w, bias=bias, **kw)[0].clone()
    y, whole = around(m, n, 8, pitch, t)
    lib.psrl_linear_fwd(x, w, bias=bias, y=y, **kw)
    torch.cuda.synchronize()
    assert torch.equal(y, want) and untouched(whole, m, n, 8)
    want = [v.clone() for v in lib.psrl_linear_fwd(x, w, bias=bias, activation="silu", mul=mul, residual=res, want_z=True, **kw)]
    (y, whole), (z, whole_z) = around(m, n, 8, pitch, t), around(m, n, 16, pitch, t)
    lib.psrl_linear_fwd(x, w, bias=bias, activation="silu", mul=mul, residual=res, y=y, z=z, want_z=True, **kw)
    torch.cuda.synchronize()
    assert torch.equal(y, want[0]) and torch.equal(z, want[1]) and untouched(whole, m, n, 8) and untouched(whole_z, m, n, 16)
    # over the residual and the factor, whose own surroundings stay
    (y, whole), (z, whole_z) = around(m, n, 8, pitch, t), around(m, n, 8, pitch, t)
    y.copy_(res)
    z.copy_(mul)
    lib.psrl_linear_fwd(x, w, bias=bias, activation="silu", mul=z, residual=y, y=y, z=z, want_z=True, **kw)
    torch.cuda.synchronize()
    assert torch.equal(y, want[0]) and torch.equal(z, want[1]) and untouched(whole, m, n, 8) and untouched(whole_z, m, n, 8)


@pytest.mark.parametrize("m,k,n", [(5, 72, 701), (300, 264, 257), (1000, 520, 9), (2050, 136, 1111)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients(lib, dtype, m, k, n):
    t = TYPES[dtype]
    x, w = torch.randn(m, k, device="cuda").to(t), torch.randn(n, k, device="cuda").to(t)
    pitch = -(-n // 8) * 8 + 24
    dy, z, mul = (around(m, n, 8, pitch, t)[0].copy_(torch.randn(m, n, device="cuda")) for _ in range(3))
    want = [v.clone() for v in lib.psrl_linear_bwd(x, w, dy, z=z, activation="gelu", mul=mul, want_bias=True)]
    shapes = [(m, k), (n, k), (1, n), (m, n)]
    out = [around(r, c, 8, -(-c // 8) * 8 + 16, t) for r, c in shapes]
    lib.psrl_linear_bwd(x, w, dy, z=z, activation="gelu", mul=mul, want_bias=True, d_x=out[0][0], d_weight=out[1][0], d_bias=out[2][0][0], d_mul=out[3][0])
    torch.cuda.synchronize()
    for (got, whole), (r, c), v in zip(out, shapes, want):
        assert torch.equal(got, v.view(r, c)) and untouched(whole, r, c, 8)

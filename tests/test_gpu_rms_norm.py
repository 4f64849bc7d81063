"""Root-mean-square norms on the GPU against the fp64 oracle.

Tolerances, e = 2^-24 (half a step of fp32).  The mean square is a sum of positive terms, each added at most 32 times by one thread
and ten times across threads: 42 e, half of that in r; rsqrt 4 e, three products 3 e: y is within 2^-19 |y| (32 e), the scale with
its division too.  d_x = d_summed + r (g - u a), u = h r, a = mean(g u): a is within 64 e of mean |g u|, u and r within 32 e, so all of
it within 2^-17 r (|g| + |u| mean |g u|) and 2 e (|d_summed| + |d_x|).  d_weight: every term within 32 e, and (rows + 64) e of the sum of
their sizes for the additions.  A bf16 result adds half a step, 2^-8 of the value; a code half a step, 2^-4 of the value or 2^-10
of the scale.  Results below the types' normal numbers have steps of 2^-149 in fp32 and 2^-133 in bf16 whatever their size: two of
the former (a product, a sum) and half of the latter are allowed besides."""
import numpy as np
import pytest
import torch

from oracle.layer import oracle_rms, oracle_rms_bwd

from util import to_np

pytestmark = pytest.mark.gpu
E = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def within(got, want, tol, name):
    g = got.detach().double().cpu().numpy()
    tol = tol + 2.0 ** -148
    if got.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (np.abs(want) + tol) + 2.0 ** -134
    err = np.abs(g - want) - tol
    assert np.isfinite(g).all() and err.max() <= 0, (name, float(err.max()))


def check_fwd(out, h, w, eps, name=""):
    y, _, codes, scales = out
    want, _ = oracle_rms(h, 1.0 if w is None else to_np(w), eps)
    if y is not None:
        within(y, want, 2.0 ** -19 * np.abs(want), name + "y")
    if codes is not None:
        s = np.maximum(np.abs(want).max(-1) / 448.0, 2.0 ** -126)
        within(scales, s, 2.0 ** -19 * s, name + "scales")
        got = codes.float().double().cpu().numpy() * s[..., None]
        assert (np.abs(got - want) <= (2.0 ** -4 * np.abs(want) + 2.0 ** -10 * s[..., None]) * (1 + 2.0 ** -17)).all(), name + "codes"


def check_bwd(got, h, w, dy, eps, ds, name=""):
    w64 = 1.0 if w is None else to_np(w)
    want_x, want_w = oracle_rms_bwd(h, w64, dy, eps, 0.0 if ds is None else ds)
    r = 1.0 / np.sqrt((h * h).mean(-1, keepdims=True) + eps)
    u, g = np.abs(h * r), np.abs(dy * w64)
    if got[0] is not None:
        within(got[0], want_x, 2.0 ** -17 * r * (g + u * (g * u).mean(-1, keepdims=True)) + 2 * E * ((0.0 if ds is None else np.abs(ds)) + np.abs(want_x)),
               name + "d_x")
    if got[1] is not None:
        size = (np.abs(dy) * u).reshape(-1, h.shape[-1])
        within(got[1], want_w, (32 + len(size) + 64) * E * size.sum(0), name + "d_weight")


def draw(shape, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g).to(TYPES[dtype])
    return rnd(*shape), rnd(*shape), rnd(shape[-1]), rnd(*shape), rnd(*shape)


DIMS = [8, 64, 72, 128, 136, 256, 264, 512, 1000, 2048, 4096, 4104, 5120, 8192, 8200, 16384, 16392, 32768]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("rows", [1, 13, 700])
def test_rows(lib, dtype, dim, rows):
    x, res, w, dy, ds = draw((rows, dim), dtype, rows + dim)
    y, summed, codes, scales = lib.psrl_rms_norm_fwd(x, w, 1e-5, residual=res, want_codes=True)
    torch.cuda.synchronize()
    assert torch.equal(summed, (x.float() + res.float()).to(x.dtype))
    check_fwd((y, summed, codes, scales), to_np(summed), w, 1e-5)
    got = lib.psrl_rms_norm_bwd(summed, w, dy, 1e-5, d_summed=ds)
    check_bwd(got, to_np(summed), w, to_np(dy), 1e-5, to_np(ds))
    # without the residual, without a gain, one output at a time; bit for bit what the whole call gives
    y2, none, c2, s2 = lib.psrl_rms_norm_fwd(summed, w, 1e-5, want_y=False, want_codes=True)
    assert y2 is None and none is None and torch.equal(c2.view(torch.uint8), codes.view(torch.uint8)) and torch.equal(s2, scales)
    assert torch.equal(lib.psrl_rms_norm_fwd(summed, w, 1e-5)[0], y)
    check_fwd(lib.psrl_rms_norm_fwd(x, None, 1e-5, want_codes=True), to_np(x), None, 1e-5, "no gain: ")
    check_bwd(lib.psrl_rms_norm_bwd(x, None, dy, 1e-5), to_np(x), None, to_np(dy), 1e-5, None, "no gain: ")
    assert torch.equal(lib.psrl_rms_norm_bwd(summed, w, dy, 1e-5, want_x=False)[1], got[1])
    only_x = lib.psrl_rms_norm_bwd(summed, w, dy, 1e-5, d_summed=ds, want_weight=False)
    assert only_x[1] is None and torch.equal(only_x[0], got[0])
    for a, b in zip(got, lib.psrl_rms_norm_bwd(summed, w, dy, 1e-5, d_summed=ds)):   # the same bits every time
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype,dim", [("f32", 1032), ("f32", 1504), ("f32", 2056), ("f32", 2560), ("f32", 2568), ("f32", 3000), ("bf16", 2056), ("bf16", 3000),
                                       ("bf16", 4800), ("bf16", 5128), ("bf16", 6144), ("bf16", 9000), ("f32", 5000), ("f32", 6144)])
def test_many_rows_of_sizes_between(lib, dtype, dim):
    """Widths between powers of two, with more rows than the blocks take at once: groups of other sizes, some threads without a vector."""
    rows = 1003
    x, _, w, dy, ds = draw((rows, dim), dtype, dim)
    check_fwd(lib.psrl_rms_norm_fwd(x, w, 1e-5, want_codes=True), to_np(x), w, 1e-5)
    check_bwd(lib.psrl_rms_norm_bwd(x, w, dy, 1e-5, d_summed=ds), to_np(x), w, to_np(dy), 1e-5, to_np(ds))
    a, b = (lib.psrl_rms_norm_bwd(x, w, dy, 1e-5) for _ in range(2))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,heads,dim", [(1, 1, 64), (5, 3, 64), (333, 7, 128), (1000, 40, 128), (257, 5, 80), (9, 2, 256), (40, 3, 1024)])
def test_heads_of_a_projections_rows(lib, dtype, rows, heads, dim):
    x, _, w, dy, _ = draw((rows, heads + 3, dim), dtype, rows + heads)
    q, dq = x[:, 2:2 + heads], dy[:, 1:1 + heads]
    before = x.clone()
    y, none, codes, scales = lib.psrl_rms_norm_fwd(q, w, want_codes=True)
    assert none is None and y.shape == q.shape and scales.shape == (rows, heads)
    check_fwd((y, None, codes, scales), to_np(q), w, 1e-6)
    out = torch.full_like(x, float("nan"))
    d_x, d_w = lib.psrl_rms_norm_bwd(q, w, dq, d_x=out[:, 2:2 + heads])
    check_bwd((d_x, d_w), to_np(q), w, to_np(dq), 1e-6, None)
    assert torch.isnan(out[:, :2]).all() and torch.isnan(out[:, 2 + heads:]).all() and torch.equal(x, before)
    lib.psrl_rms_norm_fwd(q, w, y=q)                           # in place, the slices beside it untouched
    assert torch.equal(q, y) and torch.equal(x[:, :2], before[:, :2]) and torch.equal(x[:, 2 + heads:], before[:, 2 + heads:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [64, 4096])
def test_rows_that_are_out_of_the_ordinary(lib, dtype, dim):
    """Zeros, tiny, huge, NaN and infinite rows among others, which they do not touch."""
    n = 40
    x, _, w, dy, _ = draw((n, dim), dtype, 3)
    plain = x.clone()
    x[1] = 0.0
    x[2] *= 2.0 ** -60
    x[3] *= 2.0 ** 100
    x[4] = 3e38
    x[5] *= 2.0 ** 60
    out = lib.psrl_rms_norm_fwd(x, w, want_codes=True)
    got = lib.psrl_rms_norm_bwd(x, w, dy)
    torch.cuda.synchronize()
    check_fwd(out, to_np(x), w, 1e-6)
    check_bwd(got, to_np(x), w, to_np(dy), 1e-6, None)
    x[7, 3] = float("nan")
    x[8, dim - 1] = float("inf")
    x[9] = float("nan")
    bad = lib.psrl_rms_norm_fwd(x, w, want_codes=True)
    bad_x = lib.psrl_rms_norm_bwd(x, w, dy, want_weight=False)[0]
    rest = [i for i in range(n) if i not in (7, 8, 9)]
    for a, b in zip((*bad[:1], *bad[2:], bad_x), (*out[:1], *out[2:], got[0])):
        assert torch.equal(a[rest].view(torch.uint8), b[rest].view(torch.uint8))
    assert torch.isnan(bad[0][7]).all() and torch.isnan(bad[0][8, dim - 1]) and torch.isnan(bad[0][9]).all()
    assert torch.isnan(bad[2][[7, 8, 9]].float()).all() and torch.isnan(bad[3][[7, 8, 9]]).all()
    del plain


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,dim", [(1, 8), (3, 72), (130, 4096), (1000, 1000), (4, 14336), (2, 32768)])
def test_quantised_rows(lib, dtype, rows, dim):
    x = draw((rows, dim + 8), dtype, dim)[0][:, 8:] if dtype == "f32" else draw((rows, dim + 8), dtype, dim)[0][:, :dim]
    codes, scales = lib.psrl_quantize_rows(x)
    v = to_np(x)
    s = np.maximum(np.abs(v).max(-1) / 448.0, 2.0 ** -126)
    within(scales, s, 2 * E * s, "scales")
    got = codes.float().double().cpu().numpy() * s[:, None]
    assert (np.abs(got - v) <= (2.0 ** -4 * np.abs(v) + 2.0 ** -10 * s[:, None]) * (1 + 2.0 ** -20)).all()
    assert np.abs(codes.float().cpu().numpy()).max(-1).min() == 448.0     # the largest number of a row has the largest code
    bad = x.clone()
    bad[0, dim - 1] = float("inf")
    bad[-1, 0] = float("nan")
    bc, bs = lib.psrl_quantize_rows(bad)
    assert torch.isnan(bc[[0, -1]].float()).all() and torch.isnan(bs[[0, -1]]).all()
    assert torch.equal(bc[1:-1].contiguous().view(torch.uint8), codes[1:-1].contiguous().view(torch.uint8)) and torch.equal(bs[1:-1], scales[1:-1])
    wide = torch.zeros(rows, -(-dim // 16) * 16 + 64, device="cuda").to(torch.float8_e4m3fn)
    lib.psrl_quantize_rows(x, codes=wide[:, 16:16 + dim])
    assert torch.equal(wide[:, 16:16 + dim].contiguous().view(torch.uint8), codes.contiguous().view(torch.uint8))
    assert (wide[:, :16].float() == 0).all() and (wide[:, 16 + dim:].float() == 0).all()


def test_gradient_against_differences(lib):
    """Along the gradient itself: (loss(h + s d) - loss(h - s d)) / 2s with y within 2^-19 |y|, so the quotient within
    2^-19 sum |y d_y| / s, and s^2 / 6 of the third derivative: with s |d| = 2^-6 of the rows' size (2^-6)^2 times the first."""
    x, _, w, dy, ds = draw((50, 264), "f32", 1)
    dx, dw = lib.psrl_rms_norm_bwd(x, w, dy, d_summed=ds)
    direction = to_np(dx)
    s = 2.0 ** -6 / np.abs(direction).max()
    loss = lambda h: (to_np(lib.psrl_rms_norm_fwd(h, w)[0]) * to_np(dy)).sum() + (to_np(h) * to_np(ds)).sum()
    up, down = (x.double() + s * dx.double()).float(), (x.double() - s * dx.double()).float()
    slope = (loss(up) - loss(down)) / (2 * s)
    y = np.abs(to_np(lib.psrl_rms_norm_fwd(x, w)[0]) * to_np(dy)).sum()
    assert abs(slope - (direction ** 2).sum()) <= 2.0 ** -19 * y / s + 2.0 ** -10 * (direction ** 2).sum()
    # y is linear in the weight: the quotient is exact but for roundings
    up, down = (w.double() + s * dw.double()).float(), (w.double() - s * dw.double()).float()
    slope = ((to_np(lib.psrl_rms_norm_fwd(x, up)[0]) - to_np(lib.psrl_rms_norm_fwd(x, down)[0])) * to_np(dy)).sum() / (2 * s)
    assert abs(slope - (to_np(dw) ** 2).sum()) <= 2.0 ** -18 * y / s


def test_in_place_streams_graphs_and_many_rows(lib):
    x, res, w, dy, ds = draw((777, 1024), "bf16", 5)
    want = lib.psrl_rms_norm_fwd(x, w, residual=res, want_codes=True)
    grads = lib.psrl_rms_norm_bwd(want[1], w, dy, d_summed=ds)
    # the stream's own memory takes the sum, x its norm; gradients over the incoming ones
    a, b = x.clone(), res.clone()
    got = lib.psrl_rms_norm_fwd(a, w, residual=b, y=a, summed=b)
    assert got[0] is a and got[1] is b and torch.equal(a, want[0]) and torch.equal(b, want[1])
    a, b = dy.clone(), ds.clone()
    assert torch.equal(lib.psrl_rms_norm_bwd(want[1], w, a, d_summed=ds, d_x=a)[0], grads[0])
    assert torch.equal(lib.psrl_rms_norm_bwd(want[1], w, dy, d_summed=b, d_x=b)[0], grads[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = lib.psrl_rms_norm_fwd(x, w, residual=res, want_codes=True, stream=side)
    got_g = lib.psrl_rms_norm_bwd(got[1], w, dy, d_summed=ds, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got[0], want[0]) and torch.equal(got[2].view(torch.uint8), want[2].view(torch.uint8)) and all(torch.equal(*p) for p in zip(got_g, grads))
    # two captured backward passes with workspaces of their own, replayed on new inputs
    ws = [lib.Workspace(lib.psrl_rms_norm_workspace_bytes(777, 1, 1024)) for _ in range(2)]
    outs = [[torch.empty_like(dy), torch.empty_like(w)] for _ in range(2)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for o, k in zip(outs, ws):
            lib.psrl_rms_norm_bwd(want[1], w, dy, d_summed=ds, d_x=o[0], d_weight=o[1], workspace=k)
    dy.mul_(0.5)
    grads = lib.psrl_rms_norm_bwd(want[1], w, dy, d_summed=ds)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for o in outs for a, b in zip(o, grads)) and all(k.status() == 0 for k in ws)
    # a matrix whose elements pass 32 bits
    big = torch.zeros(1100000, 4096, device="cuda", dtype=torch.bfloat16)
    big[-1], big[0] = x[0].repeat(4), x[1].repeat(4)
    y = lib.psrl_rms_norm_fwd(big, None, y=big)[0]
    check_fwd((y[-1:], None, None, None), to_np(x[:1].repeat(1, 4)), None, 1e-6)
    check_fwd((y[:1], None, None, None), to_np(x[1:2].repeat(1, 4)), None, 1e-6)
    assert not y[1:-1].any()


def test_no_rows_and_refusals(lib):
    x, res, w, dy, ds = draw((6, 128), "bf16", 6)
    y, summed, codes, scales = lib.psrl_rms_norm_fwd(x[:0], w, residual=res[:0], want_codes=True)
    assert y.shape == summed.shape == codes.shape == (0, 128) and scales.shape == (0,)
    dx, dw = lib.psrl_rms_norm_bwd(x[:0], w, dy[:0])
    assert dx.shape == (0, 128) and not dw.any()
    for bad in (dict(residual=res[:5]), dict(residual=res.float()), dict(weight=w[:64]), dict(weight=torch.cat([w, w])[::2]), dict(y=x[:, :64]),
                dict(summed=x), dict(x=x.T), dict(x=x[0]), dict(residual=res, summed=res[:3]), dict(want_codes=True, codes=x),
                dict(want_codes=True, scales=torch.zeros(5, device="cuda")), dict(residual=res.cpu())):
        with pytest.raises(ValueError):
            lib.psrl_rms_norm_fwd(**{**dict(x=x, weight=w), **bad})
    for bad in (dict(x=x.half()), dict(weight=w.float())):
        with pytest.raises(TypeError):
            lib.psrl_rms_norm_fwd(**{**dict(x=x, weight=w), **bad})
    for bad in (dict(eps=0.0), dict(residual=res, y=summed_of(x), summed=None, x=torch.cat([x.view(-1), x.view(-1)])[4:4 + 768].view(6, 128))):
        with pytest.raises(lib.PsrlError) as e:
            lib.psrl_rms_norm_fwd(**{**dict(x=x, weight=w), **bad})
        assert e.value.name == "PSRL_ERR_INVALID_ARG"
    for bad in (dict(d_y=dy[:5]), dict(d_y=dy.float()), dict(d_summed=ds[:, :64]), dict(d_x=dy[:4]), dict(d_weight=w.float()), dict(d_y=dy.cpu())):
        with pytest.raises(ValueError):
            lib.psrl_rms_norm_bwd(**{**dict(summed=x, weight=w, d_y=dy), **bad})
    with pytest.raises(lib.PsrlError) as e:
        lib.psrl_rms_norm_bwd(x, w, dy, workspace=lib.Workspace(256))
    assert e.value.name == "PSRL_ERR_WORKSPACE"
    with pytest.raises(RuntimeError):
        lib.psrl_rms_norm_fwd(x.cpu(), w.cpu())


def summed_of(x):
    return torch.empty_like(x)

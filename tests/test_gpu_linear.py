"""Matrix products with their epilogue, and their gradients, on the GPU against the fp64 oracle.

Tolerances.  A product's sum over K, S = sum |x w|: the tensor cores cut off, at every 16 terms (32 in 8 bits), what lies below the sum's
last bit, and the terms' common alignment costs as much: (K / 16 + 4) 2^-22 S; in fp32 a chain of K additions, (K + 4) 2^-24 S, is below
that for K <= 16 only, so there it is (K + 8) 2^-24 S.  Activations have slopes below 1.2 and are computed within 2^-20 of max(|z|, 1).
Results in bf16 are half a step off, 2^-8 of the value.  dz before its rounding to bf16 is within d = 2^-18 |d_y mul| (1 + |z|)
of the oracle's, so where dz + d and dz - d round apart the products may be off by their difference, and nowhere else."""
import numpy as np
import pytest
import torch

from oracle.layer import oracle_act, oracle_linear, oracle_linear_bwd

from util import to_np

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.bfloat16}
ACTS = [None, "relu", "silu", "gelu", "gelu_tanh"]


def within(got, want, tol, name):
    g = got.detach().double().cpu().numpy()
    if got.dtype == torch.bfloat16:
        tol = tol + 2.0 ** -8 * (np.abs(want) + tol)
    err = np.abs(g - want) - tol
    assert g.shape == want.shape and np.isfinite(g).all() and err.max(initial=0.0) <= 0, (name, float(err.max()))


def depth_error(k, f32):
    return (k + 8) * 2.0 ** -24 if f32 else (k / 16 + 4) * 2.0 ** -22


def product(a, b):
    return (torch.as_tensor(a, device="cuda") @ torch.as_tensor(b, device="cuda")).cpu().numpy()


def make(m, k, n, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)
    t = TYPES[dtype]
    wide = -(-n // 8) * 8
    padded = lambda: torch.full((m, wide), float("nan"), device="cuda", dtype=t)[:, :n].copy_(rnd(m, n))
    d = dict(bias=(0.3 * rnd(n)).to(t), mul=padded(), residual=padded(), d_y=padded())
    return rnd(m, k), rnd(n, k) / k ** 0.5, d


def exact_linear(x, w, bias, activation, mul, residual):
    """oracle_linear with its product on the GPU, in fp64"""
    z = product(x, w.T)
    y, z = oracle_linear(np.eye(len(z)), z.T, bias, activation, mul, residual) if len(z) <= 64 else (None, z if bias is None else z + bias)
    if y is None:
        y = oracle_act(z, activation)[0]
        y = y if mul is None else y * mul
        y = y if residual is None else y + residual
    return y, z


def check_fwd(lib, x, w, d, activation, dtype, use, want_z, scales=None):
    m, k = x.shape
    n = w.shape[0]
    kw = {name: d[name] for name in use}
    xs = to_np(x) if scales is None else to_np(x) * to_np(scales[0])[:, None]
    ws = to_np(w) if scales is None else to_np(w) * to_np(scales[1])[:, None]
    if scales is not None:
        kw.update(x_scale=scales[0], weight_scale=scales[1])
    y, z = lib.psrl_linear_fwd(x, w, activation=activation, want_z=want_z, **kw)
    torch.cuda.synchronize()
    np_ = {name: to_np(d[name]) if name in use else None for name in ("bias", "mul", "residual")}
    want_y, want_zz = exact_linear(xs, ws, np_["bias"], activation, np_["mul"], np_["residual"])
    size = product(np.abs(xs), np.abs(ws).T)
    tol_z = depth_error(k, dtype == "f32") * size + 2.0 ** -22 * (np.abs(want_zz) + (0.0 if np_["bias"] is None else np.abs(np_["bias"])))
    if want_z:
        within(z, want_zz, tol_z, "z")
    tol = 1.2 * tol_z + 2.0 ** -20 * np.maximum(np.abs(want_zz), 1.0)
    if np_["mul"] is not None:
        tol = tol * np.abs(np_["mul"]) + 2.0 ** -23 * np.abs(want_y)
    if np_["residual"] is not None:
        tol = tol + 2.0 ** -23 * (np.abs(want_y) + np.abs(np_["residual"]))
    within(y, want_y, tol, "y")
    return y, z


SIZES = [(1, 8, 1), (1, 4096, 1000), (3, 72, 5), (8, 1024, 4096), (33, 264, 130), (128, 64, 256), (129, 200, 257), (256, 8, 64), (300, 1000, 776), (777, 504, 1111),
         (1000, 4096, 264), (2050, 136, 520)]
USES = [((), None, False), (("bias",), "silu", True), (("mul",), "gelu", False), (("residual",), None, False), (("bias", "mul", "residual"), "gelu_tanh", True),
        (("mul", "residual"), "silu", False), (("bias", "residual"), "relu", True)]


@pytest.mark.parametrize("dtype", ["bf16", "e4m3", "f32"])
@pytest.mark.parametrize("m,k,n", SIZES)
@pytest.mark.parametrize("use,activation,want_z", USES)
def test_forward(lib, dtype, m, k, n, use, activation, want_z):
    x, w, d = make(m, k, n, dtype, m + k + n)
    scales = None
    if dtype == "e4m3":
        (x, sx), (w, sw) = lib.psrl_quantize_rows(x), lib.psrl_quantize_rows(w)
        scales = sx, sw
    else:
        x, w = x.to(TYPES[dtype]), w.to(TYPES[dtype])
    y, z = check_fwd(lib, x, w, d, activation, dtype, use, want_z, scales)
    kw = {} if scales is None else dict(x_scale=scales[0], weight_scale=scales[1])
    again = lib.psrl_linear_fwd(x, w, activation=activation, want_z=want_z, **{name: d[name] for name in use}, **kw)
    assert torch.equal(again[0], y) and (z is None or torch.equal(again[1], z))


def check_bwd(lib, x, w, d, z, activation, mul, dtype, **kw):
    m, k = x.shape
    n = w.shape[0]
    f32 = dtype == "f32"
    got = lib.psrl_linear_bwd(x, w, d["d_y"], z=z, activation=activation, mul=mul, want_bias=True, **kw)
    torch.cuda.synchronize()
    xs, ws, dy = to_np(x), to_np(w), to_np(d["d_y"])
    zz, mm = None if z is None else to_np(z), None if mul is None else to_np(mul)
    dz, d_mul, off = dy, None, np.zeros_like(dy)
    if activation is not None or mm is not None:
        value, slope = oracle_act(0.0 * dy if zz is None else zz, activation)
        dz = dy * slope * (1.0 if mm is None else mm)
        if zz is not None and mm is not None:
            d_mul = dy * value
        off = 2.0 ** -18 * np.abs(dy if mm is None else dy * mm) * (1.0 + (0.0 if zz is None else np.abs(zz)))
    rounded, may = dz, off
    if not f32:
        rnd = lambda v: torch.as_tensor(v).float().to(torch.bfloat16).double().numpy()   # fp64 to fp32 first: 2^-24, inside `off`
        rounded = rnd(dz)
        may = np.abs(rnd(dz + off) - rnd(dz - off)) if off.any() else off
    if got[0] is not None:
        within(got[0], product(rounded, ws), depth_error(n, f32) * product(np.abs(rounded), np.abs(ws)) + product(may, np.abs(ws)), "d_x")
    if got[1] is not None:
        within(got[1], product(rounded.T, xs), depth_error(m, f32) * product(np.abs(rounded).T, np.abs(xs)) + product(may.T, np.abs(xs)), "d_weight")
    within(got[2], dz.sum(0), (m + 8) * 2.0 ** -24 * np.abs(dz).sum(0) + off.sum(0), "d_bias")
    if got[3] is not None:
        within(got[3], d_mul, 2.0 ** -19 * np.abs(dy) * np.maximum(np.abs(zz), 1.0), "d_mul")
    return got


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,k,n", [(1, 8, 1), (1, 520, 1000), (7, 72, 5), (64, 1024, 264), (129, 200, 257), (300, 1000, 776), (777, 504, 1111), (1000, 264, 2056), (2050, 136, 520)])
@pytest.mark.parametrize("activation,with_mul", [(None, False), ("silu", True), ("gelu", False), ("gelu_tanh", True), ("relu", False), (None, True)])
def test_backward(lib, dtype, m, k, n, activation, with_mul):
    x, w, d = make(m, k, n, dtype, m + 2 * k + n)
    x, w = x.to(TYPES[dtype]), w.to(TYPES[dtype])
    mul = d["mul"] if with_mul else None
    z = lib.psrl_linear_fwd(x, w, bias=d["bias"], want_z=True)[1] if activation or with_mul else None
    got = check_bwd(lib, x, w, d, z, activation, mul, dtype)
    assert (got[3] is None) == (mul is None)
    # one at a time, the same bits
    for want in ((True, False, False, False), (False, True, False, False), (False, False, True, False), (False, False, False, mul is not None)):
        one = lib.psrl_linear_bwd(x, w, d["d_y"], z=z, activation=activation, mul=mul, want_x=want[0], want_weight=want[1], want_bias=want[2], want_mul=want[3])
        for a, b, on in zip(one, got, want):
            assert (a is None and not on) or torch.equal(a, b)


def test_d_mul_needs_z_only_there(lib):
    x, w, d = make(50, 64, 72, "bf16", 0)
    x, w = x.to(torch.bfloat16), w.to(torch.bfloat16)
    check_bwd(lib, x, w, d, None, None, d["mul"], "bf16", want_mul=False)
    with pytest.raises(lib.PsrlError):
        lib.psrl_linear_bwd(x, w, d["d_y"], mul=d["mul"])
    with pytest.raises(lib.PsrlError):
        lib.psrl_linear_bwd(x, w, d["d_y"], activation="silu")


@pytest.mark.parametrize("m,k,n", [(5, 4096, 4096), (300, 512, 776), (3000, 256, 1024)])
def test_gradient_against_differences(lib, m, k, n):
    """fp32, along the gradient.  The loss is a sum of y d_y, each y within E = (K + 8) 2^-24 S + 2^-20 max(|z|, 1), so the quotient of a
    step s is within sum E |mul d_y| / s of the slope there, and the slope's own change over the step, |d_x|^2 s times the curvature of
    silu (below 1/2) times |w|^2: the step is chosen so that no z moves by more than 2^-7, the third derivative then adds 2^-14 / 6."""
    x, w, d = make(m, k, n, "f32", 9)
    z = lib.psrl_linear_fwd(x, w, bias=d["bias"], want_z=True)[1]
    dx, dw, db, dm = lib.psrl_linear_bwd(x, w, d["d_y"], z=z, activation="silu", mul=d["mul"], want_bias=True)
    loss = lambda **kw: (lib.psrl_linear_fwd(activation="silu", **{**dict(x=x, weight=w, bias=d["bias"], mul=d["mul"], residual=d["residual"]), **kw})[0].double()
                         * d["d_y"].double()).sum().item()
    size = x.double().abs() @ w.double().abs().T
    error = (((k + 8) * 2.0 ** -24 * size + 2.0 ** -20 * z.double().abs().clamp(min=1.0)) * (d["mul"] * d["d_y"]).double().abs()).sum().item()
    for name, value, grad in (("x", x, dx), ("weight", w, dw), ("bias", d["bias"], db), ("mul", d["mul"], dm)):
        moved = {"x": lambda: (dx @ w.T), "weight": lambda: (x @ dw.T), "bias": lambda: db[None], "mul": lambda: dm}[name]().abs().max().item()
        s = 2.0 ** -7 / moved
        up, down = (value.double() + s * grad.double()).float(), (value.double() - s * grad.double()).float()
        real = ((up.double() - down.double()) / (2 * s) * grad.double()).sum().item()
        slope = (loss(**{name: up}) - loss(**{name: down})) / (2 * s)
        assert abs(slope - real) <= error / s + 2.0 ** -12 * abs(real), name


def test_values_that_are_not_numbers_stay_in_their_rows(lib):
    x, w, d = make(300, 256, 520, "bf16", 4)
    x, w = x.to(torch.bfloat16), w.to(torch.bfloat16)
    want = lib.psrl_linear_fwd(x, w, bias=d["bias"], activation="gelu", residual=d["residual"], mul=d["mul"])[0]
    x[17, 3], x[200, 255], x[201, 0] = float("nan"), float("inf"), -float("inf")
    got = lib.psrl_linear_fwd(x, w, bias=d["bias"], activation="gelu", residual=d["residual"], mul=d["mul"])[0]
    rest = [i for i in range(300) if i not in (17, 200, 201)]
    assert torch.equal(got[rest], want[rest]) and torch.isnan(got[17]).all()
    for act in ACTS:   # slopes far out: 0 on one side, 1 (or what the definition gives) on the other, for z of any size
        z = torch.tensor([[-3e38, -1e20, -1e4, -200.0, 200.0, 1e4, 1e20, 3e38]], device="cuda", dtype=torch.bfloat16)
        one = torch.ones_like(z)
        dz = lib.psrl_linear_bwd(torch.zeros(1, 8, device="cuda", dtype=torch.bfloat16), torch.eye(8, device="cuda", dtype=torch.bfloat16), one, z=z, activation=act,
                                 want_weight=False)[0]
        assert dz.tolist() == [[0.0 if act else 1.0] * 4 + [1.0] * 4], (act, dz)
    for act in ACTS:   # large logits on both sides
        big = lib.psrl_linear_fwd((x[:16] * 1e4), w, activation=act)[0]
        z = to_np(x[:16] * 1e4) @ to_np(w).T
        within(big, oracle_act(z, act)[0], 2.0 ** -10 * np.abs(z).max() * np.ones_like(z), act)


def test_slices_in_place_streams_graphs(lib):
    x, w, d = make(333, 512, 264, "bf16", 5)
    x, w = x.to(torch.bfloat16), w.to(torch.bfloat16)
    want = lib.psrl_linear_fwd(x, w, bias=d["bias"], activation="silu", mul=d["mul"], residual=d["residual"], want_z=True)
    # slices of wider matrices
    wide_x, wide_w = torch.full((333, 1040), float("nan"), device="cuda", dtype=torch.bfloat16), torch.full((264, 528), float("nan"), device="cuda", dtype=torch.bfloat16)
    wide_x[:, 16:528], wide_w[:, :512] = x, w
    out = torch.full((335, 800), 7.0, device="cuda", dtype=torch.bfloat16)
    got = lib.psrl_linear_fwd(wide_x[:, 16:528], wide_w[:, :512], bias=d["bias"], activation="silu", mul=d["mul"], residual=d["residual"], y=out[1:334, 8:272],
                              z=out[1:334, 400:664], want_z=True)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    keep = torch.ones_like(out, dtype=torch.bool)
    keep[1:334, 8:272] = keep[1:334, 400:664] = False
    assert (out[keep] == 7.0).all()
    # the residual stream updated in place, z over mul
    a, b = d["residual"].clone(), d["mul"].clone()
    got = lib.psrl_linear_fwd(x, w, bias=d["bias"], activation="silu", mul=b, residual=a, y=a, z=b, want_z=True)
    assert got[0] is a and got[1] is b and torch.equal(a, want[0]) and torch.equal(b, want[1])
    grads = lib.psrl_linear_bwd(x, w, d["d_y"], z=want[1], activation="silu", mul=d["mul"], want_bias=True)
    for over in ("d_y", "mul", "z"):
        kw = dict(d_y=d["d_y"].clone(), mul=d["mul"].clone(), z=want[1].clone())
        got = lib.psrl_linear_bwd(x, w, activation="silu", want_bias=True, d_mul=kw[over], **kw)
        assert all(torch.equal(p, q) for p, q in zip(got, grads)), over
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = lib.psrl_linear_fwd(x, w, bias=d["bias"], activation="silu", mul=d["mul"], residual=d["residual"], want_z=True, stream=side)
    got_g = lib.psrl_linear_bwd(x, w, d["d_y"], z=got[1], activation="silu", mul=d["mul"], want_bias=True, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for p, q in zip((*got, *got_g), (*want, *grads)))
    # captured twice with workspaces of their own, replayed on new inputs
    ws = [lib.Workspace(lib.psrl_linear_workspace_bytes(333, 512, 264, True)) for _ in range(2)]
    outs = [[torch.empty_like(t) for t in grads] for _ in range(2)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for o, k in zip(outs, ws):
            lib.psrl_linear_bwd(x, w, d["d_y"], z=want[1], activation="silu", mul=d["mul"], want_bias=True, d_x=o[0], d_weight=o[1], d_bias=o[2], d_mul=o[3], workspace=k)
    x.mul_(0.5)
    d["d_y"].mul_(-2.0)
    grads = lib.psrl_linear_bwd(x, w, d["d_y"], z=want[1], activation="silu", mul=d["mul"], want_bias=True)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for o in outs for p, q in zip(o, grads)) and all(k.status() == 0 for k in ws)
    work = lib.Workspace(256)
    lib.psrl_linear_fwd(x, w, workspace=work)
    assert work.status() == 0


@pytest.mark.parametrize("m", [5, 300])
def test_order_on_a_stream(lib, m):
    """Kernels that may start early still see what is before them on their stream, and nothing behind them starts early: chains of
    products over a memset, a copy and another stream's work, eager and captured."""
    x, w, d = make(m, 512, 512, "bf16", 8)
    x, w = x.to(torch.bfloat16), w.to(torch.bfloat16)
    norm = torch.ones(512, device="cuda", dtype=torch.bfloat16)
    side = torch.cuda.Stream()
    one, two, out = (torch.empty(m, 512, device="cuda", dtype=torch.bfloat16) for _ in range(3))

    def chain():
        one.zero_()                                                             # a memset right before
        lib.psrl_linear_fwd(one, w, residual=x, y=two)                          # = x
        one.copy_(two)
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            lib.psrl_rms_norm_fwd(one, norm, y=one)                             # on another stream, joined again
            lib.psrl_linear_fwd(one, w, y=two, activation="silu")
        torch.cuda.current_stream().wait_stream(side)
        for _ in range(6):                                                      # each needs all of the one before
            lib.psrl_linear_fwd(two, w, y=one, residual=x)
            lib.psrl_rms_norm_fwd(one, norm, y=two)
        lib.psrl_linear_bwd(two, w, one, d_x=out, want_weight=False)
        two.zero_()                                                             # must not reach the product before

    chain()
    torch.cuda.synchronize()
    want = out.clone()
    h = lib.psrl_rms_norm_fwd(x, norm)[0]
    h = lib.psrl_linear_fwd(h, w, activation="silu")[0]
    for _ in range(6):
        torch.cuda.synchronize()
        o = lib.psrl_linear_fwd(h, w, residual=x)[0]
        torch.cuda.synchronize()
        h = lib.psrl_rms_norm_fwd(o, norm)[0]
    torch.cuda.synchronize()
    assert torch.equal(lib.psrl_linear_bwd(h, w, o, want_weight=False)[0], want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        chain()
    for _ in range(5):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_no_rows_and_refusals(lib):
    x, w, d = make(6, 128, 72, "bf16", 6)
    x, w = x.to(torch.bfloat16), w.to(torch.bfloat16)
    y, z = lib.psrl_linear_fwd(x[:0], w, want_z=True)
    assert y.shape == z.shape == (0, 72)
    dx, dw, db, _ = lib.psrl_linear_bwd(x[:0], w, d["d_y"][:0], want_bias=True)
    assert dx.shape == (0, 128) and not dw.any() and not db.any()
    codes, scales = lib.psrl_quantize_rows(x)
    for bad in (dict(weight=w[:, :64]), dict(x=x[0]), dict(bias=d["bias"][:70]), dict(bias=d["bias"].float()), dict(mul=d["mul"][:5]), dict(residual=d["residual"].float()),
                dict(activation="tanh"), dict(x_scale=scales), dict(y=d["mul"][:, :64]), dict(x=x.T.contiguous().T), dict(mul=d["mul"].cpu()),
                dict(x=codes, weight=codes), dict(x=codes, weight=codes, x_scale=scales, weight_scale=scales[:5])):
        with pytest.raises(ValueError):
            lib.psrl_linear_fwd(**{**dict(x=x, weight=w), **bad})
    for bad in (dict(weight=w.float()), dict(x=x.half(), weight=w.half())):
        with pytest.raises(TypeError):
            lib.psrl_linear_fwd(**{**dict(x=x, weight=w), **bad})
    with pytest.raises(TypeError):
        lib.psrl_linear_bwd(codes, codes, torch.zeros(6, 6, device="cuda", dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        lib.psrl_linear_bwd(x, w, d["d_y"], want_mul=True)
    with pytest.raises(lib.PsrlError) as e:
        lib.psrl_linear_bwd(x, w, d["d_y"], z=d["mul"], activation="silu", workspace=lib.Workspace(256))
    assert e.value.name == "PSRL_ERR_WORKSPACE"
    with pytest.raises(lib.PsrlError) as e:      # a slice that starts off a 16-byte boundary
        lib.psrl_linear_fwd(torch.cat([x.view(-1), x.view(-1)])[4:4 + 768].view(6, 128), w)
    assert e.value.name == "PSRL_ERR_INVALID_ARG"
    with pytest.raises(RuntimeError):
        lib.psrl_linear_fwd(x.cpu(), w.cpu())

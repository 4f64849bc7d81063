"""Matrix products with their epilogue, host side: the oracle against closed forms and differences, workspaces, refusals."""
import ctypes

import numpy as np
import pytest

from oracle.layer import oracle_act, oracle_linear, oracle_linear_bwd

ACTS = [None, "relu", "silu", "gelu", "gelu_tanh"]


@pytest.mark.parametrize("activation", ACTS)
def test_oracle_slopes_and_gradients(activation):
    z = np.linspace(-6, 6, 241) + 0.0013
    h = 1e-6
    assert np.allclose((oracle_act(z + h, activation)[0] - oracle_act(z - h, activation)[0]) / (2 * h), oracle_act(z, activation)[1], atol=1e-8)
    rng = np.random.default_rng(1)
    x, w, b, mul, res, dy = (rng.normal(size=s) for s in ((4, 6), (5, 6), (5,), (4, 5), (4, 5), (4, 5)))
    y, zz = oracle_linear(x, w, b, activation, mul, res)
    dx, dw, db, dm = oracle_linear_bwd(x, w, dy, zz, activation, mul)
    loss = lambda **k: (oracle_linear(**{**dict(x=x, weight=w, bias=b, activation=activation, mul=mul, residual=res), **k})[0] * dy).sum()
    for name, value, grad in (("x", x, dx), ("weight", w, dw), ("bias", b, db), ("mul", mul, dm)):
        d = rng.normal(size=value.shape)
        assert abs((loss(**{name: value + h * d}) - loss(**{name: value - h * d})) / (2 * h) - (grad * d).sum()) < 1e-6


def test_oracle_pins():
    assert np.allclose(oracle_act(np.array([-1e9, 0.0, 1e9]), "silu")[0], [0, 0, 1e9])
    assert abs(oracle_act(1.0, "gelu")[0] - 0.8413447460685429) < 1e-15 and abs(oracle_act(1.0, "gelu_tanh")[0] - 0.8411919906082768) < 1e-12
    assert oracle_act(np.array([-2.0, 0.0, 3.0]), "relu")[1].tolist() == [0, 0, 1]


def test_workspace_bytes(lib):
    size = lib.psrl_linear_workspace_bytes
    assert size(0, 8, 8, False) == size(0, 8, 8, True) == 256 and size(-1, 8, 8, True) == size(1, 0, 8, True) == size(1, 8, 0, False) == 0
    for m in (1, 777, 8192):
        for n in (1, 1000, 14336):
            for dtype, es in (("bf16", 2), ("f32", 4)):
                more = 20 << 20 if dtype == "f32" else 0
                assert size(m, 4096, n, True, dtype) <= 256 + 512 + es * m * (n + 7) + 4 * n * (-(-m // 64)) + more
                assert size(m, 4096, n, False, dtype) <= 256 + more and size(m, 4096, n, False, "e4m3") == 256


def test_refusals(lib):
    L = lib.lib()
    buf = ctypes.create_string_buffer(1 << 16)
    p = (ctypes.addressof(buf) + 255) // 256 * 256
    q, r, t, u, v = (p + 4096 * i for i in range(1, 6))
    name = lambda st: lib.STATUS_NAMES[st]
    fwd = lambda **k: name(L.psrl_linear_fwd(*{**dict(dt=1, m=2, k=64, n=24, x=p, xp=64, xs=None, w=q, wp=64, ws=None, b=None, act=0, mul=None, mp=0, res=None,
                                                      rp=0, y=r, yp=24, z=None, zp=0, work=t, wb=1 << 12, stream=None), **k}.values()))
    for bad in (dict(dt=3), dict(dt=-1)):
        assert fwd(**bad) == "PSRL_ERR_UNSUPPORTED"
    for bad in (dict(m=-1), dict(m=2 ** 31), dict(act=5), dict(act=-1), dict(x=None), dict(x=p + 8), dict(w=None), dict(w=q + 2), dict(y=None), dict(y=r + 4),
                dict(b=u + 8), dict(mul=u + 2, mp=24), dict(res=u + 2, rp=24), dict(z=u + 8, zp=24), dict(z=r, zp=24), dict(dt=0, m=2, k=4096, xp=4096, wp=4096, work=None), dict(work=t + 128),
                dict(xs=u), dict(ws=u), dict(dt=2), dict(dt=2, xs=u), dict(dt=2, xs=u, ws=v + 2), dict(res=r, rp=32), dict(mul=r, mp=32), dict(mul=u, mp=24, z=u, zp=32)):
        assert fwd(**bad) == "PSRL_ERR_INVALID_ARG", bad
    for bad in (dict(k=60), dict(k=0), dict(k=4), dict(n=0), dict(n=-8), dict(xp=56), dict(xp=68), dict(wp=48), dict(yp=16), dict(yp=28), dict(mul=u, mp=16),
                dict(res=u, rp=30), dict(z=u, zp=0), dict(dt=2, xs=u, ws=u, xp=72), dict(n=2 ** 31 - 1)):
        assert fwd(**bad) == "PSRL_ERR_SHAPE", bad
    assert fwd(wb=255) == "PSRL_ERR_WORKSPACE" and fwd(m=0, work=None, wb=0) == "PSRL_OK"
    bwd = lambda **k: name(L.psrl_linear_bwd(*{**dict(dt=1, m=2, k=64, n=24, x=p, xp=64, w=q, wp=64, z=None, zp=0, act=0, mul=None, mp=0, dy=r, dyp=24, dx=t, dxp=64,
                                                      dw=u, dwp=64, db=None, dm=None, dmp=0, work=v, wb=1 << 12, stream=None), **k}.values()))
    for bad in (dict(dt=2), dict(dt=7)):
        assert bwd(**bad) == "PSRL_ERR_UNSUPPORTED"
    for bad in (dict(act=2), dict(dm=r, dmp=24), dict(dm=r, dmp=24, mul=p, mp=24), dict(dm=r, dmp=24, z=p, zp=24), dict(dy=None), dict(dy=r + 4), dict(dx=t + 2),
                dict(dw=u + 2), dict(db=u + 2), dict(z=p + 2, zp=24), dict(work=v + 4), dict(work=None, db=p), dict(work=None, act=1, z=p, zp=24), dict(m=-1), dict(mul=p, mp=24, z=q, zp=24, dm=r, dmp=32)):
        assert bwd(**bad) == "PSRL_ERR_INVALID_ARG", bad
    for bad in (dict(dyp=20), dict(dxp=56), dict(dwp=60), dict(z=p, zp=8), dict(mul=p, mp=28), dict(k=12)):
        assert bwd(**bad) == "PSRL_ERR_SHAPE", bad
    assert bwd(act=1, z=p, zp=24, wb=256 + 95) == bwd(db=p, wb=256 + 95) == bwd(wb=255) == "PSRL_ERR_WORKSPACE"

"""Root-mean-square norms, host side: the oracle against closed forms and differences, workspaces, refusals."""
import ctypes

import numpy as np
import pytest

from oracle.layer import oracle_rms, oracle_rms_bwd


def test_oracle_pins():
    rng = np.random.default_rng(0)
    h, w, dy, ds = rng.normal(size=(3, 16)), rng.normal(size=16), rng.normal(size=(3, 16)), rng.normal(size=(3, 16))
    y, r = oracle_rms(np.full((1, 4), 3.0), np.array([1.0, 2.0, 3.0, 4.0]), 0.0)
    assert np.allclose(y, [[1, 2, 3, 4]]) and np.allclose(r, 1 / 3)
    assert np.allclose(oracle_rms(2.0 ** 60 * h, w, 1e-6)[0], oracle_rms(h, w, 0.0)[0])
    loss = lambda h, w: (oracle_rms(h, w, 1e-3)[0] * dy).sum() + (h * ds).sum()
    dh, dw = oracle_rms_bwd(h, w, dy, 1e-3, ds)
    step = 1e-6
    for at in [(0, 0), (1, 7), (2, 15)]:
        e = np.zeros_like(h)
        e[at] = step
        assert abs((loss(h + e, w) - loss(h - e, w)) / (2 * step) - dh[at]) < 1e-8
    e = np.zeros(16)
    e[5] = step
    assert abs((loss(h, w + e) - loss(h, w - e)) / (2 * step) - dw[5]) < 1e-8


def test_workspace_bytes(lib):
    size = lib.psrl_rms_norm_workspace_bytes
    assert size(0, 1, 4096) == 256 and size(5, 1, 12) == 0 and size(-1, 1, 64) == 0 and size(1, 0, 64) == 0
    for dtype in ("bf16", "f32"):
        for dim in (8, 64, 80, 264, 1024, 4096, 5120, 8192, 16384, 32768):
            for rows in (1, 7, 1000, 10 ** 6):
                # at most a row of sums for each of the blocks that the SMs hold, and for each row
                assert 256 + 4 * dim <= size(rows, 1, dim, dtype) <= 256 + 4 * dim * min(rows, 148 * 8)


def test_refusals(lib):
    L = lib.lib()
    buf = ctypes.create_string_buffer(1 << 16)
    p = (ctypes.addressof(buf) + 255) // 256 * 256
    q, r, t = p + 8192, p + 16384, p + 24576
    name = lambda st: lib.STATUS_NAMES[st]
    fwd = lambda **k: name(L.psrl_rms_norm_fwd(*{**dict(dt=1, n=2, heads=1, dim=64, x=p, xp=64, res=None, rp=0, w=q, eps=1e-6, sum=None, sp=0, y=r,
                                                        yp=64, c=None, cp=0, s=None, stream=None), **k}.values()))
    assert fwd(n=0) == "PSRL_OK" and fwd(n=0, x=None, y=None) == "PSRL_OK"
    assert fwd(dt=2) == "PSRL_ERR_UNSUPPORTED"
    for bad in (dict(n=-1), dict(heads=0), dict(heads=65536), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")),
                dict(x=None), dict(x=p + 8), dict(w=q + 4), dict(y=r + 2), dict(res=q, rp=64, sum=r, sp=64), dict(c=t, cp=64), dict(s=t),
                dict(c=t + 8, cp=64, s=q), dict(c=t, cp=64, s=q + 2), dict(y=p, yp=128), dict(res=q, rp=64, sum=p, sp=72), dict(res=q, rp=72, sum=q, sp=64)):
        assert fwd(**bad) == "PSRL_ERR_INVALID_ARG", bad
    for bad in (dict(dim=60), dict(dim=0), dict(dim=32776, xp=32776, yp=32776), dict(xp=63), dict(xp=68), dict(yp=56), dict(res=q, rp=60),
                dict(res=q, rp=64, sum=t, sp=0), dict(c=t, cp=72, s=q), dict(heads=2), dict(n=0, xp=12)):
        assert fwd(**bad) == "PSRL_ERR_SHAPE", bad
    bwd = lambda **k: name(L.psrl_rms_norm_bwd(*{**dict(dt=0, n=2, heads=1, dim=64, h=p, hp=64, w=q, eps=1e-6, dy=r, dyp=64, ds=None, dsp=0, dx=t, dxp=64,
                                                        dw=q + 4096, ws=p + 32768, wsb=1 << 14, stream=None), **k}.values()))
    assert bwd(wsb=256 + 256 - 1) == bwd(wsb=0, dw=None) == bwd(n=0, wsb=255, dw=None) == "PSRL_ERR_WORKSPACE"
    assert bwd(n=0, ws=None, wsb=0, dw=None) == "PSRL_OK"
    assert bwd(dt=5) == "PSRL_ERR_UNSUPPORTED"
    for bad in (dict(h=None), dict(dy=None), dict(ws=None), dict(ws=p + 32768 + 16), dict(w=None), dict(dw=q + 4098), dict(eps=0.0), dict(dx=r, dxp=72),
                dict(dx=p, dxp=128), dict(ds=t, dsp=68)):
        assert bwd(**bad) == "PSRL_ERR_INVALID_ARG", bad
    for bad in (dict(dim=36), dict(hp=62), dict(dyp=66), dict(ds=t, dsp=32), dict(dxp=0)):
        assert bwd(**bad) == "PSRL_ERR_SHAPE", bad
    quant = lambda **k: name(L.psrl_quantize_rows(*{**dict(dt=1, n=2, dim=64, x=p, xp=64, c=q, cp=64, s=r, stream=None), **k}.values()))
    assert quant(n=0) == "PSRL_OK" and quant(dt=9) == "PSRL_ERR_UNSUPPORTED"
    assert quant(x=None) == quant(c=None) == quant(s=None) == quant(s=r + 1) == quant(n=-3) == "PSRL_ERR_INVALID_ARG"
    assert quant(cp=72) == quant(xp=32) == quant(dim=65) == "PSRL_ERR_SHAPE"

"""Codes of 8 bits over the rows that they are made of."""
import ctypes

import pytest


def test_refusals(lib):
    """Codes whose rows would reach into rows (or heads) that are still to be read, and two outputs in one place."""
    L = lib.lib()
    buf = ctypes.create_string_buffer(1 << 16)
    x = (ctypes.addressof(buf) + 255) // 256 * 256
    r, s, y, c, t = (x + 8192 * i for i in range(1, 6))
    name = lambda st: lib.STATUS_NAMES[st]
    norm = lambda **k: name(L.psrl_rms_norm_fwd(*{**dict(dt=1, n=2, heads=1, dim=64, x=x, xp=64, res=r, rp=64, w=None, eps=1e-6, sum=s, sp=64, y=y, yp=64, codes=c, cp=128,
                                                       scales=t, stream=None), **k}.values()))
    for bad in (dict(codes=x, cp=64), dict(codes=x, cp=256), dict(codes=r, cp=64), dict(codes=r, rp=128), dict(codes=x, dt=0), dict(codes=x, heads=2, xp=128, rp=128, sp=128, yp=128, cp=256),
                dict(codes=y), dict(codes=s), dict(codes=x, n=1, heads=2, xp=128, rp=128, sp=128, yp=128)):
        assert norm(**bad) == "PSRL_ERR_INVALID_ARG", bad
    rows = lambda **k: name(L.psrl_quantize_rows(*{**dict(dt=1, n=2, dim=64, x=x, xp=64, codes=c, cp=64, scales=t, stream=None), **k}.values()))
    for bad in (dict(codes=x), dict(codes=x, dt=0), dict(codes=x, cp=256)):
        assert rows(**bad) == "PSRL_ERR_INVALID_ARG", bad


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,dim", [(1, 64), (5, 128), (700, 512), (1003, 3000), (4, 8200)])
def test_in_place(lib, dtype, rows, dim):
    import torch

    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    pitch = -(-dim // 16) * 16
    x, res = (torch.randn(rows, pitch, device="cuda").to(t)[:, :dim] for _ in range(2))
    w = torch.randn(dim, device="cuda").to(t)
    same = lambda a, b: torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))
    over = lambda v: v.view(torch.float8_e4m3fn)[:, :dim]
    codes, scales = lib.psrl_quantize_rows(x)
    a = torch.empty(rows, pitch, device="cuda", dtype=t)[:, :dim].copy_(x)
    full = a.as_strided((rows, pitch), (pitch, 1))
    got = lib.psrl_quantize_rows(a, codes=over(full))
    assert same(got[0], codes) and torch.equal(got[1], scales)
    y, summed, codes, scales = lib.psrl_rms_norm_fwd(x, w, residual=res, want_codes=True)
    for which in (0, 1):
        v = [torch.empty(rows, pitch, device="cuda", dtype=t)[:, :dim].copy_(u) for u in (x, res)]
        full = v[which].as_strided((rows, pitch), (pitch, 1))
        got = lib.psrl_rms_norm_fwd(v[0], w, residual=v[1], want_codes=True, codes=over(full))
        assert same(got[0], y) and same(got[1], summed) and same(got[2], codes) and torch.equal(got[3], scales)

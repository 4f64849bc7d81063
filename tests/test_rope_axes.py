"""Rotary positions with several axes, host side: sections, the one-axis form unchanged, refusals."""
import ctypes

import numpy as np
import pytest

from oracle.layer import oracle_axes, oracle_rope_axes
from oracle.rope import oracle_rope, oracle_rope_frequencies


def test_oracle_pins():
    assert oracle_axes([2, 1, 3], "blocks").tolist() == [0, 0, 1, 2, 2, 2]
    assert oracle_axes([3, 2, 1], "cyclic").tolist() == [0, 1, 2, 0, 1, 0]
    assert [oracle_axes([24, 20, 20], "cyclic").tolist().count(a) for a in range(3)] == [24, 20, 20]
    # one position on every axis is the ordinary rotation; a pair only sees its own axis
    x = np.random.default_rng(0).normal(size=(7, 2, 16))
    freq, _ = oracle_rope_frequencies(16, 10000.0)
    pos = np.arange(7) * 11
    axis = oracle_axes([3, 3, 2], "blocks")
    assert np.allclose(oracle_rope_axes(x, [pos] * 3, axis, freq, 1.5), oracle_rope(x, pos, freq, 1.5))
    a, b = (oracle_rope_axes(x, [pos, p, pos], axis, freq, 1.0) for p in (pos, pos + 5))
    same = np.isin(np.arange(16) % 8, [3, 4, 5])
    assert np.array_equal(a[..., ~same], b[..., ~same]) and not np.allclose(a[..., same], b[..., same])


def test_sections(lib):
    for sections, order in (([16, 24, 24], "blocks"), ([24, 20, 20], "cyclic"), ([0, 64, 0], "blocks"), ([64], "blocks"), ([64], "cyclic"),
                            ([32, 32], "cyclic"), ([0, 0, 0, 64], "blocks"), ([16, 16, 16, 16], "cyclic"), ([64, 0, 0], "cyclic")):
        rope = lib.Rope(128, sections=sections, order=order)
        assert rope.n_axes == len(sections) and np.array_equal(rope.freq, lib.Rope(128).freq) and rope.scale == 1.0
    for sections, order in (([16, 24, 23], "blocks"), ([16, 24, 25], "blocks"), ([-1, 65], "blocks"), ([20, 24, 20], "cyclic"),
                            ([0, 32, 32], "cyclic"), ([65, 0, -1], "cyclic"), ([2 ** 31 - 1, 2 ** 31 - 1, 66], "blocks")):
        with pytest.raises(lib.PsrlError) as e:
            lib.Rope(128, sections=sections, order=order)
        assert e.value.name == "PSRL_ERR_SHAPE", sections
    for sections in ([], [16, 16, 16, 8, 8]):
        with pytest.raises(lib.PsrlError) as e:
            lib.Rope(128, sections=sections)
        assert e.value.name == "PSRL_ERR_INVALID_ARG"
    with pytest.raises(ValueError):
        lib.Rope(128, sections=[64], order="other")
    with pytest.raises(lib.PsrlError) as e:      # the dimensions are looked at first, as in the one-axis form
        lib.Rope(12, sections=[6])
    assert e.value.name == "PSRL_ERR_SHAPE"


def test_refusals(lib):
    L, plan, rope = lib.lib(), lib.Plan([-1, 0], [20, 5], [16], 2, 1, 64, "f32"), lib.Rope(64, sections=[12, 10, 10])
    buf = ctypes.create_string_buffer(8192)
    p = (ctypes.addressof(buf) + 255) // 256 * 256
    name = lambda st: lib.STATUS_NAMES[st]
    fwd = lambda *a: name(L.psrl_rope_axes_qkv_fwd(*a))
    good = [plan.handle, rope._h, p, 25, p, 128, p, 64, p, 64, p, p, p, 64, None]
    change = lambda i, v: good[:i] + [v] + good[i + 1:]
    assert fwd(*good) == fwd(*change(3, 1000)) == "PSRL_ERR_WORKSPACE"           # accepted: only the upload is missing
    assert fwd(*change(2, None)) == fwd(*change(2, p + 2)) == "PSRL_ERR_INVALID_ARG"
    assert fwd(*change(3, 24)) == fwd(*change(3, -1)) == fwd(*change(5, 64)) == "PSRL_ERR_SHAPE"
    bwd = lambda *a: name(L.psrl_rope_axes_qkv_bwd(*a))
    good = [plan.handle, rope._h, p, 25, p, p, p, 64, p, 128, p, 64, p, 64, None]
    assert bwd(*good) == "PSRL_ERR_WORKSPACE"
    assert bwd(*change(2, None)) == "PSRL_ERR_INVALID_ARG" and bwd(*change(3, 24)) == "PSRL_ERR_SHAPE"
    rows = lambda *a: name(L.psrl_rope_axes_rows(*a))
    good = [rope._h, 0, p, 64, p, 3, 3, 1, p, 64, 0, None]
    assert rows(*change(5, 2)) == "PSRL_ERR_SHAPE"
    assert rows(*change(4, None)) == rows(*change(6, -1)) == rows(*change(7, 0)) == "PSRL_ERR_INVALID_ARG"
    assert rows(*change(1, 5)) == "PSRL_ERR_UNSUPPORTED"
    assert rows(*change(6, 0)) == "PSRL_OK"

"""Rotary positions, host side: frequencies against the oracle's, the plan's positions and slots of the query rows, refusals."""
import ctypes
import os
import subprocess
import sys

import numpy as np
import pytest

from oracle import oracle_plan
from oracle.rope import oracle_rope, oracle_rope_frequencies
from paper_2608_25683_b200.workloads import random_forest

from test_schedule import decode


@pytest.mark.parametrize("head_dim,rotary", [(64, 64), (128, 128), (128, 32), (128, 6), (256, 256), (8, 2)])
@pytest.mark.parametrize("scaling,kw", [
    (None, {}), ("linear", dict(factor=4.0)), ("ntk", dict(factor=8.0)),
    ("yarn", dict(factor=4.0, original_positions=4096)), ("yarn", dict(factor=40.0, original_positions=100, low=2.0, high=9.0)),
    ("banded", dict(factor=8.0, original_positions=8192)),
    ("banded", dict(factor=2.0, original_positions=64, low=0.5, high=3.0, attention_scale=1.25)),
])
def test_frequencies_match_oracle(lib, head_dim, rotary, scaling, kw):
    if scaling == "ntk" and rotary == 2:
        with pytest.raises(lib.PsrlError):
            lib.Rope(head_dim, rotary, scaling=scaling, **kw)
        return
    rope = lib.Rope(head_dim, rotary, base=10000.0, scaling=scaling, **kw)
    freq, scale = oracle_rope_frequencies(rotary, 10000.0, scaling, **kw)
    # a handful of fp64 operations each: 2^-53 apiece, the power loses the logarithm's size more
    assert np.allclose(rope.freq, freq, rtol=1e-13, atol=0) and abs(rope.scale - scale) <= 1e-14 * scale


def test_oracle_pins():
    """The oracle against closed forms: a quarter turn, norms kept, inverse, positions add up, layouts are permutations."""
    x = np.random.default_rng(0).normal(size=(5, 3, 8))
    f = np.array([np.pi / 2, 0.1])
    y = oracle_rope(x, [1] * 5, f, 1.0)
    assert np.allclose(y[..., 0], -x[..., 2]) and np.allclose(y[..., 2], x[..., 0]) and np.array_equal(y[..., 4:], x[..., 4:])
    freq, _ = oracle_rope_frequencies(8, 10000.0)
    assert np.allclose(freq, [1.0, 0.1, 0.01, 0.001])
    pos = np.array([0, 1, 7, 1000, 10 ** 6])
    y = oracle_rope(x, pos, freq, 1.0)
    assert np.allclose(np.linalg.norm(y, axis=-1), np.linalg.norm(x, axis=-1)) and np.array_equal(y[0], x[0])
    assert np.allclose(oracle_rope(y, pos, freq, 1.0, inverse=True), x)
    assert np.allclose(oracle_rope(oracle_rope(x, pos, freq, 1.0), pos, freq, 1.0), oracle_rope(x, 2 * pos, freq, 1.0))
    swap = np.array([0, 4, 1, 5, 2, 6, 3, 7])
    assert np.allclose(oracle_rope(x[..., swap], pos, freq, 1.0, "interleaved"), y[..., swap])


def test_plan_positions_and_slots_of_query_rows(lib):
    rng = np.random.default_rng(3)
    for it in range(20):
        parent, seg_len, gbs, flags = random_forest(rng, int(rng.integers(2, 14)), 90, 1 + it % 2, cached_roots=it % 3 == 0)
        plan = lib.Plan(parent, seg_len, gbs, 4, 2, 128, "bf16", seg_flags=flags)
        V = oracle_plan(parent, seg_len, gbs, flags)
        w = plan.schedule()
        H = decode(plan)["H"]
        pos, slot = (w[H[k]:H[k] + V["T_q"]] for k in ("off_qrow_pos", "off_qrow_slot"))
        for c in range(V["n_seg"]):
            if V["seg_q_off"][c] < 0:
                continue
            r, t, n = int(V["seg_q_off"][c]), int(V["seg_tok_off"][c]), int(V["seg_len"][c])
            assert np.array_equal(pos[r:r + n], V["seg_anc_tokens"][c] + np.arange(n))
            assert np.array_equal(slot[r:r + n], V["tok_slot"][t:t + n])


def test_refusals(lib):
    for kw, name in [
        (dict(head_dim=12), "SHAPE"), (dict(head_dim=0), "SHAPE"), (dict(head_dim=264), "SHAPE"),
        (dict(head_dim=64, rotary_dim=7), "SHAPE"), (dict(head_dim=64, rotary_dim=66), "SHAPE"),
        (dict(head_dim=64, base=1.0), "INVALID_ARG"), (dict(head_dim=64, base=float("nan")), "INVALID_ARG"),
        (dict(head_dim=64, scaling="linear", factor=0.0), "INVALID_ARG"),
        (dict(head_dim=64, scaling="yarn", factor=4.0), "INVALID_ARG"),
        (dict(head_dim=64, scaling="yarn", factor=0.5, original_positions=4096), "INVALID_ARG"),
        (dict(head_dim=64, scaling="banded", factor=4.0, original_positions=4096, low=4.0, high=4.0), "INVALID_ARG"),
        (dict(head_dim=64, attention_scale=-1.0), "INVALID_ARG"),
    ]:
        with pytest.raises(lib.PsrlError) as e:
            lib.Rope(**kw)
        assert e.value.name == "PSRL_ERR_" + name, kw
    with pytest.raises(ValueError):
        lib.Rope(64, layout="other")
    L, plan, rope = lib.lib(), lib.Plan([-1, 0], [20, 5], [16], 2, 1, 64, "f32"), lib.Rope(64)
    buf = ctypes.create_string_buffer(4096)
    p = (ctypes.addressof(buf) + 255) // 256 * 256
    fwd = lambda *a: lib.STATUS_NAMES[L.psrl_rope_qkv_fwd(*a)]
    good = [plan.handle, rope._h, p, 128, p, 64, p, 64, p, p, p, 64, None]
    change = lambda i, v: good[:i] + [v] + good[i + 1:]
    assert fwd(*good) == "PSRL_ERR_WORKSPACE"                    # not uploaded
    assert fwd(*change(0, None)) == fwd(*change(1, None)) == "PSRL_ERR_INVALID_ARG"
    assert fwd(*change(2, p + 4)) == fwd(*change(8, None)) == fwd(*change(9, p + 8)) == "PSRL_ERR_INVALID_ARG"
    assert fwd(*change(3, 64)) == fwd(*change(5, 63)) == fwd(*change(7, 66)) == fwd(*change(11, 16)) == "PSRL_ERR_SHAPE"
    assert fwd(*change(1, lib.Rope(128)._h)) == "PSRL_ERR_SHAPE"
    bwd = lambda *a: lib.STATUS_NAMES[L.psrl_rope_qkv_bwd(*a)]
    good = [plan.handle, rope._h, p, p, p, 64, p, 128, p, 64, p, 64, None]
    assert bwd(*good) == "PSRL_ERR_WORKSPACE"
    assert bwd(*change(6, None)) == bwd(*change(3, p + 4)) == "PSRL_ERR_INVALID_ARG"
    assert bwd(*change(5, 31)) == bwd(*change(7, 126)) == "PSRL_ERR_SHAPE"
    rows = lambda *a: lib.STATUS_NAMES[L.psrl_rope_rows(*a)]
    good = [rope._h, 0, p, 64, p, 3, 1, p, 64, 0, None]
    assert rows(*change(1, 7)) == "PSRL_ERR_UNSUPPORTED"
    assert rows(*change(2, None)) == rows(*change(4, None)) == rows(*change(5, -1)) == rows(*change(6, 0)) == rows(*change(6, 65536)) == "PSRL_ERR_INVALID_ARG"
    assert rows(*change(8, 68)) == "PSRL_ERR_INVALID_ARG"        # in place with two pitches
    assert rows(*change(3, 60)) == "PSRL_ERR_SHAPE"
    assert rows(*change(5, 0)) == "PSRL_OK"                      # no rows, nothing launched


def test_in_place_only_with_one_pitch(lib):
    """q_out may be q, and dq_out d_q, where both are contiguous.  With rows further apart on one side a row would be written
    over one that has yet to be read."""
    L, plan, rope = lib.lib(), lib.Plan([-1, 0], [20, 5], [16], 2, 1, 64, "f32"), lib.Rope(64)
    buf = ctypes.create_string_buffer(1 << 16)
    p = (ctypes.addressof(buf) + 255) // 256 * 256
    far = p + 32768
    name = lambda st: lib.STATUS_NAMES[st]
    fwd = lambda q, pitch, out: name(L.psrl_rope_qkv_fwd(plan.handle, rope._h, q, pitch, far, 64, far, 64, out, far, far, 64, None))
    bwd = lambda q, out, pitch: name(L.psrl_rope_qkv_bwd(plan.handle, rope._h, q, far, far, 64, out, pitch, far, 64, far, 64, None))
    assert fwd(p, 128, p) == fwd(p, 256, p + 8192) == "PSRL_ERR_WORKSPACE"      # accepted: only the upload is missing
    assert bwd(p, p, 128) == bwd(p, p + 8192, 256) == "PSRL_ERR_WORKSPACE"
    assert fwd(p, 256, p) == fwd(p, 132, p) == "PSRL_ERR_INVALID_ARG"
    assert bwd(p, p, 256) == bwd(p, p, 132) == "PSRL_ERR_INVALID_ARG"
    one = lib.Plan([-1], [1], [16], 2, 1, 64, "f32")                             # one row has no next one
    assert name(L.psrl_rope_qkv_fwd(one.handle, rope._h, p, 256, far, 64, far, 64, p, far, far, 64, None)) == "PSRL_ERR_WORKSPACE"


def test_handles_that_outlive_the_interpreter(lib):
    """Plans, rotary embeddings and caches held in a module's names until the process ends: nothing is complained about."""
    code = ("import torch\n"
            "from paper_2608_25683_b200 import binding as b\n"
            "kept = [b.Rope(64), b.Plan([-1], [20], [16], 2, 1, 64, 'f32'), b.Cache([-1], [16], [16], [0], 1)]\n"
            "def use(): return b\n")
    out = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert out.returncode == 0 and out.stderr == ""

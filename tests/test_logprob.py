"""Token log-probabilities, host side: the oracle's pins, the tree's next tokens, workspace sizes, refusals."""
import ctypes

import numpy as np
import pytest

from oracle import oracle_plan
from oracle.logprob import oracle_logprob, oracle_next_tokens
from paper_2608_25683_b200.workloads import random_forest


def test_oracle_pins():
    rng = np.random.default_rng(0)
    h, w = rng.normal(size=(5, 6)), rng.normal(size=(11, 6))
    targets, off = np.array([3, 10, 3, 3, -1, 4, 11, 0]), np.array([0, 2, 4, 4, 7, 8])
    g = rng.normal(size=8)
    out = oracle_logprob(h, w, targets, off, 0.7, g)
    assert out["logprob"][4] == out["logprob"][6] == 0.0 and np.all(out["d_hidden"][2] == 0)
    loss = lambda h, w: float(g @ oracle_logprob(h, w, targets, off, 0.7)["logprob"])
    eps = 1e-5
    for x, d in ((h, out["d_hidden"]), (w, out["d_weight"])):
        for i in np.ndindex(x.shape):
            x[i] += eps
            up = loss(h, w)
            x[i] -= 2 * eps
            down = loss(h, w)
            x[i] += eps
            assert abs((up - down) / (2 * eps) - d[i]) < 1e-8
    even = oracle_logprob(np.zeros((1, 6)), w, np.array([2]))
    assert np.isclose(even["lse"][0], np.log(11)) and np.isclose(even["logprob"][0], -np.log(11))


def test_next_tokens_of_the_tree(lib):
    """Against the samples themselves.  (Every segment of these forests lies on a sample.)"""
    rng = np.random.default_rng(9)
    for it in range(30):
        parent, seg_len, gbs, flags = random_forest(rng, int(rng.integers(1, 16)) + 1, 40, 1 + it % 2, cached_roots=it % 3 == 0,
                                                    step_samples=it % 4 == 0)
        plan = lib.Plan(parent, seg_len, gbs, 4, 2, 128, "bf16", seg_flags=flags)
        off, tok = plan.next_tokens()
        want = oracle_next_tokens(oracle_plan(parent, seg_len, gbs, flags))
        assert len(off) == plan.view["T_q"] + 1 and off[0] == 0
        got = {r: sorted(tok[off[r]:off[r + 1]].tolist()) for r in range(len(off) - 1)}
        assert got == want
    plan = lib.Plan([-1, 0], [20, 5], [16], 2, 1, 128, "bf16", seg_flags=[0, 2])     # no query rows
    off, tok = plan.next_tokens()
    assert off.tolist() == [0] and len(tok) == 0
    assert lib.lib().psrl_plan_next_tokens(None, None, None) == 1


def test_workspace_does_not_grow_with_the_vocabulary(lib):
    size = lambda n, h, v, b: lib.psrl_token_logprob_workspace_bytes(n, h, v, n, b)
    assert size(4096, 4096, 1 << 20, True) == size(4096, 4096, 1 << 17, True) <= 8 * 4096 * 4096 * 2
    assert size(200000, 8192, 1 << 17, True) <= 6 * 200000 * 8192 * 2
    assert size(8192, 4096, 1 << 17, False) <= 8192 * 4096
    assert size(0, 64, 10, True) == 256 and size(-1, 64, 10, False) == 0


def test_refusals(lib):
    L = lib.lib()
    buf = ctypes.create_string_buffer(8192)
    p = (ctypes.addressof(buf) + 255) // 256 * 256
    big = 1 << 40
    good = [1, 4, 64, 100, p, 64, p, 64, p, 4, None, 1.0, p, p, p, big, None]
    fwd = lambda *a: lib.STATUS_NAMES[L.psrl_token_logprob_fwd(*a)]
    change = lambda i, v: good[:i + 1] + [v] + good[i + 2:]
    assert fwd(*change(-1, 2)) == "PSRL_ERR_UNSUPPORTED"
    for i, v in [(0, -1), (0, 2 ** 30 + 1), (8, 2 ** 30 + 1), (3, None), (3, p + 8), (5, p + 2), (7, None), (9, p + 2), (10, 0.0), (10, float("nan")),
                 (10, float("inf")), (13, None), (13, p + 16)]:
        assert fwd(*change(i, v)) == "PSRL_ERR_INVALID_ARG", (i, v)
    for i, v in [(1, 60), (1, 0), (2, 0), (2, 2 ** 30 + 1), (4, 56), (4, 68), (6, 63), (8, 5)]:
        assert fwd(*change(i, v)) == "PSRL_ERR_SHAPE", (i, v)
    assert fwd(*change(14, 255)) == "PSRL_ERR_WORKSPACE"
    need = lib.psrl_token_logprob_workspace_bytes(4, 64, 100, 4, True)
    good = [1, 4, 64, 100, p, 64, p, 64, p, 4, None, 1.0, p, p, p, p, 64, p, 64, p, need, None]
    bwd = lambda *a: lib.STATUS_NAMES[L.psrl_token_logprob_bwd(*a)]
    assert bwd(*change(19, need - 1)) == "PSRL_ERR_WORKSPACE"
    assert bwd(*change(14, p + 4)) == bwd(*change(16, p + 8)) == bwd(*change(18, p + 8)) == "PSRL_ERR_INVALID_ARG"
    assert bwd(*change(15, 60)) == bwd(*change(17, 72 - 4)) == "PSRL_ERR_SHAPE"


def test_next_tokens_are_made_once_for_all_threads(lib):
    """The plan makes them when they are first asked for, whoever asks: the same arrays for every thread, at the same place."""
    from concurrent.futures import ThreadPoolExecutor

    rng = np.random.default_rng(4)
    parent, seg_len, gbs, flags = random_forest(rng, 40, 900, 2, cached_roots=True, step_samples=True)
    L = lib.lib()

    def ask(plan):
        off, nxt = ctypes.POINTER(ctypes.c_int32)(), ctypes.POINTER(ctypes.c_int32)()
        assert L.psrl_plan_next_tokens(plan.handle, ctypes.byref(off), ctypes.byref(nxt)) == 0
        return ctypes.addressof(off.contents), ctypes.addressof(nxt.contents)

    with ThreadPoolExecutor(8) as pool:
        for _ in range(20):
            plan = lib.Plan(parent, seg_len, gbs, 4, 2, 128, "bf16", seg_flags=flags)
            assert len(set(pool.map(ask, [plan] * 16))) == 1
    want = oracle_next_tokens(oracle_plan(parent, seg_len, gbs, flags))
    off, tok = plan.next_tokens()
    assert {r: sorted(tok[off[r]:off[r + 1]].tolist()) for r in range(len(off) - 1)} == want


def workspace_bound(dtype, n, h, v, m, backward):
    """What include/psrl.h says a call may take."""
    if n == 0:
        return 256
    if not backward:
        return 16 * n * (v // 128 + 2) + (8 << 20)
    es, rows = (4 if dtype == "f32" else 2), max(256, -(-n // 128) * 128)
    wide = -(-h // 32) * 32
    return es * max(64 << 20, 8192 * rows) + es * rows * h + max(4 * rows * wide, 64 << 20) + 40 * n + 24 * m + 4096


def test_workspace_keeps_to_its_bounds(lib):
    """Few rows, many rows, narrow and wide: never more than the header says, whatever the vocabulary."""
    for dtype in ("bf16", "f32"):
        for n in (0, 1, 2, 4, 5, 8, 16, 40, 64, 100, 128, 129, 200, 256, 257, 342, 512, 520, 777, 1000, 4096, 8192, 8193, 50000, 200000):
            for h in (8, 64, 72, 1024, 3584, 4096, 8192, 16384):
                for v in (1, 7, 100, 1000, 20000, 50257, 131072, 1 << 18, (1 << 18) + 1, 1 << 20, 1 << 24, 1 << 30):
                    for m in (0, n, 3 * n):
                        for backward in (False, True):
                            got = lib.psrl_token_logprob_workspace_bytes(n, h, v, m, backward, dtype)
                            assert got <= workspace_bound(dtype, n, h, v, m, backward), (dtype, n, h, v, m, backward, got)

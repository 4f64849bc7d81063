"""Compaction of the cache manager's arena and the argument checks of the block copies (host logic, no GPU)."""
import ctypes

import numpy as np
import pytest

from paper_2608_25683_b200 import binding

from test_oracle_cache import random_case


def place(step, seg_len, bs_of):
    return {s: (b, -(-seg_len[s] // bs_of[s]) * bs_of[s]) for s, b in zip(step["seg_id"], step["seg_slot_base"])}


def test_compaction_of_random_schedules(lib):
    """Compacting after every micro-batch: the moves are what slides the resident blocks together, every block is found
    where the moves put it, nothing else changes (trees, reference counts), and a bounded arena never does worse."""
    rng = np.random.default_rng(5)
    moved = 0
    for it in range(80):
        n, M = int(rng.integers(2, 30)), int(rng.integers(2, 9))
        parent, seg_len, gbs, mb = random_case(rng, n, M, max_len=300)
        cache, plain = (binding.Cache(parent, seg_len, gbs, mb, M) for _ in range(2))
        group, bs_of = -1, []
        for s, p in enumerate(parent):
            group += p == -1
            bs_of.append((gbs[group] or 16) if p == -1 else bs_of[p])
        arena = np.full(1 << 16, -1, dtype=np.int64)   # which segment's slot (segment * 4096 + offset) a slot holds
        resident = {}
        for m in range(M):
            step, other = cache.begin(m), plain.begin(m)
            for key in ("seg_id", "parent", "seg_flags", "new", "live_slots"):
                assert step[key] == other[key]
            assert step["pool_slots"] <= other["pool_slots"] or step["pool_slots"] == step["live_slots"]
            for s, (base, ext) in place(step, seg_len, bs_of).items():
                if s in step["new"]:
                    arena[base:base + ext] = s * 4096 + np.arange(ext)
                    resident[s] = (base, ext)
                assert resident[s] == (base, ext)
                assert np.array_equal(arena[base:base + ext], s * 4096 + np.arange(ext))     # every block is where it is said to be
            for s in cache.end(m)["freed"]:
                base, ext = resident.pop(s)
                arena[base:base + ext] = -1
            plain.end(m)
            moves, top = cache.compact()
            moved += len(moves)
            src_end = dst_end = 0
            for src, dst, k in moves.tolist():
                assert k > 0 and dst < src and src >= src_end and dst >= dst_end and k % 16 == 0
                src_end, dst_end = src + k, dst + k
            before = arena.copy()
            for src, dst, k in moves.tolist():
                arena[dst:dst + k] = before[src:src + k]
            at = 0
            for s, (base, ext) in sorted(resident.items(), key=lambda x: x[1]):
                resident[s] = (at, ext)
                at += ext
            assert top == at
            assert len(cache.compact()[0]) == 0          # nothing left to do
        assert cache.refcounts() == plain.refcounts()
    assert moved > 40       # the schedules do leave holes


def test_compaction_makes_room(lib):
    """Free slots in two pieces: a block that fits neither evicts a resident one, but not after a compaction."""
    parent, seg_len, gbs = [-1, -1, 1, -1, -1], [64, 32, 32, 64, 128], [16] * 4
    mb = [0, 0, 3, 1, 2]        # A 64 | B 32 (again in 3) | C 64 leaves; D 128 comes last
    def run(compact):
        c = binding.Cache(parent, seg_len, gbs, mb, 4, capacity_slots=176)
        for m in range(2):
            c.begin(m)
            c.end(m)
        if compact:
            moves, top = c.compact()
            assert moves.tolist() == [[64, 0, 32]] and top == 32
        return c.begin(2)["evict"]
    assert run(False) == [(1, 64)] and run(True) == []


def test_compaction_refusals(lib):
    c = binding.Cache([-1], [16], [16], [0], 1)
    c.begin(0)
    with pytest.raises(binding.PsrlError) as e:
        c.compact()                                       # inside a micro-batch
    assert e.value.name == "PSRL_ERR_INVALID_ARG"
    c.end(0)
    assert c.compact()[1] == 0
    assert lib.lib().psrl_cache_compact(None, None, None, None) == 1


def ext(*rows):
    return np.array(rows, dtype=np.int32)


def test_copy_and_move_refusals(lib):
    """Everything wrong with the extents is found on the host."""
    L = lib.lib()
    buf = ctypes.create_string_buffer(1 << 16)
    p = (ctypes.addressof(buf) + 255) // 256 * 256
    k, v, k2, v2 = p, p + 8192, p + 16384, p + 24576      # 2 heads x 32 slots x 128 bytes each

    def copy(e, ks=k, vs=v, kd=k2, vd=v2, heads=2, row=128, cap=32, cap2=32):
        return lib.STATUS_NAMES[L.psrl_kv_copy(e.ctypes.data, len(e), heads, row, ks, vs, cap, kd, vd, cap2, None)]

    none = np.zeros((0, 3), dtype=np.int32)
    assert copy(none) == copy(ext([3, 4, 0])) == "PSRL_OK"
    assert copy(ext([0, 0, 33])) == copy(ext([20, 0, 13])) == copy(ext([-1, 0, 4])) == copy(ext([0, 30, 4])) == "PSRL_ERR_SHAPE"
    assert copy(ext([0, 0, -1])) == copy(ext([2 ** 31 - 1, 0, 2 ** 31 - 1])) == "PSRL_ERR_SHAPE"
    assert copy(ext([0, 0, 8], [8, 7, 8])) == "PSRL_ERR_INVALID_ARG"            # destinations overlap
    assert copy(none, row=64) == copy(none, row=1024) == copy(none, heads=0) == copy(none, cap=-1) == "PSRL_ERR_SHAPE"
    assert copy(none, ks=k + 4) == copy(none, kd=None) == "PSRL_ERR_INVALID_ARG"
    assert copy(none, kd=k + 4096) == copy(none, vd=k2) == copy(none, vd=k) == "PSRL_ERR_INVALID_ARG"   # tensors overlap
    # inside one pool: no written slot may be read
    assert copy(ext([0, 4, 8]), kd=k, vd=v) == "PSRL_ERR_INVALID_ARG"
    assert copy(ext([0, 16, 8], [16, 24, 4]), kd=k, vd=v) == "PSRL_ERR_INVALID_ARG"
    assert copy(ext([0, 16, 8], [23, 8, 4]), kd=k, vd=v) == "PSRL_ERR_INVALID_ARG"
    assert copy(none, kd=k, vd=v, cap2=31) == "PSRL_ERR_INVALID_ARG"

    def move(e, kp=k, vp=v, heads=2, row=128, cap=32, ws=p + 32768, wsb=256):
        return lib.STATUS_NAMES[L.psrl_kv_move(e.ctypes.data, len(e), heads, row, kp, vp, cap, ws, wsb, None)]

    assert move(ext([0, 4, 4])) == "PSRL_ERR_INVALID_ARG"                       # upwards
    assert move(ext([8, 0, 4], [4, 4, 4])) == move(ext([8, 4, 4], [12, 2, 4])) == "PSRL_ERR_INVALID_ARG"   # not ascending
    assert move(ext([8, 0, 4], [11, 4, 4])) == move(ext([8, 0, 4], [12, 3, 4])) == "PSRL_ERR_INVALID_ARG"  # overlap
    assert move(ext([30, 0, 4])) == move(ext([-4, -8, 4])) == "PSRL_ERR_SHAPE"
    assert move(none, ws=p + 8) == move(none, ws=None) == move(none, kp=k + 8) == move(none, vp=k) == "PSRL_ERR_INVALID_ARG"
    assert move(none, wsb=255) == "PSRL_ERR_WORKSPACE"
    with pytest.raises(ValueError):
        binding._extents([[1, 2], [3, 4]])


def test_empty_extents_of_a_move_do_nothing(lib):
    """Wherever they are listed, as in a copy: only the extents with slots have to ascend."""
    L = lib.lib()
    buf = ctypes.create_string_buffer(1 << 16)
    p = (ctypes.addressof(buf) + 255) // 256 * 256

    def move(e):
        # no pools: a call that passes the checks has nothing to move, and clears the workspace where there is a GPU
        return lib.STATUS_NAMES[L.psrl_kv_move(e.ctypes.data, len(e), 2, 128, None, None, 32, p, 256, None)]

    for e in (ext([3, 9, 0]), ext([8, 4, 4], [2, 2, 0], [12, 8, 4]), ext([8, 8, 4], [2, 3, 0])):
        assert move(e) not in ("PSRL_ERR_INVALID_ARG", "PSRL_ERR_SHAPE")
    assert move(ext([31, 33, 0])) == "PSRL_ERR_SHAPE"                            # out of the pool all the same
    assert move(ext([3, 9, 1])) == move(ext([8, 4, 4], [2, 2, 1])) == "PSRL_ERR_INVALID_ARG"

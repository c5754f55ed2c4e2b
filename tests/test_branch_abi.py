"""Refusals of the entry points for sequences that branch, and the moves that empty
units: host only (pointers are made up and never followed)."""
import ctypes
import os
import random

import pytest
import torch

from paper_2609_34380_amd import dps
from test_kv_abi import CACHES, cache

INVALID, ALIGNMENT, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(dps.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return dps.load_library()


def struct(cls, defaults, kw):
    f = dict(defaults, **kw)
    return cls(*[f[n] for n, _ in cls._fields_])


FORKED = dict(rows=8, table=0x100000, seq_len=0x110000, src=0x120000, dst=0x130000,
              tokens=0x140000, freed=0x150000, n_freed=100, counts=0x160000)
FORK = dict(parent=0x10000, seq_len=0x20000, old_rows=8, block_tokens=16, table=0x30000, cols=64,
            fresh=0x40000, n_fresh=10, n_blocks=1000, ws=0x1000, ws_bytes=1 << 20)


def fork(lib, **kw):
    out = struct(dps.CKvForked, FORKED, {k: v for k, v in kw.pop("out", {}).items()})
    a = dict(FORK, **kw)
    return lib.dps_kv_fork(a["parent"], a["seq_len"], a["old_rows"], a["block_tokens"], a["table"],
                           a["cols"], a["fresh"], a["n_fresh"], a["n_blocks"],
                           None if a.get("no_out") else ctypes.byref(out), a["ws"], a["ws_bytes"],
                           None)


@pytest.mark.parametrize("kw,status", [
    (dict(no_out=True), INVALID), (dict(old_rows=-1), INVALID), (dict(cols=-1), INVALID),
    (dict(n_fresh=-1), INVALID), (dict(n_blocks=-1), INVALID), (dict(out=dict(rows=-1)), INVALID),
    (dict(out=dict(n_freed=-1)), INVALID),
    (dict(old_rows=4097), UNSUPPORTED), (dict(out=dict(rows=4097)), UNSUPPORTED),
    (dict(block_tokens=8), UNSUPPORTED), (dict(block_tokens=24), UNSUPPORTED),
    (dict(block_tokens=512), UNSUPPORTED), (dict(cols=1 << 31), UNSUPPORTED),
    (dict(cols=1 << 29), UNSUPPORTED), (dict(n_blocks=1 << 31), UNSUPPORTED),
    (dict(parent=None), INVALID), (dict(seq_len=None), INVALID), (dict(table=None), INVALID),
    (dict(fresh=None), INVALID), (dict(out=dict(table=None)), INVALID),
    (dict(out=dict(seq_len=None)), INVALID), (dict(out=dict(src=None)), INVALID),
    (dict(out=dict(freed=None)), INVALID), (dict(out=dict(counts=None)), INVALID),
    (dict(parent=0x10002), ALIGNMENT), (dict(out=dict(counts=0x160001)), ALIGNMENT),
    # outputs over inputs
    (dict(out=dict(table=0x30000)), INVALID), (dict(out=dict(table=0x307fc)), INVALID),
    (dict(out=dict(table=0x30004 - 8 * 64 * 4)), INVALID), (dict(out=dict(seq_len=0x20000)), INVALID),
    (dict(out=dict(freed=0x40000)), INVALID), (dict(out=dict(counts=0x1001c)), INVALID),
    (dict(ws=None), WORKSPACE), (dict(ws_bytes=2303), WORKSPACE), (dict(ws=0x1080), ALIGNMENT),
])
def test_fork_refuses(lib, kw, status):
    assert fork(lib, **kw) == status
    assert lib.dps_last_error()


def test_fork_workspace(lib):
    assert lib.dps_kv_fork_workspace_bytes(8, 1000) == 256 + 2048
    assert lib.dps_kv_fork_workspace_bytes(4096, 1 << 20) == 4 * 4096 + (1 << 21)
    assert lib.dps_kv_fork_workspace_bytes(4097, 10) == 0
    assert lib.dps_kv_fork_workspace_bytes(-1, 10) == 0


@pytest.mark.parametrize("kw,status", CACHES)
def test_copy_cache(lib, kw, status):
    assert lib.dps_kv_copy(ctypes.byref(cache(**kw)), 0x1000, 0x2000, None, 3, None, None) == status


def test_copy_and_remap_refuse(lib):
    c = ctypes.byref(cache())
    assert lib.dps_kv_copy(None, 0x1000, 0x2000, None, 3, None, None) == INVALID
    assert lib.dps_kv_copy(c, 0x1000, 0x2000, None, -1, None, None) == INVALID
    assert lib.dps_kv_copy(c, None, 0x2000, None, 3, None, None) == INVALID
    assert lib.dps_kv_copy(c, 0x1000, None, None, 3, None, None) == INVALID
    assert lib.dps_kv_copy(c, 0x1002, 0x2000, None, 3, None, None) == ALIGNMENT
    assert lib.dps_kv_copy(c, 0x1000, 0x2000, 0x3001, 3, None, None) == ALIGNMENT
    assert lib.dps_kv_copy(c, 0x1000, 0x2000, None, 3, 0x3002, None) == ALIGNMENT
    assert lib.dps_kv_copy(c, 0x1000, 0x2000, None, 0x7fffffff, None, None) == UNSUPPORTED
    assert lib.dps_kv_copy(c, None, None, None, 0, None, None) == 0
    remap = lib.dps_kv_remap
    assert remap(0x1000, -1, 0x20000, 0x30000, 3, None) == INVALID
    assert remap(0x1000, 10, 0x20000, 0x30000, -3, None) == INVALID
    assert remap(0x1000, 1 << 31, 0x20000, 0x30000, 3, None) == INVALID
    assert remap(None, 10, 0x20000, 0x30000, 3, None) == INVALID
    assert remap(0x1000, 10, None, 0x30000, 3, None) == INVALID
    assert remap(0x1000, 10, 0x20000, None, 3, None) == INVALID
    assert remap(0x1002, 10, 0x20000, 0x30000, 3, None) == ALIGNMENT
    assert remap(0x1000, 10, 0x1024, 0x30000, 3, None) == INVALID
    assert remap(0x1000, 10, 0x20000, 0xff8, 3, None) == INVALID
    assert remap(None, 0, None, None, 0, None) == 0


BEAM = dict(batch=2, beams=4, vocab=1000, logits=0x100000, logits_stride=1000, type=dps.BEAM_F16,
            end=2, score=0x10000, done=0x20000, keep=4, new_score=0x30000, parent=0x40000,
            token=0x50000, new_done=0x60000)


@pytest.mark.parametrize("kw,status", [
    (dict(type=3), INVALID), (dict(type=-1), INVALID),
    (dict(batch=-1), UNSUPPORTED), (dict(batch=(1 << 20) + 1), UNSUPPORTED),
    (dict(batch=1 << 19), UNSUPPORTED), (dict(beams=0), UNSUPPORTED), (dict(beams=1025), UNSUPPORTED),
    (dict(vocab=0), UNSUPPORTED), (dict(vocab=(1 << 24) + 1), UNSUPPORTED),
    (dict(keep=0), UNSUPPORTED), (dict(keep=257), UNSUPPORTED),
    (dict(end=-2), INVALID), (dict(end=1000), INVALID), (dict(end=-1), INVALID),
    (dict(logits_stride=999), INVALID), (dict(logits_stride=(1 << 40) + 1), UNSUPPORTED),
    (dict(logits=None), INVALID), (dict(score=None), INVALID), (dict(new_score=None), INVALID),
    (dict(parent=None), INVALID), (dict(token=None), INVALID), (dict(new_done=None), INVALID),
    (dict(logits=0x100001), ALIGNMENT), (dict(type=dps.BEAM_F32, logits=0x100002), ALIGNMENT),
    (dict(score=0x10002), ALIGNMENT), (dict(token=0x50001), ALIGNMENT),
    (dict(new_score=0x10000), INVALID), (dict(parent=0x1001c), INVALID),
    (dict(new_done=0x20007), INVALID), (dict(token=0x100000 + 15998), ALIGNMENT),
    (dict(token=0x100000 + 15996), INVALID),
    (dict(batch=1024, beams=1024, vocab=1 << 24, logits_stride=1 << 24, done=0, score=1 << 45,
          logits=1 << 46), UNSUPPORTED),
])
def test_beam_refuses(lib, kw, status):
    a = struct(dps.CBeamArgs, BEAM, kw)
    assert lib.dps_beam_select(ctypes.byref(a), 0x1000, 1 << 40, None) == status
    assert lib.dps_last_error()


def test_beam_workspace(lib):
    a = ctypes.byref(struct(dps.CBeamArgs, BEAM, {}))
    need = lib.dps_beam_workspace_bytes(2, 4, 1000, 4)
    assert need > 0
    assert lib.dps_beam_select(a, None, need, None) == WORKSPACE
    assert lib.dps_beam_select(a, 0x1000, 100, None) == WORKSPACE
    assert lib.dps_beam_select(a, 0x1010, need, None) == ALIGNMENT
    assert lib.dps_beam_select(None, 0x1000, need, None) == INVALID
    for bad in ((0, 4, 1000, 4), (-1, 4, 1000, 4), (2, 0, 1000, 4), (2, 4, 0, 4), (2, 4, 1000, 0),
                (2, 4, 1000, 257), (2, 1025, 1000, 4)):
        assert lib.dps_beam_workspace_bytes(*bad) == 0


def test_binding_refuses_host_tensors():
    i = torch.zeros(4, dtype=torch.int32)
    for call in (lambda: dps.kv_fork(i, i, i.view(2, 2), i, 16, 10),
                 lambda: dps.kv_remap(i, i, i), lambda: dps.kv_copy(None, i, i),
                 lambda: dps.beam_select(torch.zeros(4, 5), torch.zeros(4), 2),
                 lambda: dps.beam_select(torch.zeros(4, 5, dtype=torch.int32), i, 2)):
        with pytest.raises(ValueError):
            call()


# ---- moves that empty units ----------------------------------------------------------


def state(s, held):
    return [sorted(b for b in held if b // s.blocks_per_unit == u) for u in range(s.n_units)]


@pytest.mark.parametrize("seed", range(20))
def test_compact(seed):
    """Against the rule: which units are emptied, where their blocks go, and what the
    manager says of every unit before and after the old places are freed."""
    rng = random.Random(seed)
    units, per, res = rng.randint(1, 9), rng.randint(1, 8), rng.randint(0, 3)
    s = dps.SumManager(units, per, min(res, units))
    held = set(s.alloc(rng.randint(0, units * per)))
    gone = [b for b in sorted(held) if rng.random() < 0.5]
    if gone:
        s.free(gone)
    held -= set(gone)
    most = rng.choice((0, 1, 3, 1000))
    src, dst = s.compact(most)
    # the rule
    by = state(s, held)
    avail = [u for u in range(units) if 0 < len(by[u]) < per]
    order = sorted(avail, key=lambda u: (len(by[u]), u))
    want, emptied = [], []
    free = {u: [u * per + i for i in range(per) if u * per + i not in held] for u in avail}
    for i, u in enumerate(order):
        others = order[i + 1:]
        if not others or len(by[u]) > sum(len(free[o]) for o in others) or \
                len(want) + len(by[u]) > most:
            break
        for b in by[u]:
            to = [o for o in others if free[o]][-1]
            want.append((b, free[to].pop(0)))
        emptied.append(u)
    assert list(zip(src, dst)) == sorted(want)
    # both ends are allocated until src is freed
    before = s.counts()["free"]
    for b in dst:
        assert b not in held
    after = (held | set(dst)) - set(src)
    if src:
        s.free(src)
    assert s.counts()["free"] == before + len(emptied)
    for u, blocks in enumerate(state(s, after)):
        if blocks:
            assert s.unit_state(u) == (dps.UNIT_FULL if len(blocks) == per else dps.UNIT_AVAIL)
    if after:
        s.free(sorted(after))


def test_compact_brings_full_mode_back():
    """Two half-empty units: one of them takes the other's blocks, and the residual
    that KV blocks had pushed out gets the unit."""
    s = dps.SumManager(2, 8, 1)
    blocks = s.alloc(16)
    assert s.mode == dps.MODE_FAST
    assert not s.free(blocks[:5] + blocks[8:13])
    assert s.restore_begin() is None
    src, dst = s.compact(100)
    assert len(src) == 3 and not set(src) & set(dst)
    assert s.restore_begin() is None          # until the old places are freed
    assert s.free(src)                        # worth waking the restore worker
    r, u = s.restore_begin()
    s.restore_done(r)
    assert s.mode == dps.MODE_FULL


def test_compact_refuses(lib):
    s = dps.SumManager(2, 8, 0)
    s.alloc(3)
    with pytest.raises(dps.DpsError):
        s.compact(-1)
    n = ctypes.c_int64(0)
    assert lib.dps_sum_compact(None, 0, None, None, ctypes.byref(n)) == INVALID
    assert lib.dps_sum_compact(s._h, 3, None, None, ctypes.byref(n)) == INVALID
    assert lib.dps_sum_compact(s._h, 0, None, None, None) == INVALID
    assert s.compact(0) == ([], []) and s.compact(10) == ([], [])


# ---- attention of rows that share prefixes ----------------------------------------------


def shared(lib, kw=(), c=None, starts=0x60000, lens=0x70000, groups=2, ws=0x1000, ws_bytes=1 << 40):
    from test_kv_abi import attn
    a = attn(**dict(kw))
    return lib.dps_attn_shared(ctypes.byref(a), ctypes.byref(c or cache()), starts, lens, groups, ws,
                               ws_bytes, None)


@pytest.mark.parametrize("kw,status", CACHES)
def test_shared_cache(lib, kw, status):
    assert shared(lib, c=cache(**kw)) == status


@pytest.mark.parametrize("kw,status", [
    (dict(window=3), UNSUPPORTED), (dict(window=-1), INVALID), (dict(heads=12), INVALID),
    (dict(rows=-1), INVALID), (dict(q=0), INVALID), (dict(kv_len=0), INVALID),
    (dict(req=0, requests=3), INVALID), (dict(out=0x50008), ALIGNMENT),
    (dict(rows=(1 << 20) + 1), UNSUPPORTED), (dict(rows=1 << 20, heads=512, q_stride=1 << 16, out_stride=1 << 16), UNSUPPORTED),
    (dict(scale=float("inf")), INVALID), (dict(type=dps.KV_E4M3), INVALID),
])
def test_shared_refuses(lib, kw, status):
    assert shared(lib, kw) == status
    assert lib.dps_last_error()


def test_shared_groups_and_workspace(lib):
    assert shared(lib, groups=-1) == INVALID
    assert shared(lib, groups=1025) == UNSUPPORTED
    assert shared(lib, starts=None) == INVALID and shared(lib, lens=None) == INVALID
    assert shared(lib, starts=0x60002) == ALIGNMENT and shared(lib, lens=0x70001) == ALIGNMENT
    need = lib.dps_attn_shared_workspace_bytes(4, 2, 32, 8, 128)
    assert need > lib.dps_attn_workspace_bytes(4, 32, 8, 128)
    assert shared(lib, ws=None) == WORKSPACE and shared(lib, ws_bytes=256) == WORKSPACE
    assert shared(lib, ws=0x1010) == ALIGNMENT
    assert lib.dps_attn_shared(None, ctypes.byref(cache()), 0x1000, 0x2000, 1, 0x1000, need,
                               None) == INVALID
    for bad in ((0, 2, 32, 8, 128), (4, -1, 32, 8, 128), (4, 1025, 32, 8, 128), (4, 2, 30, 8, 128),
                (4, 2, 32, 0, 128), (4, 2, 32, 8, 257), ((1 << 20) + 1, 2, 32, 8, 128)):
        assert lib.dps_attn_shared_workspace_bytes(*bad) == 0

"""Refusals of the paged KV cache's entry points: every one on the host, before
anything is enqueued (no GPU; pointers are made up and never followed)."""
import ctypes
import os

import pytest
import torch

from paper_2609_34380_amd import dps

INVALID, ALIGNMENT, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4
NAN = float("nan")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(dps.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return dps.load_library()


def cache(**kw):
    f = dict(pool=0x10000, pool_bytes=1 << 30, block_stride=1 << 16, kv_heads=8, head_dim=128,
             block_tokens=16, type=dps.KV_F16, k_scale=1.0, v_scale=1.0)
    f.update(kw)
    return dps.CKvCache(*[f[n] for n, _ in dps.CKvCache._fields_])


def store(**kw):
    f = dict(rows=4, heads=32, qkv=0x10000, qkv_stride=48 * 128, slot=0x20000, pos=0x30000,
             rope=0x40000, max_pos=100, rot=128, adjacent=0, q_weight=0x50000, k_weight=0x50000,
             eps=1e-6, type=dps.KV_F16, q_out=0x60000, q_out_stride=32 * 128, k_out=0,
             k_out_stride=0)
    f.update(kw)
    return dps.CKvStoreArgs(*[f[n] for n, _ in dps.CKvStoreArgs._fields_])


def attn(**kw):
    f = dict(rows=4, heads=32, q=0x10000, q_stride=32 * 128, table=0x20000, requests=4,
             table_cols=64, req=0x30000, kv_len=0x40000, window=0, type=dps.KV_F16, scale=0.1,
             out=0x50000, out_stride=32 * 128, lse=0)
    f.update(kw)
    return dps.CAttnArgs(*[f[n] for n, _ in dps.CAttnArgs._fields_])


CACHES = [
    (dict(type=3), INVALID), (dict(type=-1), INVALID),
    (dict(kv_heads=0), INVALID), (dict(kv_heads=4097), INVALID),
    (dict(block_tokens=8), UNSUPPORTED), (dict(block_tokens=48), UNSUPPORTED),
    (dict(block_tokens=512), UNSUPPORTED), (dict(block_tokens=0), UNSUPPORTED),
    (dict(head_dim=80), UNSUPPORTED), (dict(head_dim=32), UNSUPPORTED),
    (dict(head_dim=96, type=dps.KV_E4M3), UNSUPPORTED),
    (dict(block_stride=(1 << 16) - 16), INVALID),
    (dict(block_stride=(1 << 16) + 8), ALIGNMENT),
    (dict(pool=0), INVALID), (dict(pool=0x10008), ALIGNMENT),
    (dict(pool_bytes=(1 << 16) - 1), INVALID),
    (dict(k_scale=0.0), INVALID), (dict(v_scale=-1.0), INVALID), (dict(k_scale=NAN), INVALID),
    (dict(v_scale=float("inf")), INVALID),
]


@pytest.mark.parametrize("kw,status", CACHES)
def test_cache_descriptor(lib, kw, status):
    c = cache(**kw)
    assert lib.dps_kv_store(ctypes.byref(store()), ctypes.byref(c), None) == status
    assert lib.dps_last_error()
    assert lib.dps_attn_decode(ctypes.byref(attn()), ctypes.byref(c), 0x100, 1 << 30, None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(type=dps.KV_E4M3), INVALID), (dict(type=dps.KV_BF16), INVALID),
    (dict(rows=-1), INVALID), (dict(rows=1 << 31), INVALID),
    (dict(heads=-1), INVALID), (dict(heads=65537), INVALID),
    (dict(qkv_stride=48 * 128 - 8), INVALID), (dict(qkv_stride=48 * 128 + 4), ALIGNMENT),
    (dict(q_out_stride=100), INVALID), (dict(q_out_stride=32 * 128 + 1), ALIGNMENT),
    (dict(k_out=0x70000, k_out_stride=8), INVALID),
    (dict(k_out=0x70000, k_out_stride=8 * 128 + 2), ALIGNMENT),
    (dict(rot=8), INVALID), (dict(rot=24), INVALID), (dict(rot=144), INVALID),
    (dict(rot=0), INVALID), (dict(max_pos=0), INVALID), (dict(pos=0), INVALID),
    (dict(q_weight=0), INVALID), (dict(k_weight=0), INVALID),
    (dict(eps=-1.0), INVALID), (dict(eps=NAN), INVALID),
    (dict(qkv=0), INVALID), (dict(slot=0), INVALID), (dict(q_out=0), INVALID),
    (dict(qkv=0x10008), ALIGNMENT), (dict(q_out=0x60002), ALIGNMENT), (dict(rope=0x40004), ALIGNMENT),
    (dict(q_weight=0x50004), ALIGNMENT), (dict(slot=0x20004), ALIGNMENT), (dict(pos=0x30001), ALIGNMENT),
])
def test_store_refuses(lib, kw, status):
    assert lib.dps_kv_store(ctypes.byref(store(**kw)), ctypes.byref(cache()), None) == status
    assert lib.dps_last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(type=dps.KV_E4M3), INVALID), (dict(type=dps.KV_BF16), INVALID),
    (dict(rows=-1), INVALID), (dict(requests=-1), INVALID), (dict(table_cols=-1), INVALID),
    (dict(heads=0), INVALID), (dict(heads=30), INVALID), (dict(heads=1 << 17), INVALID),
    (dict(window=-1), INVALID), (dict(scale=NAN), INVALID), (dict(scale=float("inf")), INVALID),
    (dict(q_stride=32 * 128 - 8), INVALID), (dict(out_stride=8), INVALID),
    (dict(q_stride=32 * 128 + 4), ALIGNMENT), (dict(out_stride=32 * 128 + 4), ALIGNMENT),
    (dict(q=0), INVALID), (dict(out=0), INVALID), (dict(kv_len=0), INVALID), (dict(table=0), INVALID),
    (dict(req=0, requests=3), INVALID),
    (dict(q=0x10008), ALIGNMENT), (dict(out=0x50004), ALIGNMENT), (dict(lse=0x50002), ALIGNMENT),
    (dict(table=0x20002), ALIGNMENT), (dict(req=0x30001), ALIGNMENT),
    (dict(rows=1 << 24, requests=1 << 24), UNSUPPORTED),
    (dict(rows=4000, requests=4000, table_cols=1 << 27), UNSUPPORTED),
    (dict(rows=1, table_cols=1 << 31), UNSUPPORTED), (dict(rows=1, table_cols=1 << 62), UNSUPPORTED),
])
def test_attn_refuses(lib, kw, status):
    got = lib.dps_attn_decode(ctypes.byref(attn(**kw)), ctypes.byref(cache()), 0x100, 1 << 40, None)
    assert got == status
    assert lib.dps_last_error()


def test_attn_workspace(lib):
    need = lib.dps_attn_workspace_bytes(4, 32, 8, 128)
    assert need > 0
    args, c = attn(), cache()
    run = lambda ws, n: lib.dps_attn_decode(ctypes.byref(args), ctypes.byref(c), ws, n, None)
    assert run(0x100, need - 1) == WORKSPACE and run(None, 0) == WORKSPACE
    assert run(0x180, need) == ALIGNMENT
    for bad in ((0, 32, 8, 128), (4, 30, 8, 128), (4, 0, 8, 128), (4, 32, 0, 128), (-1, 32, 8, 128)):
        assert lib.dps_attn_workspace_bytes(*bad) == 0


def test_empty_calls_are_noops(lib):
    c = cache()
    assert lib.dps_kv_store(ctypes.byref(store(rows=0, qkv=0, q_out=0)), ctypes.byref(c), None) == 0
    assert lib.dps_attn_decode(ctypes.byref(attn(rows=0, q=0)), ctypes.byref(c), None, 0, None) == 0


def _map(lib, ctx=0x1000, new=0x2000, requests=4, tokens=16, fresh=0x3000, n_fresh=9, table=0x4000,
         cols=8, **kw):
    f = dict(rows=4, q_start=0x100, seq_len=0x200, counts=0x300, pos=0x400, slot=0x500, req=0x600,
             kv_len=0x700)
    f.update(kw)
    step = dps.CKvStep(*[f[n] for n, _ in dps.CKvStep._fields_])
    return lib.dps_kv_map(ctx, new, requests, tokens, fresh, n_fresh, table, cols,
                          ctypes.byref(step), None)


@pytest.mark.parametrize("kw,status", [
    (dict(requests=-1), INVALID), (dict(requests=4097), UNSUPPORTED), (dict(cols=-1), INVALID),
    (dict(n_fresh=-1), INVALID), (dict(tokens=8), UNSUPPORTED), (dict(tokens=24), UNSUPPORTED),
    (dict(cols=1 << 30), UNSUPPORTED), (dict(rows=-1), INVALID), (dict(rows=1 << 31), INVALID),
    (dict(ctx=None), INVALID), (dict(new=None), INVALID), (dict(table=None), INVALID),
    (dict(fresh=None), INVALID), (dict(q_start=0), INVALID), (dict(seq_len=0), INVALID),
    (dict(counts=0), INVALID), (dict(pos=0), INVALID), (dict(slot=0), INVALID), (dict(req=0), INVALID),
    (dict(kv_len=0), INVALID), (dict(slot=0x504), ALIGNMENT), (dict(ctx=0x1001), ALIGNMENT),
    (dict(table=0x4002), ALIGNMENT), (dict(kv_len=0x702), ALIGNMENT),
])
def test_map_refuses(lib, kw, status):
    assert _map(lib, **kw) == status
    assert lib.dps_last_error()


def test_binding_refuses_host_tensors():
    i32 = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        dps.kv_map(i32, i32, i32, i32.reshape(2, 1), 16, rows=2)
    with pytest.raises(ValueError):
        dps.KvCache(torch.zeros(1 << 16, dtype=torch.uint8), 16, 8, 128, torch.float16)
    with pytest.raises(ValueError):
        dps.KvCache(torch.zeros(1 << 16, dtype=torch.uint8), 16, 8, 128, torch.float32)


@pytest.mark.parametrize("kw", [dict(k_scale=1e-39), dict(v_scale=1e-45)])
def test_scales_without_a_reciprocal(lib, kw):
    c = cache(type=dps.KV_E4M3, **kw)
    assert lib.dps_kv_store(ctypes.byref(store()), ctypes.byref(c), None) == INVALID
    assert lib.dps_attn_decode(ctypes.byref(attn()), ctypes.byref(c), 0x100, 1 << 30, None) == INVALID


def test_score_factor_overflow(lib):
    c = cache(type=dps.KV_E4M3, k_scale=1e10)
    for scale in (1e30, -1e30):
        args = attn(scale=scale)
        got = lib.dps_attn_decode(ctypes.byref(args), ctypes.byref(c), 0x100, 1 << 30, None)
        assert got == INVALID


@pytest.mark.parametrize("sizes", [(4, 1 << 40, 1, 128), (4, 8192, 8192, 128), (4, 32, 8, 1 << 40)])
def test_attn_workspace_of_sizes_that_no_call_has(lib, sizes):
    assert lib.dps_attn_workspace_bytes(*sizes) == 0


@pytest.mark.parametrize("seq_len", [0x1000, 0x2000])
def test_map_does_not_write_its_lengths(lib, seq_len):
    assert _map(lib, seq_len=seq_len) == INVALID

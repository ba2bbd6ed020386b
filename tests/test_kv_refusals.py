"""What moa_kv_append, moa_decode_attn and moa_kv_evict refuse, before anything is launched (no GPU needed)."""
import ctypes as C

import pytest
import torch

import paper_2410_03804_amd as moa
from paper_2410_03804_amd import binding

FAKE = 1 << 20          # an address that is never dereferenced
lib = binding._lib


def cache(**kw):
    d = dict(dtype=moa.BF16, n_kv_heads=8, head_dim=128, B=2, n_pages=100, page_size=16, max_pages=40, k=FAKE, v=FAKE, table=FAKE, len=FAKE,
             pos=FAKE, seen=FAKE, score=FAKE)
    d.update(kw)
    return binding._KvCache(**d)


def append(c, k=FAKE, v=FAKE, M=1):
    return lib.moa_kv_append(None if c is None else C.byref(c), k, v, M, None, None, None, None)


def decode_bytes(c, H=32):
    n = C.c_size_t(0)
    return lib.moa_decode_attn_workspace_bytes(C.byref(c), H, C.byref(n)), n.value


def decode(c, H=32, q=FAKE, out=FAKE, acc=0, ws=FAKE, ws_bytes=1 << 40):
    return lib.moa_decode_attn(None if c is None else C.byref(c), H, q, out, acc, None, ws, ws_bytes, None)


def evict(c, budget=100, recent=10, ws=FAKE, ws_bytes=1 << 40):
    return lib.moa_kv_evict(None if c is None else C.byref(c), budget, recent, None, ws, ws_bytes, None)


NULL, SHAPE, RANGE, DTYPE, WORKSPACE = -1, -2, -4, -5, -6


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), DTYPE), (dict(n_kv_heads=0), SHAPE), (dict(head_dim=0), SHAPE), (dict(head_dim=257), SHAPE), (dict(B=0), SHAPE),
    (dict(n_pages=0), SHAPE), (dict(page_size=0), SHAPE), (dict(max_pages=-1), SHAPE), (dict(k=None), NULL), (dict(v=None), NULL),
    (dict(table=None), NULL), (dict(len=None), NULL), (dict(pos=None), NULL), (dict(seen=None), NULL),
    (dict(max_pages=1 << 27), SHAPE), (dict(n_pages=1 << 30), SHAPE), (dict(n_pages=2 ** 31 // 128), SHAPE), (dict(B=1 << 18), SHAPE),
    (dict(k=FAKE + 1), SHAPE), (dict(table=FAKE + 2), SHAPE), (dict(score=FAKE + 1), SHAPE),
])
def test_every_call_refuses_such_a_cache(kw, status):
    c = cache(**kw)
    assert append(c) == status and decode(c) == status and evict(c) == status
    assert decode_bytes(c)[0] == status
    n = C.c_size_t(0)
    assert lib.moa_kv_evict_workspace_bytes(C.byref(c), 100, C.byref(n)) == status
    assert append(None) == decode(None) == evict(None) == NULL


def test_append_arguments():
    assert append(cache(), k=None) == NULL and append(cache(), v=None) == NULL
    assert append(cache(), M=0) == SHAPE and append(cache(), M=(1 << 24) + 1) == SHAPE and append(cache(head_dim=256), M=1 << 24) == SHAPE
    assert append(cache(), k=FAKE + 1) == SHAPE
    assert append(cache(B=70000, n_kv_heads=1)) == SHAPE


def test_decode_arguments():
    assert decode(cache(), H=0) == SHAPE and decode(cache(), H=12) == SHAPE
    assert decode(cache(), q=None) == NULL and decode(cache(), out=None) == NULL
    assert decode(cache(), q=FAKE + 1) == SHAPE
    assert decode(cache(score=None), acc=1) == NULL
    assert decode(cache(B=1 << 17), H=64) == SHAPE
    assert decode(cache(max_pages=1 << 24, B=128), H=64) == SHAPE             # tiles are counted in 32 bits
    rc, n = decode_bytes(cache())
    assert rc == 0 and n > 0
    assert decode(cache(), ws_bytes=n - 1, acc=1) == WORKSPACE and decode(cache(), ws=None, acc=1) == WORKSPACE
    assert decode(cache(), ws=FAKE + 16, ws_bytes=1 << 40, acc=1) == WORKSPACE
    assert decode_bytes(cache(score=None))[1] < n                             # scores are only stored for accounts
    assert lib.moa_decode_attn_workspace_bytes(C.byref(cache()), 32, None) == NULL


def test_evict_arguments():
    assert evict(cache(pos=None, seen=None)) == NULL and evict(cache(score=None)) == NULL
    assert evict(cache(), budget=0) == RANGE and evict(cache(), recent=-1) == RANGE and evict(cache(), budget=5, recent=6) == RANGE
    assert evict(cache(B=10000)) == SHAPE
    n = C.c_size_t(0)
    assert lib.moa_kv_evict_workspace_bytes(C.byref(cache()), 100, C.byref(n)) == 0
    assert n.value >= 2 * 8 * (2 * 100 + 1) * 4
    assert evict(cache(), ws=None) == WORKSPACE and evict(cache(), ws_bytes=n.value - 1) == WORKSPACE and evict(cache(), ws=FAKE + 64) == WORKSPACE
    # a budget that no sequence can pass: nothing to do, no workspace, nothing launched
    assert evict(cache(), budget=640, ws=None, ws_bytes=0) == 0 and evict(cache(), budget=10 ** 9, ws=None, ws_bytes=0) == 0
    assert lib.moa_kv_evict_workspace_bytes(C.byref(cache()), 640, C.byref(n)) == 0 and n.value == 0
    assert lib.moa_kv_evict_workspace_bytes(C.byref(cache()), 0, C.byref(n)) == RANGE


def test_binding_refuses_host_tensors_and_wrong_shapes():
    k = torch.zeros(4, 2, 16, 64)
    table, n = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        moa.KVCache(k, k, table, n)
    with pytest.raises(ValueError, match="same shape"):
        moa.KVCache(k, k[:, :1], table, n)
    with pytest.raises(ValueError, match="dtype"):
        moa.KVCache(k.half(), k.half(), table, n)

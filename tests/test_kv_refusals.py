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


class OnGpu(torch.Tensor):
    """Stands in for a tensor on the GPU with that index."""
    is_cuda = True

    def get_device(self):
        return getattr(self, "at", 0)


def on_gpu(*shape, dtype=torch.int32, at=0):
    t = torch.zeros(*shape, dtype=dtype).as_subclass(OnGpu)
    t.at = at
    return t


def test_checks_of_tensors_on_a_device():
    t = on_gpu(4, 6, at=1)
    assert binding._dev_on(t, torch.int32, 24, "x", 1) == t.data_ptr() and binding._dev_on(None, torch.int32, 24, "x", 1) is None
    with pytest.raises(ValueError, match="x: must be on the cache's device"):
        binding._dev_on(t, torch.int32, 24, "x", 0)
    with pytest.raises(ValueError, match="x: 24 elements, the call touches 25"):
        binding._dev_on(t, torch.int32, 25, "x", 1)
    with pytest.raises(TypeError):
        binding._dev_on(t, torch.int32, 24, "x")
    w = on_gpu(100, dtype=torch.float32)
    assert binding._room_on(w, "ws", 0) == (w.data_ptr(), 400) and binding._room_on(None, "ws", 0) == (None, 0)
    for bad, at, error, text in ((w, 1, ValueError, "ws: must be on the cache's device"), (torch.zeros(4), 0, ValueError, "contiguous CUDA"),
                                 (on_gpu(4, 6).t(), 0, ValueError, "contiguous CUDA"), (3, 0, TypeError, "expected a torch tensor")):
        with pytest.raises(error, match=text):
            binding._room_on(bad, "ws", at)
    with pytest.raises(TypeError):
        binding._room_on(w, "ws")


def test_a_cache_has_its_tensors_on_one_device_and_of_one_kind():
    k = on_gpu(4, 2, 16, 64, dtype=torch.bfloat16)
    table, n, acc = on_gpu(1, 2), on_gpu(1), on_gpu(1, 2, 32, dtype=torch.float32)
    moa.KVCache(k, k, table, n, pos=on_gpu(1, 2, 32), seen=on_gpu(1), score=acc)
    for kw, text in ((dict(table=on_gpu(1, 2, at=1)), "table: must be on"), (dict(v=on_gpu(4, 2, 16, 64, dtype=torch.bfloat16, at=1)), "v: must be on"),
                     (dict(len=on_gpu(1, dtype=torch.int64)), "len: dtype"), (dict(score=on_gpu(1, 2, 31, dtype=torch.float32)), "score: 62 elements"),
                     (dict(pos=on_gpu(1, 2, 32, at=1)), "pos: must be on"), (dict(v=on_gpu(4, 2, 16, 64, dtype=torch.float32)), "v: dtype")):
        d = dict(k=k, v=k, table=table, len=n, score=acc)
        d.update(kw)
        with pytest.raises(ValueError, match=text):
            moa.KVCache(**d)


def test_shapes_the_calls_refuse():
    k = on_gpu(4, 2, 16, 64, dtype=torch.bfloat16)
    c = moa.KVCache(k, k, on_gpu(1, 2), on_gpu(1))
    new = lambda *shape: on_gpu(*shape, dtype=torch.bfloat16)
    for kn, vn in ((new(1, 2, 64), new(1, 2, 64)), (new(2, 2, 1, 64), new(2, 2, 1, 64)), (new(1, 2, 1, 64), new(1, 2, 2, 64)),
                   (new(1, 4, 1, 64), new(1, 4, 1, 64)), (new(1, 2, 1, 32), new(1, 2, 1, 32))):
        with pytest.raises(ValueError, match="of the cache"):
            moa.kv_append(c, kn, vn)
    for q in (new(1, 4, 32), new(2, 4, 64), new(1, 256)):
        with pytest.raises(ValueError, match="of the cache"):
            moa.decode_attn(c, q, q, None)


def test_numbers_beyond_32_bits_are_refused_not_wrapped(monkeypatch):
    monkeypatch.setattr(moa.KVCache, "_stream", lambda self, stream: None)     # (nothing gets as far as a launch)
    k = on_gpu(4, 2, 16, 64, dtype=torch.bfloat16)
    c = moa.KVCache(k, k, on_gpu(1, 2), on_gpu(1), pos=on_gpu(1, 2, 32), seen=on_gpu(1), score=on_gpu(1, 2, 32, dtype=torch.float32))
    for budget, recent in ((2 ** 32 + 1000, 0), (-2 ** 32 + 1000, 0), (1000, 2 ** 32), (1000, -2 ** 32)):
        with pytest.raises(ValueError, match="32 bits"):
            moa.kv_evict(c, budget, recent, None)
    for call in (moa.kv_evict_workspace_bytes, moa.decode_attn_workspace_bytes):
        with pytest.raises(ValueError, match="32 bits"):
            call(c, 2 ** 32 + 4)
    many = torch.zeros(1, dtype=torch.bfloat16).expand(2 ** 32 + 4, 1, 1, 1).as_subclass(OnGpu)
    with pytest.raises(ValueError, match="32 bits"):
        moa.KVCache(many, many, on_gpu(1, 2), on_gpu(1))
    one = on_gpu(4, 1, 16, 1, dtype=torch.bfloat16)
    c = moa.KVCache(one, one, on_gpu(1, 2), on_gpu(1))
    with pytest.raises(ValueError, match="32 bits"):
        moa.kv_append(c, many.view(1, 1, -1, 1), many.view(1, 1, -1, 1))
    with pytest.raises(ValueError, match="32 bits"):
        moa.decode_attn(c, many.view(1, -1, 1), many.view(1, -1, 1), None)


def test_a_caches_tensors_stay_the_checked_ones():
    k = on_gpu(4, 2, 16, 64, dtype=torch.bfloat16)
    table = on_gpu(1, 2)
    c = moa.KVCache(k, k, table, on_gpu(1))
    for name in ("k", "v", "table", "len", "pos", "seen", "score"):
        with pytest.raises(AttributeError):
            setattr(c, name, on_gpu(1, 2))
    assert c.table is table and c.k is k and c.pos is None

"""What the calls on a cache held in 8 bits, on pages and on queries and keys refuse, before anything is launched (no GPU needed)."""
import ctypes as C

import pytest
import torch

import paper_2410_03804_amd as moa
from paper_2410_03804_amd import binding

FAKE = 1 << 20          # an address that is never dereferenced
lib = binding._lib
NULL, SHAPE, RANGE, DTYPE, WORKSPACE = -1, -2, -4, -5, -6


def cache(**kw):
    d = dict(dtype=moa.BF16, n_kv_heads=8, head_dim=128, B=2, n_pages=100, page_size=16, max_pages=40, k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE,
             table=FAKE, len=FAKE)
    d.update(kw)
    return binding._KvqCache(**d)


def ref(c):
    return None if c is None else C.byref(c)


def append(c, k=FAKE, v=FAKE, M=1):
    return lib.moa_kvq_append(ref(c), k, v, M, None, None, None, None)


def append_rows(c, k=FAKE, v=FAKE, T=5, ks=1024, vs=1024, off=FAKE):
    return lib.moa_kvq_append_rows(ref(c), k, ks, v, vs, T, off, None, None, None)


def read(c, P=10, k=FAKE, v=FAKE):
    return lib.moa_kvq_read(ref(c), P, k, v, None, None)


def decode_bytes(c, H=32):
    n = C.c_size_t(0)
    return lib.moa_kvq_decode_attn_workspace_bytes(ref(c), H, C.byref(n)), n.value


def decode(c, H=32, q=FAKE, out=FAKE, ws=FAKE, ws_bytes=1 << 40):
    return lib.moa_kvq_decode_attn(ref(c), H, q, out, None, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=2), DTYPE), (dict(n_kv_heads=0), SHAPE), (dict(head_dim=0), SHAPE), (dict(head_dim=257), SHAPE), (dict(B=0), SHAPE),
    (dict(n_pages=0), SHAPE), (dict(page_size=0), SHAPE), (dict(max_pages=-1), SHAPE), (dict(k=None), NULL), (dict(v=None), NULL),
    (dict(table=None), NULL), (dict(len=None), NULL), (dict(k_scale=None), NULL), (dict(v_scale=None), NULL),
    (dict(max_pages=1 << 27), SHAPE), (dict(n_pages=1 << 30), SHAPE), (dict(n_pages=2 ** 31 // 128), SHAPE), (dict(B=1 << 18), SHAPE),
    (dict(k_scale=FAKE + 1), SHAPE), (dict(v_scale=FAKE + 2), SHAPE), (dict(table=FAKE + 2), SHAPE),
])
def test_every_call_refuses_such_a_cache(kw, status):
    c = cache(**kw)
    assert append(c) == append_rows(c) == read(c) == decode(c) == decode_bytes(c)[0] == status
    assert append_rows(c, T=0) == status
    assert append(None) == append_rows(None) == read(None) == decode(None) == decode_bytes(None)[0] == NULL


def test_append_arguments():
    assert append(cache(), k=None) == NULL and append(cache(), v=None) == NULL
    assert append(cache(), M=0) == SHAPE and append(cache(), M=(1 << 24) + 1) == SHAPE and append(cache(head_dim=256), M=1 << 24) == SHAPE
    assert append(cache(), k=FAKE + 1) == SHAPE and append(cache(dtype=moa.F32), v=FAKE + 2) == SHAPE
    assert append(cache(B=70000, n_kv_heads=1)) == SHAPE
    # blocks of all heads are counted in 32 bits
    many = dict(n_kv_heads=256, head_dim=8, n_pages=4)
    assert append(cache(**many), M=(1 << 21) + 1) == SHAPE and append_rows(cache(**many), T=(1 << 21) + 1, ks=2048, vs=2048) == SHAPE
    assert append_rows(cache(), k=None) == NULL and append_rows(cache(), off=None) == NULL
    assert append_rows(cache(), T=-1) == SHAPE and append_rows(cache(), T=(1 << 24) + 1) == SHAPE
    assert append_rows(cache(), ks=1023) == SHAPE and append_rows(cache(), vs=-1024) == SHAPE and append_rows(cache(), ks=1 << 60) == SHAPE
    assert append_rows(cache(), T=0, k=None, v=None, off=None) == 0                        # an empty batch: nothing is launched


def test_read_arguments():
    assert read(cache(), k=None) == NULL and read(cache(), v=None) == NULL and read(cache(), P=0) == SHAPE
    assert read(cache(), P=1 << 25) == SHAPE and read(cache(), v=FAKE + 1) == SHAPE and read(cache(n_kv_heads=40000, B=1, n_pages=4)) == SHAPE


def test_decode_arguments():
    assert decode(cache(), H=0) == SHAPE and decode(cache(), H=12) == SHAPE
    assert decode(cache(), q=None) == NULL and decode(cache(), out=None) == NULL
    assert decode(cache(), q=FAKE + 1) == SHAPE and decode(cache(dtype=moa.F32), out=FAKE + 2) == SHAPE
    assert decode(cache(B=1 << 17), H=64) == SHAPE
    assert decode(cache(max_pages=1 << 24, B=128), H=64) == SHAPE             # tiles are counted in 32 bits
    rc, n = decode_bytes(cache())
    assert rc == 0 and n > 0
    assert decode(cache(), ws_bytes=n - 1) == WORKSPACE and decode(cache(), ws=None) == WORKSPACE and decode(cache(), ws=FAKE + 16) == WORKSPACE
    assert lib.moa_kvq_decode_attn_workspace_bytes(C.byref(cache()), 32, None) == NULL


def reserve(B=4, n_pages=100, page=16, mp=10, T=64, **kw):
    d = dict(len=FAKE, n_new=FAKE, seen=None, table=FAKE, free=FAKE, n_free=FAKE, off=FAKE, got=FAKE, pos=None, slot=None)
    d.update(kw)
    return lib.moa_kv_reserve(B, n_pages, page, mp, d["len"], d["n_new"], d["seen"], d["table"], d["free"], d["n_free"], T, d["off"], d["got"], d["pos"], d["slot"], None, None)


def release(B=4, n_pages=100, page=16, mp=10, **kw):
    d = dict(len=FAKE, table=FAKE, free=FAKE, n_free=FAKE)
    d.update(kw)
    return lib.moa_kv_release(B, n_pages, page, mp, d["len"], d["table"], d["free"], d["n_free"], None, None)


@pytest.mark.parametrize("kw", [dict(B=0), dict(n_pages=0), dict(page=0), dict(mp=0), dict(B=(1 << 20) + 1), dict(mp=1 << 27), dict(n_pages=1 << 28),
                                dict(B=1 << 20, mp=1 << 12)], ids=str)
def test_pages_of_impossible_sizes(kw):
    assert reserve(**kw) == SHAPE and release(**kw) == SHAPE


def test_pages_arguments():
    for name in ("len", "table", "free", "n_free"):
        assert reserve(**{name: None}) == NULL and release(**{name: None}) == NULL
        assert reserve(**{name: FAKE + 2}) == SHAPE and release(**{name: FAKE + 2}) == SHAPE
    for name in ("n_new", "off", "got"):
        assert reserve(**{name: None}) == NULL and reserve(**{name: FAKE + 1}) == SHAPE
    for name in ("seen", "pos", "slot"):
        assert reserve(**{name: FAKE + 3}) == SHAPE
    assert reserve(T=-1) == SHAPE and reserve(T=(1 << 21) + 1) == SHAPE


def rope(dtype=moa.BF16, H=32, Hkv=8, T=5, dh=128, theta=1e4, eps=1e-6, rot=128, **kw):
    d = dict(q=FAKE, qs=6144, k=FAKE, ks=6144, gq=None, gk=None, pos=FAKE, qo=FAKE, qos=4096, ko=FAKE, kos=1024)
    d.update(kw)
    return lib.moa_qk_norm_rope(dtype, d["q"], d["qs"], H, d["k"], d["ks"], Hkv, T, dh, d["gq"], d["gk"], eps, d["pos"], theta, rot, d["qo"], d["qos"], d["ko"], d["kos"], None)


def test_norm_and_rotation_arguments():
    assert rope(dtype=2) == DTYPE
    for kw in (dict(dh=0, rot=0), dict(dh=257), dict(H=-1), dict(Hkv=-1), dict(T=-1), dict(T=(1 << 23) + 1), dict(H=(1 << 20) + 1), dict(rot=-2), dict(rot=130),
               dict(rot=127), dict(qs=4095), dict(ks=1023), dict(qos=4095), dict(kos=0), dict(qs=1 << 61), dict(q=FAKE + 1), dict(ko=FAKE + 1),
               dict(gq=FAKE + 1), dict(pos=FAKE + 2), dict(dtype=moa.F32, k=FAKE + 2)):
        assert rope(**kw) == SHAPE, kw
    for kw in (dict(q=None), dict(k=None), dict(qo=None), dict(ko=None), dict(pos=None)):
        assert rope(**kw) == NULL, kw
    for kw in (dict(theta=0.0), dict(theta=-1.0), dict(theta=float("nan")), dict(theta=float("inf")), dict(gq=FAKE, eps=-1e-6), dict(gk=FAKE, eps=float("nan"))):
        assert rope(**kw) == RANGE, kw
    # nothing to do: nothing is launched, and nothing looked at
    assert rope(T=0, q=None, k=None, pos=None) == 0 and rope(H=0, Hkv=0, q=None, k=None) == 0


# ---------------------------------------------------------------- the binding

class OnGpu(torch.Tensor):
    """Stands in for a tensor on the GPU with that index."""
    is_cuda = True

    def get_device(self):
        return getattr(self, "at", 0)


def on_gpu(*shape, dtype=torch.int32, at=0):
    t = torch.zeros(*shape, dtype=torch.uint8 if dtype == torch.float8_e4m3fn else dtype)
    t = (t.view(dtype) if dtype == torch.float8_e4m3fn else t).as_subclass(OnGpu)
    t.at = at
    return t


E4 = torch.float8_e4m3fn
F32, BF16 = torch.float32, torch.bfloat16


def quant(**kw):
    d = dict(k=on_gpu(4, 2, 40, 64, dtype=E4), v=on_gpu(4, 2, 40, 64, dtype=E4), k_scale=on_gpu(4, 2, 3, dtype=F32), v_scale=on_gpu(4, 2, 3, dtype=F32),
             table=on_gpu(1, 2), len=on_gpu(1), dtype=BF16)
    d.update(kw)
    return moa.QuantKVCache(**d)


def test_a_quantised_cache_has_its_tensors_of_one_kind():
    c = quant()
    for kw, text in ((dict(v=on_gpu(4, 2, 39, 64, dtype=E4)), "same shape"), (dict(dtype=torch.float16), "expected float32 or bfloat16"),
                     (dict(k_scale=on_gpu(4, 2, 2, dtype=F32)), "k_scale and v_scale: must be"), (dict(v_scale=on_gpu(4, 1, 3, dtype=F32)), "must be"),
                     (dict(k=on_gpu(4, 2, 40, 64, dtype=torch.uint8), v=on_gpu(4, 2, 40, 64, dtype=torch.uint8)), "k: dtype"), (dict(v_scale=on_gpu(4, 2, 3, dtype=BF16)), "v_scale: dtype"),
                     (dict(table=on_gpu(1, 2, at=1)), "table: must be on"), (dict(len=on_gpu(0)), "len: 0 elements"), (dict(k=torch.zeros(4, 2, 40, 64, dtype=torch.uint8).view(E4)), "CUDA")):
        with pytest.raises(ValueError, match=text):
            quant(**kw)
    for name in ("k", "v", "k_scale", "v_scale", "table", "len"):
        with pytest.raises(AttributeError):
            setattr(c, name, on_gpu(1, 2))


def test_shapes_the_quantised_calls_refuse(monkeypatch):
    monkeypatch.setattr(moa.QuantKVCache, "_stream", lambda self, stream: None)
    c = quant()
    new = lambda *shape, **kw: on_gpu(*shape, dtype=BF16, **kw)
    for shape in ((1, 2, 64), (2, 2, 1, 64), (1, 4, 1, 64), (1, 2, 1, 32)):
        with pytest.raises(ValueError, match="of the cache"):
            moa.kvq_append(c, new(*shape), new(*shape))
        with pytest.raises(ValueError, match="of the cache"):
            moa.kvq_read(c, new(*shape), new(*shape))
    with pytest.raises(ValueError, match="of the cache"):
        moa.kvq_append(c, new(1, 2, 1, 64), new(1, 2, 2, 64))
    with pytest.raises(ValueError, match="path: 4 elements per sequence"):
        moa.kvq_append(c, new(1, 2, 3, 64), new(1, 2, 3, 64), path=on_gpu(2, 4))
    for shape in ((1, 4, 32), (2, 4, 64), (1, 256)):
        with pytest.raises(ValueError, match="of the cache"):
            moa.kvq_decode_attn(c, new(*shape), new(*shape), None)
    off = on_gpu(2)
    for k, v, text in ((new(5, 2, 32), new(5, 2, 64), r"k_new: must be \[T, 2, 64\]"), (new(5, 2, 64), new(4, 2, 64), "same number of rows"),
                       (new(5, 2, 64), on_gpu(5, 2, 64, dtype=F32), "v_new: dtype"), (new(5, 2, 64, at=1), new(5, 2, 64), "same device"),
                       (new(5, 64, 2).transpose(1, 2), new(5, 2, 64), "behind each other"), (new(1, 2, 64).expand(5, 2, 64), new(5, 2, 64), "behind each other"),
                       (torch.zeros(5, 2, 64, dtype=BF16), new(5, 2, 64), "CUDA")):
        with pytest.raises(ValueError, match=text):
            moa.kvq_append_rows(c, k, v, off)
    with pytest.raises(TypeError):
        moa.kvq_append_rows(c, 3, new(5, 2, 64), off)
    with pytest.raises(ValueError, match="tok_off: 1 elements"):
        moa.kvq_append_rows(c, new(5, 2, 64), new(5, 2, 64), on_gpu(1))
    with pytest.raises(ValueError, match="32 bits"):
        moa.kvq_decode_attn_workspace_bytes(c, 2 ** 32 + 4)


def test_rows_that_lie_apart():
    x = on_gpu(6, 9, 64, dtype=BF16)
    part = x[:, 2:5]
    assert binding._rows_on(part, BF16, 3, 64, "x", 0) == (part.data_ptr(), 9 * 64)
    assert binding._rows_on(x[:1, 2:5], BF16, 3, 64, "x", 0)[1] == 9 * 64 or binding._rows_on(x[:1, 2:5], BF16, 3, 64, "x", 0)[1] == 3 * 64
    assert binding._rows_on(x[:0, 2:5], BF16, 3, 64, "x", 0)[1] == 3 * 64
    with pytest.raises(TypeError):
        binding._rows_on(part, BF16, 3, 64, "x")
    with pytest.raises(ValueError, match=r"x: must be \[T, 3, 64\]"):
        binding._rows_on(part[0], BF16, 3, 64, "x", 0)


def test_pages_the_binding_refuses(monkeypatch):
    monkeypatch.setattr(binding, "_device_of", lambda t, stream: (0, None))
    ok = dict(table=on_gpu(3, 4), length=on_gpu(3), n_new=on_gpu(3), page_size=16, free=on_gpu(20), n_free=on_gpu(1), tok_off=on_gpu(4), n_got=on_gpu(3),
              pos=on_gpu(9), slot=on_gpu(9))
    for kw, error, text in ((dict(tok_off=on_gpu(3)), ValueError, "tok_off: 3 elements"), (dict(length=on_gpu(2)), ValueError, "length: 2"), (dict(n_got=on_gpu(2)), ValueError, "n_got"),
                            (dict(pos=on_gpu(9, dtype=torch.int64)), ValueError, "pos: dtype"), (dict(slot=on_gpu(9, at=1)), ValueError, "slot: must be on"),
                            (dict(rows=10), ValueError, "pos: 9 elements"), (dict(page_size=2 ** 32 + 16), ValueError, "32 bits"), (dict(page_size=1.5), TypeError, None),
                            (dict(n_free=on_gpu(0)), ValueError, "n_free"), (dict(seen=on_gpu(2)), ValueError, "seen")):
        with pytest.raises(error, match=text):
            moa.kv_reserve(**{**ok, **kw})
    with pytest.raises(ValueError, match="table: dtype"):
        moa.kv_release(on_gpu(3, 4, dtype=torch.int64), on_gpu(3), 16, on_gpu(20), on_gpu(1))


def test_norm_and_rotation_the_binding_refuses(monkeypatch):
    monkeypatch.setattr(binding, "_device_of", lambda t, stream: (0, None))
    x = lambda *s, dtype=BF16, **kw: on_gpu(*s, dtype=dtype, **kw)
    ok = dict(q=x(5, 4, 64), k=x(5, 2, 64), q_out=x(5, 4, 64), k_out=x(5, 2, 64), pos=on_gpu(5))
    for kw, text in ((dict(q=None, k=None), "one of them"), (dict(k=x(4, 2, 64)), "same number of rows"), (dict(k=x(5, 2, 32)), r"k: must be"), (dict(q=x(5, 4, 64, dtype=torch.float16)), "dtype"),
                     (dict(k=x(5, 2, 64, dtype=F32)), "k: dtype"), (dict(q_out=None), "q_out: must be as q"), (dict(k_out=x(5, 3, 64)), "k_out: must be as k"), (dict(pos=on_gpu(4)), "pos: 4 elements"),
                     (dict(gq=x(63)), "gq: 63"), (dict(gk=x(64, dtype=F32)), "gk: dtype"), (dict(pos=on_gpu(5, at=1)), "pos: must be on"), (dict(q_out=x(5, 4, 64, at=2)), "same device")):
        with pytest.raises(ValueError, match=text):
            moa.qk_norm_rope(**{**ok, **kw})
    with pytest.raises(ValueError, match="32 bits"):
        moa.qk_norm_rope(**ok, rot_dim=2 ** 32)

"""Tensors whose sequences are further apart than a call on a cache of pages takes them to be are refused, not misread (no GPU needed)."""
import pytest
import torch

import paper_2410_03804_amd as moa
from test_kv_refusals import on_gpu

B, Hkv, dh, cap = 2, 3, 64, 32


def cache(**kw):
    k = on_gpu(4, Hkv, 16, dh, dtype=torch.bfloat16)
    return moa.KVCache(k, k, on_gpu(B, 2), on_gpu(B), **kw)


def test_positions_and_accounts_of_another_capacity():
    i32, f32 = torch.int32, torch.float32
    for shape in ((B, Hkv, cap + 1), (B, Hkv + 1, cap), (B, 2 * Hkv * cap)):
        with pytest.raises(ValueError, match="pos: "):
            cache(pos=on_gpu(*shape, dtype=i32), seen=on_gpu(B))
        with pytest.raises(ValueError, match="score: "):
            cache(score=on_gpu(*shape, dtype=f32))
    # the same rows seen otherwise, or of more sequences than there are
    for shape in ((B, Hkv, cap), (B, Hkv, 2, 16), (B, Hkv * cap), (B * Hkv, cap), (B * Hkv * cap,), (B * Hkv * cap + 5,), (B + 3, Hkv, cap)):
        cache(pos=on_gpu(*shape, dtype=i32), seen=on_gpu(B), score=on_gpu(*shape, dtype=f32))


def test_a_path_of_another_tree(monkeypatch):
    class Reached(Exception):
        pass

    def stream(self, stream):
        raise Reached

    monkeypatch.setattr(moa.KVCache, "_stream", stream)                       # (nothing gets as far as a launch)
    c, new = cache(), on_gpu(B, Hkv, 5, dh, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="path: "):
        moa.kv_append(c, new, new, path=on_gpu(B, 8))
    for shape in ((B, 5), (B + 1, 5), (B * 5,)):
        with pytest.raises(Reached):
            moa.kv_append(c, new, new, path=on_gpu(*shape))


def test_a_path_that_is_no_tensor():
    new = on_gpu(B, Hkv, 2, dh, dtype=torch.bfloat16)
    with pytest.raises(TypeError, match="path: expected a torch tensor"):
        moa.kv_append(cache(), new, new, path=[[0, 1], [0, 1]])

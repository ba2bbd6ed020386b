"""Numbers that the calls on a cache of pages take: whole ones only (no GPU needed)."""
import numpy as np
import pytest
import torch

import paper_2410_03804_amd as moa
from test_kv_refusals import on_gpu


@pytest.fixture
def cache(monkeypatch):
    monkeypatch.setattr(moa.KVCache, "_stream", lambda self, stream: None)     # (nothing gets as far as a launch)
    k = on_gpu(4, 2, 16, 64, dtype=torch.bfloat16)
    return moa.KVCache(k, k, on_gpu(1, 2), on_gpu(1), pos=on_gpu(1, 2, 32), seen=on_gpu(1), score=on_gpu(1, 2, 32, dtype=torch.float32))


@pytest.mark.parametrize("bad", [7.9, 8.0, "8", None, np.float32(8)])
def test_a_fraction_is_refused_not_cut(cache, bad):
    for call in (lambda: moa.kv_evict(cache, bad, 1, None), lambda: moa.kv_evict(cache, 8, bad, None), lambda: moa.kv_evict_workspace_bytes(cache, bad),
                 lambda: moa.decode_attn_workspace_bytes(cache, bad)):
        with pytest.raises(TypeError):
            call()


def test_whole_numbers_of_other_types(cache):
    want = moa.kv_evict_workspace_bytes(cache, 8), moa.decode_attn_workspace_bytes(cache, 4)
    for kind in (np.int32, np.int64, lambda n: torch.tensor(n)):
        assert (moa.kv_evict_workspace_bytes(cache, kind(8)), moa.decode_attn_workspace_bytes(cache, kind(4))) == want

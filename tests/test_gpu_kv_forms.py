"""moa_kv_append and moa_kv_evict on an MI355X in forms that a cache may have: accepted nodes in more rows than one launch takes, positions or
accounts alone, a pool of more than 4 GiB."""
import copy

import numpy as np
import pytest
import torch

import paper_2410_03804_amd as moa
from kv_util import Cache
from test_gpu_kv_cache import HEADS, append_reference, evict, new_rows, same, state

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads,M", [("8b", 256), ("tiny", 300), ("d33", 256)])
def test_append_accepted_nodes_of_a_large_tree(heads, M):
    """More than one launch; the same node twice, entries outside the tree, nothing of one sequence, all M of another."""
    lens = [5, 100, 0, 31]
    c = Cache(HEADS[heads], lens, 16, seed=71, accounts=True, room=M)
    k_new, v_new = new_rows(c, M, 71)
    n_new = [4, 0, M, 9]
    path = np.full((4, M), -1, np.int32)
    path[0, :4] = [0, 3, 17, M - 1]
    path[2] = np.random.default_rng(71).integers(0, M, M)
    path[3, :9] = [8, 8, M, 5, -2, 1 << 30, 0, 0, -(1 << 31)]
    want = append_reference(c, k_new, v_new, path.clip(0, M - 1), n_new, lens)
    moa.kv_append(c.moa(), k_new, v_new, path=torch.from_numpy(path).cuda(), n_new=torch.tensor(n_new, dtype=torch.int32, device="cuda"),
                  dev_status=c.status)
    same(state(c), want)
    assert c.status.item() == moa.DEV_BAD_PARENT


@pytest.mark.parametrize("M", [1, 700])
@pytest.mark.parametrize("kept", ["positions", "accounts"])
def test_append_to_positions_or_accounts_alone(kept, M):
    lens = [0, 33, 6]
    c = Cache(HEADS["8b"], lens, 16, seed=72, accounts=True, room=M)
    if kept == "positions":
        c.score = None
    else:
        c.pos = c.seen = None
    k_new, v_new = new_rows(c, M, 72)
    want = append_reference(c, k_new, v_new, None, None, lens)
    moa.kv_append(c.moa(), k_new, v_new, dev_status=c.status)
    same(state(c), want)
    assert c.status.item() == 0


def test_pages_beyond_4_gib():
    """Rows appended to and moved between pages at the end of a large pool: as in a small one."""
    near = Cache(HEADS["8b"], [600, 700], 64, seed=73, accounts=True, room=40, spare=0)
    n_pages = (5 << 30) // (8 * 64 * 128 * 2) + 1
    far = copy.copy(near)
    at = torch.arange(near.k.shape[0], device="cuda") + n_pages - near.k.shape[0]
    for name in ("k", "v"):
        pool = torch.empty(n_pages, 8, 64, 128, dtype=torch.bfloat16, device="cuda")
        pool[at] = getattr(near, name)
        setattr(far, name, pool)
    far.t_table = torch.where(near.t_table < near.k.shape[0], near.t_table + int(at[0]), near.t_table)
    for name in ("t_len", "pos", "seen", "score", "status"):
        setattr(far, name, getattr(near, name).clone())
    k_new, v_new = new_rows(near, 40, 73)
    for c in (near, far):
        moa.kv_append(c.moa(), k_new, v_new, dev_status=c.status)
        evict(c, 300, 50)
        assert c.status.item() == 0
    far.k, far.v = far.k[at].contiguous(), far.v[at].contiguous()
    assert near.t_len.tolist() == [300, 300]
    same(state(far), state(near))

"""The second launch of moa_kvq_decode_attn where a workgroup joins several query heads, and the first one over the lengths of many sequences.

test_kvq_join_plan.py checks, without a GPU, that these cases are all the forms that the second launch has."""
import numpy as np
import pytest
import torch

import kvq_util as U
import paper_2410_03804_amd as moa

PAGE = 16
# name -> (query heads, KV heads, head_dim, sequences): what the plan then gives a workgroup
SHAPES = {
    "4 heads of 4": (32, 8, 128, 64),
    "3 heads of 8, 2 in the last": (16, 2, 128, 100),
    "2 heads of 4": (4, 1, 64, 256),
    "3 heads of 3": (6, 2, 80, 256),
    "8 heads of 8": (8, 1, 64, 512),
    "5 heads of 7, 2 in the last": (7, 1, 208, 384),
    "9 heads of 12, 3 in the last": (12, 1, 144, 400),
    "16 heads of 16": (16, 1, 128, 512),
    "16 heads of 16, two passes": (16, 1, 256, 512),
    "15 heads of 15, two passes, the second not full": (15, 1, 240, 600),
    "9 heads of 9, two passes": (9, 1, 256, 600),
    "16 heads of 20, 4 in the last tile": (20, 1, 64, 300),
    "11 heads of 23, 5 and then 7 in the last": (23, 1, 192, 180),
    "12 heads of 16, 4 in the last, two passes": (16, 1, 224, 400),
    "14 heads of 14, of 16 dims": (14, 1, 16, 700),
    "16 heads of 33, 1 in the last tile": (33, 1, 48, 260),
    "2 heads of 9, 1 in the last": (9, 1, 64, 150),
    "16 heads of 46, 14 in the last tile, two passes": (46, 1, 160, 171),
    "16 heads of 24, 8 in the last tile": (24, 1, 128, 256),
    "16 heads of 40, 8 in the last tile, of 256 dims": (40, 1, 256, 171),
    "1 head": (32, 8, 128, 6),
    "1 head of 176 dims": (3, 1, 176, 4),
    "1 head of 256 dims": (3, 1, 256, 5),
}
CASES = {f"{dtype} {name}": (*heads, dtype, B) for name, (*heads, B) in SHAPES.items() for dtype in ("bf16", "f32")}
LONGEST = 1400


def lengths(B, seed):
    """Mostly short ones, some empty, a few that take many runs; the capacity is beyond what one workgroup a pair is for."""
    rng = np.random.default_rng(seed)
    lens = rng.integers(0, 90, B)
    lens[rng.random(B) < 0.1] = 0
    for n in (LONGEST, 1025, 700, 321):
        lens[rng.integers(0, B)] = n
    lens[B // 2] = LONGEST
    return [int(n) for n in lens]


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(CASES))
def test_join(name):
    from test_gpu_kvq_decode import attend, both, queries

    H, Hkv, dh, dtype, B = CASES[name]
    c = U.QCache((H, Hkv, dh, dtype), lengths(B, seed=dh + B), PAGE, seed=B + H)
    q = queries(c)
    out = both(c, q, name)
    empty = [b for b, n in enumerate(c.lens) if n == 0]
    assert c.status.item() == (moa.DEV_EMPTY_KEYS if empty else 0)
    assert torch.all(out[empty] == 0)
    assert torch.equal(out, attend(c, q))


@pytest.mark.gpu
def test_what_is_not_a_number_stays_with_its_head():
    """A head without a softmax among the four that a workgroup joins, a slot without a page, and a value that is no number."""
    from test_gpu_kvq_decode import attend, queries

    c = U.QCache((32, 8, 128, "bf16"), lengths(64, seed=3), PAGE, seed=4)
    b = 32
    c.table[b, 40] = -1
    c.codes[1][c.table[b, 50], 2, 5, 7] = U.NAN                # a value: its dimension of the four heads 8 .. 11
    c.upload()
    q = queries(c)
    q[b, 13] = float("inf")
    out = U.host(attend(c, q))
    c.codes[1][c.table[b, 50], 2, 5, 7] = 0x40                 # (a number, for the bounds)
    q[b, 13] = 0.0
    want, tol = U.decode_reference(c, q, {(b, 40)})
    fine = np.ones(out.shape, bool)
    fine[b, 8:12, 7] = False
    fine[b, 13] = False
    assert np.all(np.isnan(out[b, 8:12, 7])) and np.all(np.isnan(out[b, 13]))
    assert np.all(np.isfinite(out[fine])) and np.all(np.abs(out - want)[fine] <= tol[fine])
    assert c.status.item() == moa.DEV_BAD_PAGE | (moa.DEV_EMPTY_KEYS if 0 in c.lens else 0)


@pytest.mark.gpu
@pytest.mark.parametrize("heads", [(2, 1, 64, "bf16"), (2, 1, 64, "f32"), (2, 1, 33, "bf16")], ids=str)       # the last one element by element
@pytest.mark.parametrize("B", [64, 65, 4100])
def test_lengths_of_many_sequences(heads, B):
    """Every run finds its first sequence among all lengths, 64 at a time; there are more sequences than runs, and stretches of empty ones."""
    from test_gpu_kvq_decode import both, queries

    lens = lengths(B, seed=B)
    lens[:3] = 0, 0, 0
    if B > 1000:
        lens[300:700] = [0] * 400
        lens[-200:] = [0] * 199 + [1300]
    c = U.QCache(heads, lens, PAGE, seed=B)
    both(c, queries(c), f"{heads} {B}")
    assert c.status.item() == moa.DEV_EMPTY_KEYS

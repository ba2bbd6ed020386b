"""moa_decode_attn on an MI355X where scores are -infinity: keys that are there but have no weight, and rows of nothing else."""
import numpy as np
import pytest
import torch

import paper_2410_03804_amd as moa
from kv_util import Cache, check, decode_reference, workspace
from test_gpu_decode import HEADS, queries, run

pytestmark = pytest.mark.gpu

# lengths that one workgroup has (with a short capacity), that are cut into runs, and that are both
LENS = {"one": [1], "short": [40, 0, 129], "runs": [5000, 3, 0, 2100]}
FORMS = ["8b", "tiny", "mha64", "g20", "g33", "d72", "d33", "d256", "g9f"]
INF = float("inf")


def reference(c, q, skip=()):
    """decode_reference, with NaN (and no bound) in the rows whose scores are all -infinity and in the accounts they are added to."""
    with np.errstate(invalid="ignore"):
        return decode_reference(c, q, skip=skip)


def check_rows(c, q, accumulate):
    want, tol, weight, wtol = reference(c, q)
    before = c.score.cpu().double().numpy()
    out = run(c, q, accumulate=accumulate)
    assert c.status.item() == (moa.DEV_EMPTY_KEYS if 0 in c.lens else 0)
    none = np.isnan(want)
    assert none.any()
    assert np.array_equal(torch.isnan(out).cpu().numpy(), none)
    check(torch.where(torch.from_numpy(none).cuda(), torch.zeros_like(out), out), np.where(none, 0, want), np.where(none, 0, tol), "out")
    if not accumulate:
        assert np.array_equal(c.score.cpu().double().numpy(), before)
        return
    for b, n in enumerate(c.lens):
        for h in range(c.Hkv):
            got = c.score[b, h].cpu().double().numpy()
            assert np.array_equal(got[n:], before[b, h, n:])
            if none[b, h * c.H // c.Hkv:(h + 1) * c.H // c.Hkv].any():
                assert np.isnan(got[:n]).all()
            else:
                bound = wtol[b, h, :n] + 2.0 ** -23 * (np.abs(before[b, h, :n]) + weight[b, h, :n])
                assert np.all(np.abs(got[:n] - before[b, h, :n] - weight[b, h, :n]) <= bound)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("lens", list(LENS))
@pytest.mark.parametrize("heads", FORMS)
def test_a_row_of_nothing_but_minus_infinity_has_no_softmax(heads, lens, accumulate):
    """An infinite element of a query whose keys all have the same sign there: NaN, as the softmax of such a row is, and not the zeros
    and the status of a sequence without keys.  The other heads keep their results."""
    c = Cache(HEADS[heads], LENS[lens], 16, seed=31, accounts=True)
    c.k[..., 0] = c.k[..., 0].abs() + 0.5                   # (NaN stays where nothing is held)
    q = queries(c, 31)
    q[:, 0, 0] = -INF
    check_rows(c, q, accumulate)


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("at", ["first", "middle", "last"])
@pytest.mark.parametrize("heads", FORMS)
def test_one_key_has_all_the_weight(heads, at, accumulate):
    """All keys but one give -infinity: its weight is one and its value the result, exactly, whatever runs of nothing but -infinity
    come before and after it."""
    lens = [5000, 129, 1]
    c = Cache(HEADS[heads], lens, 16, seed=32, accounts=True)
    q = queries(c, 32).abs() + 0.5
    want, weight = torch.zeros_like(q), np.zeros((len(lens), c.Hkv, c.cap))
    for b, n in enumerate(lens):
        one = dict(first=0, middle=n // 2, last=n - 1)[at]
        want[b] = c.v[int(c.table[b, one // 16]), :, one % 16].repeat_interleave(c.H // c.Hkv, dim=0)
        weight[b, :, one] = c.H // c.Hkv
        for page in range(-(-n // 16)):
            rows = [s % 16 for s in range(16 * page, min(16 * page + 16, n)) if s != one]
            c.k[int(c.table[b, page]), :, rows, 0] = -INF
    before = c.score.cpu().double().numpy()
    assert torch.equal(run(c, q, accumulate=accumulate), want) and c.status.item() == 0
    got = c.score.cpu().double().numpy()
    assert np.all(np.abs(got - before - (weight if accumulate else 0)) <= 2.0 ** -23 * weight * (weight + np.abs(before)))


@pytest.mark.parametrize("heads", ["8b", "tiny", "d72"])
def test_what_is_left_out_does_not_make_a_row_empty(heads):
    """Keys left out for their pages beside keys whose scores are -infinity: still keys; without the latter, none."""
    c = Cache(HEADS[heads], [40, 700, 32], 16, seed=33, accounts=True)
    skip = {(0, 0), (1, 3), (1, 40), (2, 0), (2, 1)}
    c.k[..., 0] = c.k[..., 0].abs() + 0.5
    q = queries(c, 33)
    q[:, 0, 0] = -INF
    want, tol, _, _ = reference(c, q, skip)
    for b, p in skip:
        c.t_table[b, p] = -1
    out = run(c, q)
    assert c.status.item() == moa.DEV_BAD_PAGE | moa.DEV_EMPTY_KEYS           # (sequence 2 has no keys left)
    assert torch.isnan(out[:2, 0]).all() and (out[2] == 0).all()
    check(out[:, 1:], want[:, 1:], tol[:, 1:], "the other heads")

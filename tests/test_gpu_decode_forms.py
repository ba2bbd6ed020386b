"""moa_decode_attn on an MI355X in every form that its plan can choose: one case each, with accounts and without.

test_decode_plan.py checks, without a GPU, that these cases are all the forms there are."""
import copy

import numpy as np
import pytest

import paper_2410_03804_amd as moa
from kv_util import Cache, check, decode_reference

PAGE = 16
LENS = {"one": [200, 0, 33, 17], "runs": [1300, 0, 129, 5]}
# more than 16 query heads of a KV head in one pass takes 512 tiles of 128 keys
RAGGED = (np.random.default_rng(61).integers(1, 51, 130) * np.where(np.arange(130) % 13, 1, 10)).tolist()
MANY = {"one": [500, 0] + RAGGED[2:], "runs": [600, 0] + RAGGED[2:]}


def _cases():
    """name -> (heads, lengths, elements in front of the pools)"""
    out = {}
    for dh in (64, 56, 128, 96, 256, 200):
        for G in (4, 20) if dh > 128 else (4, 20, 24, 40):
            for kind in ("one", "runs"):
                many = G >= 24
                # (20 heads are two tiles of 16 where there is little work)
                out[f"bf16 d{dh} G{G} {kind}"] = ((G, 1, dh, "bf16") if many else (2 * G, 2, dh, "bf16"), (MANY if many else LENS)[kind], 0)
    for dh in (64, 100, 192):
        for G in (2, 3, 8, 11):
            for kind in ("one", "runs"):
                out[f"f32 d{dh} G{G} {kind}"] = ((2 * G, 2, dh, "f32"), LENS[kind], 0)
    for dtype, dims, offset in (("f32", (60, 128, 252), 1), ("bf16", (33, 100, 255), 0)):
        for dh in dims:
            for G in (2, 5):
                for kind in ("one", "runs"):
                    out[f"{dtype} unaligned d{dh} G{G} {kind}"] = ((2 * G, 2, dh, dtype), LENS[kind], offset)
    return out


CASES = _cases()


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(CASES))
def test_form(name):
    from test_gpu_decode import queries, run

    heads, lens, offset = CASES[name]
    c = Cache(heads, lens, PAGE, seed=61, accounts=True, offset=offset)
    q = queries(c, 61)
    host = copy.copy(c)
    host.k, host.v = c.k.cpu(), c.v.cpu()
    want, tol, weight, wtol = decode_reference(host, q)
    before = c.score.cpu().double().numpy()
    for accumulate in (False, True):
        check(run(c, q, accumulate=accumulate), want, tol, f"{name} {'with' if accumulate else 'without'} accounts")
        # an addition of a weight to an account and one more where there are several row tiles
        after = before + weight if accumulate else before
        check(c.score, after, (wtol + 2.0 ** -23 * (np.abs(before) + weight)) * accumulate, "accounts")
    assert c.status.item() == moa.DEV_EMPTY_KEYS

"""moa_kvq_decode_attn on an MI355X in every form that its plan can choose: one case each.

test_kvq_plan.py checks, without a GPU, that these cases are all the forms there are."""
import pytest

import kvq_util as U
import paper_2410_03804_amd as moa

PAGE = 16
LENS = {"one": [200, 0, 33, 17], "runs": [1300, 0, 129, 5]}


def _cases():
    """name -> (heads, lengths, bytes in front of the codes)"""
    out = {}
    for dtype in ("bf16", "f32"):
        for kind in ("one", "runs"):
            for dh in (64, 48, 128, 80, 256, 176):
                for G in (4, 20):
                    out[f"{dtype} d{dh} G{G} {kind}"] = ((2 * G, 2, dh, dtype), LENS[kind], 0)
            for dh, offset in ((60, 0), (33, 0), (100, 0), (64, 2), (255, 0), (252, 0)):
                for G in (3, 6):
                    out[f"{dtype} elements d{dh} at {offset} G{G} {kind}"] = ((2 * G, 2, dh, dtype), LENS[kind], offset)
            out[f"{dtype} elements d128 G1 {kind}"] = ((1, 1, 126, dtype), LENS[kind], 0)
            out[f"{dtype} elements d127 G5 {kind}"] = ((5, 1, 127, dtype), LENS[kind], 0)
    return out


CASES = _cases()


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(CASES))
def test_form(name):
    from test_gpu_kvq_decode import both, queries

    heads, lens, offset = CASES[name]
    c = U.QCache(heads, lens, PAGE, seed=61, offset=offset)
    both(c, queries(c), name)
    assert c.status.item() == moa.DEV_EMPTY_KEYS

"""moa_qk_norm_rope in every form that its plan can choose: one case each, against the formula in 64 bits.

test_rope_plan.py checks, without a GPU, that these cases are all the forms there are."""
import pytest
import torch

import paper_2410_03804_amd as moa

# head dims by the lanes that a head has: a full one and, where there is one, one that leaves lanes idle; of pieces of 16 bytes and of 8
DIMS = {("bf16", 4): {4: (64, 48), 8: (128, 80), 16: (256, 176)}, ("bf16", 2): {4: (24, 8), 8: (56, 40), 16: (120, 72), 32: (248, 136)},
        ("f32", 4): {4: (32, 8), 8: (64, 40), 16: (128, 72), 32: (256, 136)}, ("f32", 2): {4: (12, 4), 8: (28, 20), 16: (60, 36), 32: (124, 68), 64: (252, 132)}}
TOKENS = {1: (5, 1023), 4: (1027, 4095), 16: (4111, 4096)}


def _cases():
    """name -> (query heads, KV heads, head_dim, type, tokens, dims that are rotated)"""
    out = {}
    for (dtype, words), by_lanes in DIMS.items():
        unit = 8 * words // (2 if dtype == "bf16" else 4)                    # dims of two pieces
        for lanes, dims in by_lanes.items():
            for tokens, Ts in TOKENS.items():
                for dh, T in zip(dims, Ts):
                    H, Hkv = (1, 1) if lanes == 64 else (3, 1) if dh == dims[0] else (2, 3)
                    out[f"{dtype} {4 * words} bytes, d{dh}, {T} tokens"] = (H, Hkv, dh, dtype, T, dh // (2 * unit) * unit)
        out[f"{dtype} {4 * words} bytes, many heads, 4100 tokens"] = (40, 4, by_lanes[8][0], dtype, 4100, unit)
    # pieces of 8 bytes because of the rotated part alone
    for dtype, dh, part in (("bf16", 64, 24), ("f32", 32, 12)):
        for T in (1029, 4099):
            out[f"{dtype} 8 bytes, d{dh} of which {part}, {T} tokens"] = (3, 1, dh, dtype, T, part)
    out["8b prompt"] = (32, 8, 128, "bf16", 1030, 64)
    for dtype in ("bf16", "f32"):
        out[f"{dtype} any, d34, 4103 tokens"] = (2, 1, 34, dtype, 4103, 18)
    return out


CASES = _cases()


@pytest.mark.gpu
@pytest.mark.parametrize("name", list(CASES))
def test_form(name):
    from test_gpu_qk_norm_rope import Case, check

    H, Hkv, dh, dtype, T, part = CASES[name]
    Case(H, Hkv, dh, dtype, T, seed=T + dh).run(what="all dims")
    c = Case(H, Hkv, dh, dtype, T, seed=T + dh, norm=False)
    c.run(rot=part, what="part of them, no norm")
    c.run(what="all, no norm")
    c = Case(H, Hkv, dh, dtype, T, seed=T + dh + 1)
    c.run(rot=0, what="norm alone")
    # either of them alone; the other's results are nobody's to touch
    qo, ko = (torch.full(x.shape, 99.0, dtype=x.dtype, device="cuda") for x in (c.q, c.k))
    moa.qk_norm_rope(c.q, None, qo, None, c.pos, rope_theta=c.theta, rot_dim=part, gq=c.gq)
    assert torch.all(ko == 99.0)
    check(qo, *c.want(c.q, c.gq, part), dtype, "q alone")
    qo.fill_(99.0)
    moa.qk_norm_rope(None, c.k, None, ko, c.pos, rope_theta=c.theta, rot_dim=part, gk=c.gk)
    assert torch.all(qo == 99.0)
    check(ko, *c.want(c.k, c.gk, part), dtype, "k alone")
    # the whole projection's output: what is neither query nor key stays
    rest = c.q.untyped_storage()
    before = torch.tensor([], dtype=c.q.dtype, device="cuda").set_(rest)[:T * (H + 2 * Hkv) * dh].view(T, H + 2 * Hkv, dh)
    values = before[:, H + Hkv:].clone()
    c.run(rot=part, inplace=True, what="in place")
    assert torch.equal(before[:, H + Hkv:], values)

"""The form that the norm and rotation of queries and keys takes (csrc/moa_rope_plan.h: host arithmetic, compiled here with g++), and that
test_gpu_rope_forms.py has a case of every one."""
import ctypes as C
import random
import subprocess
from collections import namedtuple
from pathlib import Path

import pytest

from test_gpu_rope_forms import CASES

CSRC = Path(__file__).resolve().parent.parent / "paper_2410_03804_amd" / "csrc"
Plan = namedtuple("Plan", "words lanes tokens apart")
Form = namedtuple("Form", "dtype plan")


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("rope_plan")
    (d / "plan.cpp").write_text('#include "moa_rope_plan.h"\nextern "C" void plan(int size, int dh, int half, uint64_t at, uint64_t strides, int64_t T, int heads, int *out)\n'
                                "{\n    const moa::RopePlan p = moa::rope_plan(size, dh, half, at, strides, T, heads);\n"
                                "    out[0] = p.words, out[1] = p.lanes, out[2] = p.tokens, out[3] = p.apart;\n}\n")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-O1", "-shared", "-fPIC", f"-I{CSRC}", "-o", str(d / "plan.so"), str(d / "plan.cpp")], check=True)
    f = C.CDLL(str(d / "plan.so")).plan

    def call(size, dh, half, at, strides, T, heads):
        out = (C.c_int * 4)()
        f(C.c_int(size), C.c_int(dh), C.c_int(half), C.c_uint64(at), C.c_uint64(strides), C.c_int64(T), C.c_int(heads), out)
        return Plan(*out[:3], bool(out[3]))
    return call


def form(plan, H, Hkv, dh, dtype, T, rot, at=0, strides=None):
    size = 2 if dtype == "bf16" else 4
    return Form(dtype, plan(size, dh, rot // 2, at, (H + 2 * Hkv) * dh | H * dh | Hkv * dh if strides is None else strides, T, max(H, Hkv)))


def test_every_form_has_a_case(plan):
    have = set()
    for H, Hkv, dh, dtype, T, part in CASES.values():
        # (each case runs with a part of the dims rotated, which is the harder one to have in pieces)
        assert 0 < part < dh or dh in (4, 8), (dh, part)
        have.add(form(plan, H, Hkv, dh, dtype, T, part))
    rng, missing = random.Random(1), {}
    for _ in range(60000):
        dtype, dh = rng.choice(["bf16", "f32"]), rng.choice([64, 128, 256, 8 * rng.randint(1, 32), 4 * rng.randint(1, 64), rng.randint(1, 256)])
        H, Hkv = rng.choice([(32, 8), (1, 1), (rng.randint(1, 40), rng.randint(1, 40))])
        call = (H, Hkv, dh, dtype, int(2 ** rng.uniform(0, 20)), rng.choice([dh // 2 * 2, 0, dh // 4 * 2, 2 * rng.randint(0, dh // 2)]), rng.choice([0, 0, 4, 8, 16]),
                rng.choice([None, None, H * dh + rng.randint(0, 16)]))
        f = form(plan, *call)
        if f not in have:
            missing[f] = call
    assert not missing, "\n".join(f"{f}: {call}" for f, call in missing.items())


def test_cases_are_what_their_names_say(plan):
    """Heads that leave lanes idle and that do not, last workgroups with and without all tokens, of either piece and number of tokens."""
    seen = set()
    for name, (H, Hkv, dh, dtype, T, part) in CASES.items():
        p = form(plan, H, Hkv, dh, dtype, T, part).plan
        if "bytes" not in name:
            continue
        assert p.words == int(name.split()[1]) // 4, (name, p)
        pairs = dh * (2 if dtype == "bf16" else 4) // (8 * p.words)
        assert pairs <= p.lanes < 2 * pairs or p.lanes == 4
        seen.add((dtype, p, pairs < p.lanes, T % p.tokens != 0))
    for dtype in ("bf16", "f32"):
        for words in (4, 2):
            for tokens in (4, 16):
                of = {s[2:] for s in seen if s[0] == dtype and s[1].words == words and s[1].tokens == tokens}
                assert {i for i, _ in of} == {t for _, t in of} == {True, False}, (dtype, words, tokens, of)


def test_a_workgroup_s_threads_and_angles(plan):
    """Lanes of a head are a power of two that holds its pairs of pieces, and divide a wavefront; angles of a workgroup fit its 128 a token."""
    rng = random.Random(2)
    for _ in range(20000):
        size, dh = rng.choice([2, 4]), rng.randint(1, 256)
        half = rng.randint(0, dh // 2)
        at, strides = rng.choice([0, 4, 8, 16, 2 ** 40 + 8]), rng.choice([dh, 4 * dh, rng.randint(1, 5000)])
        p = plan(size, dh, half, at, strides, int(2 ** rng.uniform(0, 23)), rng.randint(1, 200))
        assert p.tokens in (1, 4, 16) and p.apart == (p.words > 0 and p.tokens == 1)
        if p.words:
            elems = 4 * p.words // size
            assert dh % (2 * elems) == half % elems == at % (4 * p.words) == strides % elems == 0
            assert p.lanes in (4, 8, 16, 32, 64) and dh // (2 * elems) <= p.lanes and half <= 128

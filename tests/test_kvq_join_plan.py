"""How the second launch of the attention over a cache held in 8 bits deals query heads to workgroups (csrc/moa_kvq_plan.h: host arithmetic,
compiled here with g++), and that test_gpu_kvq_join.py has a case of every form of it."""
import ctypes as C
import random
import subprocess
from collections import namedtuple
from pathlib import Path

import pytest

from test_gpu_kvq_join import CASES, LONGEST, PAGE

CSRC = Path(__file__).resolve().parent.parent / "paper_2410_03804_amd" / "csrc"
Plan = namedtuple("Plan", "HG rtiles runs per chunks")
JT = 512                              # threads of a workgroup, as in moa_kvq_decode.hip
# of a workgroup: several heads; fewer than the others have; several wavefronts a head for the sums; how often its threads go over its elements, or
# how many of them a result has; whether threads are left over
Form = namedtuple("Form", "dtype several short waves elements idle")


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("kvq_join_plan")
    (d / "plan.cpp").write_text('#include "moa_kvq_plan.h"\nextern "C" void plan(int B, int Hkv, int dh, int cap, int H, int64_t *out)\n'
                                "{\n    const moa::KvqPlan p = moa::kvq_plan(B, Hkv, dh, cap, H, true);\n"
                                "    out[0] = p.HG, out[1] = p.rtiles, out[2] = p.runs, out[3] = p.per, out[4] = p.chunks;\n}\n")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-O1", "-shared", "-fPIC", f"-I{CSRC}", "-o", str(d / "plan.so"), str(d / "plan.cpp")], check=True)
    f = C.CDLL(str(d / "plan.so")).plan

    def call(*args):
        out = (C.c_int64 * 5)()
        f(*[C.c_int(a) for a in args], out)
        return Plan(*out)
    return call


def heads_of_workgroups(p, G):
    """Query heads of each workgroup of a KV head, as k_kvq_join takes them."""
    out = []
    for tile in range(p.rtiles):
        for chunk in range(p.chunks):
            first = chunk * p.per
            heads = range(tile * 16 + first, tile * 16 + first + max(0, min(p.per, min(16, G - tile * 16) - first)))
            out.append(heads)
    return out


def forms(plan, H, Hkv, dh, dtype, B, cap):
    p = plan(B, Hkv, dh, cap, H)
    if not p.runs:
        return set()
    out = set()
    for heads in heads_of_workgroups(p, H // Hkv):
        rows = len(heads)
        if rows == 0:
            continue
        E = rows * dh // 4
        many = "passes" if E > JT else "one" if JT // E == 1 else "groups"
        out.add(Form(dtype, rows > 1, rows < p.per, JT // 64 // rows > 1, many, JT % E != 0 if E <= JT else E % JT != 0))
    return out


def test_every_form_has_a_case(plan):
    have = set()
    for H, Hkv, dh, dtype, B in CASES.values():
        have |= forms(plan, H, Hkv, dh, dtype, B, -(-LONGEST // PAGE) * PAGE)
    rng, missing = random.Random(1), {}
    for _ in range(60000):
        Hkv = rng.choice([1, 1, 2, 4, 8])
        G, dh = rng.choice([1, 2, 3, 4, 5, 8, 9, 12, 15, 16, 17, 20, 32, 33, rng.randint(1, 70)]), 16 * rng.randint(1, 16)
        call = (G * Hkv, Hkv, dh, rng.choice(["bf16", "f32"]), int(2 ** rng.uniform(0, 12)), int(2 ** rng.uniform(9, 16)))
        for f in forms(plan, *call) - have:
            missing[f] = call
    assert not missing, "\n".join(f"{f}: {call}" for f, call in missing.items())


def test_every_head_is_joined_by_one_workgroup(plan):
    rng = random.Random(2)
    for _ in range(5000):
        Hkv, G, dh, B = rng.randint(1, 8), rng.randint(1, 70), 16 * rng.randint(1, 16), int(2 ** rng.uniform(0, 11))
        p = plan(B, Hkv, dh, 1 << 14, G * Hkv)
        assert 1 <= p.per <= p.HG and (p.chunks - 1) * p.per < p.HG <= p.chunks * p.per
        assert sorted(h for heads in heads_of_workgroups(p, G) for h in heads) == list(range(G))
        # one head a workgroup, or at least 512 of them
        assert p.per == 1 or B * Hkv * p.rtiles * p.chunks >= 512

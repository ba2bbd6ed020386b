"""The form that the attention of one token per sequence takes (csrc/moa_decode_plan.h: host arithmetic, compiled here with g++), and that
test_gpu_decode_forms.py has a case of every one."""
import ctypes as C
import random
import subprocess
from collections import namedtuple
from pathlib import Path

import pytest

from test_gpu_decode_forms import CASES, PAGE

CSRC = Path(__file__).resolve().parent.parent / "paper_2410_03804_amd" / "csrc"
Plan = namedtuple("Plan", "HG rtiles runs cap32 part_o part_ml raw")
# the kernel (with what it is instantiated for), whether accounts are kept, one workgroup per pair, several row tiles
Form = namedtuple("Form", "kernel accounts one tiles")


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("decode_plan")
    (d / "plan.cpp").write_text('#include "moa_decode_plan.h"\nextern "C" void plan(int B, int Hkv, int dh, int cap, int H, int accounts, int mfma, int wide, int64_t *out)\n'
                                "{\n    const moa::DecodePlan p = moa::decode_plan(B, Hkv, dh, cap, H, accounts != 0, mfma != 0, wide != 0);\n"
                                "    out[0] = p.HG, out[1] = p.rtiles, out[2] = p.runs, out[3] = p.cap32, out[4] = p.part_o, out[5] = p.part_ml, out[6] = p.raw;\n}\n")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-O1", "-shared", "-fPIC", f"-I{CSRC}", "-o", str(d / "plan.so"), str(d / "plan.cpp")],
                   check=True)
    f = C.CDLL(str(d / "plan.so")).plan

    def call(*args):
        out = (C.c_int64 * 7)()
        f(*[C.c_int(a) for a in args], out)
        return Plan(*out)
    return call


def form(plan, B, H, Hkv, dh, dtype, cap, accounts, offset):
    rows16 = offset == 0 and dh * (2 if dtype == "bf16" else 4) % 16 == 0
    mfma, wide = rows16 and dtype == "bf16", rows16 and dtype == "f32"
    p = plan(B, Hkv, dh, cap, H, accounts, mfma, wide)
    # (as launch_decode goes about it)
    held = 64 if dh <= 64 else 128 if dh <= 128 else 256
    kernel = ("mfma", held, 2 if p.HG > 16 else 1, dh != held) if mfma else (dtype, held, p.HG, wide)
    return Form(kernel, accounts, p.runs == 0, p.rtiles > 1)


def with_a_case(plan):
    out = set()
    for (H, Hkv, dh, dtype), lens, offset in CASES.values():
        cap = -(-max(lens) // PAGE) * PAGE
        out |= {form(plan, len(lens), H, Hkv, dh, dtype, cap, acc, offset) for acc in (False, True)}
    return out


def test_every_form_has_a_case(plan):
    rng = random.Random(1)
    have, missing = with_a_case(plan), {}
    for _ in range(60000):
        Hkv = rng.choice([1, 1, 2, 4, 8])
        G, dh = rng.choice([1, 2, 3, 4, 5, 8, 9, 16, 17, 24, 32, 33, 64, rng.randint(1, 70)]), rng.choice([64, 128, 256, 8 * rng.randint(1, 32), rng.randint(1, 256)])
        cap, B = int(2 ** rng.uniform(0, 16)), int(2 ** rng.uniform(0, 11))
        call = (B, G * Hkv, Hkv, dh, rng.choice(["bf16", "f32"]), cap, rng.random() < 0.5, int(rng.random() < 0.2))
        f = form(plan, *call)
        if f not in have:
            missing[f] = call
    assert not missing, "\n".join(f"{f}: {call}" for f, call in missing.items())


def test_workspace_of_a_plan(plan):
    """Room for the partial results of every run and pair and for a score of every slot and query head; none where one workgroup has a pair."""
    rng = random.Random(2)
    for _ in range(5000):
        Hkv, G, dh, cap, B = rng.randint(1, 8), rng.randint(1, 70), rng.randint(1, 256), int(2 ** rng.uniform(0, 16)), int(2 ** rng.uniform(0, 9))
        kind, acc = rng.choice([(1, 0), (0, 1), (0, 0)]), rng.random() < 0.5
        p = plan(B, Hkv, dh, cap, G * Hkv, acc, *kind)
        assert 1 <= p.HG <= (32 if kind[0] and dh <= 128 else 16 if kind[0] else 8) and (p.rtiles - 1) * p.HG < G <= p.rtiles * p.HG
        pairs = B * Hkv * p.rtiles
        assert p.runs & (p.runs - 1) == 0 and p.cap32 % 32 == 0 and 0 <= p.cap32 - cap < 32
        assert p.part_o >= 4 * (p.runs + pairs) * p.HG * dh * (p.runs > 0) and p.part_ml >= 8 * (p.runs + pairs) * p.HG * (p.runs > 0)
        assert p.raw >= 4 * pairs * p.cap32 * p.HG * acc
        assert all(n % 256 == 0 for n in (p.part_o, p.part_ml, p.raw)) and (p.runs or p.part_o == p.part_ml == 0) and (acc or p.raw == 0)
        assert p.runs or not (acc and p.rtiles > 1)                           # accounts of several row tiles are the second launch's

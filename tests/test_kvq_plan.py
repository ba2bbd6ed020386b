"""The form that the attention over a cache held in 8 bits takes (csrc/moa_kvq_plan.h: host arithmetic, compiled here with g++), and that
test_gpu_kvq_forms.py has a case of every one."""
import ctypes as C
import random
import subprocess
from collections import namedtuple
from pathlib import Path

import pytest

from test_gpu_kvq_forms import CASES, PAGE

CSRC = Path(__file__).resolve().parent.parent / "paper_2410_03804_amd" / "csrc"
Plan = namedtuple("Plan", "HG rtiles runs part_o part_ml")
# the kernel (with what it is instantiated for), one workgroup per pair, several row tiles
Form = namedtuple("Form", "kernel one tiles")


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("kvq_plan")
    (d / "plan.cpp").write_text('#include "moa_kvq_plan.h"\nextern "C" void plan(int B, int Hkv, int dh, int cap, int H, int mfma, int64_t *out)\n'
                                "{\n    const moa::KvqPlan p = moa::kvq_plan(B, Hkv, dh, cap, H, mfma != 0);\n"
                                "    out[0] = p.HG, out[1] = p.rtiles, out[2] = p.runs, out[3] = p.part_o, out[4] = p.part_ml;\n}\n")
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-O1", "-shared", "-fPIC", f"-I{CSRC}", "-o", str(d / "plan.so"), str(d / "plan.cpp")], check=True)
    f = C.CDLL(str(d / "plan.so")).plan

    def call(*args):
        out = (C.c_int64 * 5)()
        f(*[C.c_int(a) for a in args], out)
        return Plan(*out)
    return call


def form(plan, B, H, Hkv, dh, dtype, cap, offset):
    mfma = offset % 16 == 0 and dh % 16 == 0
    p = plan(B, Hkv, dh, cap, H, mfma)
    # (as launch_decode goes about it)
    held = 64 if dh <= 64 else 128 if dh <= 128 else 256
    kernel = (dtype, "mfma", held, dh != held) if mfma else (dtype, held, dh % 4 == 0 and offset % 4 == 0)
    return Form(kernel, p.runs == 0, p.rtiles > 1)


def with_a_case(plan):
    return {form(plan, len(lens), H, Hkv, dh, dtype, -(-max(lens) // PAGE) * PAGE, offset) for (H, Hkv, dh, dtype), lens, offset in CASES.values()}


def test_every_form_has_a_case(plan):
    rng = random.Random(1)
    have, missing = with_a_case(plan), {}
    for _ in range(40000):
        Hkv = rng.choice([1, 1, 2, 4, 8])
        G, dh = rng.choice([1, 2, 3, 4, 5, 8, 9, 16, 17, 32, 33, rng.randint(1, 70)]), rng.choice([64, 128, 256, 16 * rng.randint(1, 16), 4 * rng.randint(1, 64), rng.randint(1, 256)])
        call = (int(2 ** rng.uniform(0, 11)), G * Hkv, Hkv, dh, rng.choice(["bf16", "f32"]), int(2 ** rng.uniform(0, 16)), rng.choice([0, 0, 0, 1, 4, 16]))
        f = form(plan, *call)
        if f not in have:
            missing[f] = call
    assert not missing, "\n".join(f"{f}: {call}" for f, call in missing.items())


def test_workspace_of_a_plan(plan):
    """Room for the partial results of every run and pair, none where one workgroup has a pair; runs are a power of two."""
    rng = random.Random(2)
    for _ in range(5000):
        Hkv, G, dh, cap, B, mfma = rng.randint(1, 8), rng.randint(1, 70), rng.randint(1, 256), int(2 ** rng.uniform(0, 16)), int(2 ** rng.uniform(0, 9)), rng.randint(0, 1)
        p = plan(B, Hkv, dh, cap, G * Hkv, mfma)
        assert 1 <= p.HG <= (16 if mfma else 4) and (p.rtiles - 1) * p.HG < G <= p.rtiles * p.HG
        pairs = B * Hkv * p.rtiles
        assert p.runs & (p.runs - 1) == 0
        assert p.part_o >= 4 * (p.runs + pairs) * p.HG * dh * (p.runs > 0) and p.part_ml >= 8 * (p.runs + pairs) * p.HG * (p.runs > 0)
        assert p.part_o % 256 == p.part_ml % 256 == 0 and (p.runs or p.part_o == p.part_ml == 0)


def places(lens, HB, runs):
    """The list of places dealt to runs as the kernel has it (PlaceList)."""
    total = sum((-(-n // 32) + 1) * HB for n in lens if n)
    log2 = min(runs.bit_length() - 1, max(total, 1).bit_length() - 1)
    first = lambda w: w * total >> log2
    run_of = lambda f: (((f + 1) << log2) - 1) // total
    return total, 1 << log2, first, run_of


def test_places_and_runs_are_each_other_s_inverse():
    rng = random.Random(3)
    for _ in range(300):
        lens, HB, runs = [rng.choice([0, 1, 32, 33, rng.randint(0, 5000)]) for _ in range(rng.randint(1, 40))], rng.randint(1, 9), rng.choice([1024, 2048])
        total, dealt, first, run_of = places(lens, HB, runs)
        assert 1 <= dealt <= runs
        of = {}
        for w in range(dealt):
            for f in range(first(w), first(w + 1)):
                of[f] = w
        assert sorted(of) == list(range(total)) and all(run_of(f) == w for f, w in of.items())
        sizes = [first(w + 1) - first(w) for w in range(dealt)]
        assert max(sizes) - min(sizes) <= 1 and (min(sizes) >= 1 or total < 1)
        # the runs of a pair are one behind the other, so that the second launch finds a partial result in each; no two pairs' have the same number
        f, pair, slots = 0, 0, set()
        for n in lens:
            for _ in range(HB):
                if n:
                    runs_of_it = sorted({of[g] for g in range(f + 1, f + 1 + -(-n // 32))})
                    assert runs_of_it == list(range(run_of(f + 1), run_of(f + -(-n // 32)) + 1))
                    mine = {w + pair for w in runs_of_it}
                    assert not mine & slots and max(mine) < runs + len(lens) * HB
                    slots |= mine
                    f += -(-n // 32) + 1
                pair += 1

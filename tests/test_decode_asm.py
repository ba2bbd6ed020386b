"""The gathering loads into LDS of the decode attention, which are written as inline asm, in the assembly the compiler makes of them
(gfx950 only, no GPU needed)."""
import re
import subprocess

from paper_2410_03804_amd import build


def test_gathers_have_their_wait_state_and_the_counts_hold():
    """Between the write of m0 and the load that uses it stands a wait state, and m0 holds nothing else.  The kernels on the matrix cores
    spill nothing and make no memory access through the general address space: either would be counted among the loads that
    their waits count."""
    src = "moa_decode_attn.hip"
    cmd = [build._hipcc(), *build.FLAGS, *build.SOURCE_FLAGS.get(src, []), "--cuda-device-only", "-S", "-o", "-", str(build.CSRC / src)]
    asm = subprocess.run(cmd, capture_output=True, text=True, check=True).stdout
    lines = [l.split(";")[0].strip() for l in asm.splitlines()]
    lines = [l for l in lines if l and not l.startswith(".")]
    loads = [i for i, l in enumerate(lines) if l.startswith("global_load_lds_dword")]
    assert loads
    for i in loads:
        assert re.fullmatch(r"global_load_lds_dword(x4)? v\[\d+:\d+\], off( nt)?", lines[i]), lines[i]
        assert lines[i - 1] == "s_nop 0" and re.fullmatch(r"s_mov_b32 m0, \w+", lines[i - 2]), lines[i - 2:i + 1]
    assert sum(bool(re.search(r"\bm0\b", l)) for l in lines) == len(loads)
    bodies = re.findall(r"^(\S*k_decode_attn_mfma\S*):(.*?)s_endpgm.*?\.section", asm, flags=re.S | re.M)
    assert len(bodies) == 20
    for name, body in bodies:
        assert "scratch_" not in body and "flat_" not in body, name

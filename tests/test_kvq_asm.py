"""The kernels of the cache held in 8 bits in the assembly the compiler makes of them (gfx950 only, no GPU needed)."""
import re
import subprocess

from paper_2410_03804_amd import build


def assembly(src):
    cmd = [build._hipcc(), *build.FLAGS, *build.SOURCE_FLAGS.get(src, []), "--cuda-device-only", "-S", "-o", "-", str(build.CSRC / src)]
    return subprocess.run(cmd, capture_output=True, text=True, check=True).stdout


def test_gathers_have_their_wait_state_and_the_counts_hold():
    """Between the write of m0 and the load that uses it stands a wait state, and m0 holds nothing else.  The kernels on the matrix cores
    spill nothing and make no memory access through the general address space: either would be counted among the loads that their waits
    count."""
    asm = assembly("moa_kvq_decode.hip")
    lines = [l.split(";")[0].strip() for l in asm.splitlines()]
    lines = [l for l in lines if l and not l.startswith(".")]
    loads = [i for i, l in enumerate(lines) if l.startswith("global_load_lds_dword")]
    assert loads
    for i in loads:
        assert re.fullmatch(r"global_load_lds_dword(x4)? v\[\d+:\d+\], off( nt)?", lines[i]), lines[i]
        assert lines[i - 1] == "s_nop 0" and re.fullmatch(r"s_mov_b32 m0, s\d+", lines[i - 2]), lines[i - 2:i + 1]
    assert sum(bool(re.search(r"\bm0\b", l)) for l in lines) == len(loads)
    bodies = re.findall(r"^(\S*k_kvq_decode_mfma\S*):(.*?)s_endpgm.*?\.section", asm, flags=re.S | re.M)
    assert len(bodies) == 2 * 3 * 2 * 2                    # types, head dims, padded, one workgroup a pair
    for name, body in bodies:
        assert "scratch_" not in body and "flat_" not in body, name
        assert "v_cvt_scalef32_pk_bf16_fp8" in body and "ds_read_b64_tr_b8" in body and "v_mfma_f32_16x16x32_bf16" in body, name


def test_no_kernel_spills():
    for src, kernels in (("moa_kvq_decode.hip", 24 + 12 + 2), ("moa_kvq.hip", 16 + 1 + 4), ("moa_kv_pages.hip", 7), ("moa_qk_norm_rope.hip", 3 * (3 + 4 + 4 + 5) + 2)):
        cmd = [build._hipcc(), *build.FLAGS, "--cuda-device-only", "-c", "-o", "/dev/null", "-Rpass-analysis=kernel-resource-usage", str(build.CSRC / src)]
        said = subprocess.run(cmd, capture_output=True, text=True, check=True).stderr
        scratch = re.findall(r"Function Name: (\S*k_k?[vq]\S*) .*?ScratchSize \[bytes/lane\]: (\d+)", said, flags=re.S)
        assert len(scratch) == kernels, (src, len(scratch))
        assert not [name for name, size in scratch if size != "0"]

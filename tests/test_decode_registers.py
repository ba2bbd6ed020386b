"""No form of the attention of one token per sequence spills registers (gfx950 only, no GPU needed)."""
import re
import subprocess

from paper_2410_03804_amd import build


def test_no_form_spills():
    src = "moa_decode_attn.hip"
    cmd = [build._hipcc(), *build.FLAGS, *build.SOURCE_FLAGS.get(src, []), "--cuda-device-only", "-c", "-o", "/dev/null",
           "-Rpass-analysis=kernel-resource-usage", str(build.CSRC / src)]
    said = subprocess.run(cmd, capture_output=True, text=True, check=True).stderr
    scratch = re.findall(r"Function Name: (\S*k_decode\S*) .*?ScratchSize \[bytes/lane\]: (\d+)", said, flags=re.S)
    assert len(scratch) == 20 + 15 + 2              # on the matrix cores, element by element, the joins
    assert not [name for name, size in scratch if size != "0"]

"""Matrix instructions ignore EXEC: in the assembly of the kernels for shared prefixes whatever narrows EXEC is followed by a jump for
the case that no lane is left before the next of them."""
import os
import re
import subprocess

import pytest

from paper_2502_00425_amd import build
from test_attention_branches import HIPCC, unguarded

KERNELS = ["shared_few_kernel", "shared_both_kernel", "shared_suffix_kernel", "shared_whole_kernel"]


def assembly(source, tmp_path):
    out = tmp_path / "kernels.s"
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run([HIPCC, *flags, "-S", "--cuda-device-only", "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC,
                    os.path.join(build.CSRC, source), "-o", str(out)], check=True, capture_output=True)
    return out.read_text()


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="needs hipcc")
def test_matrix_instructions_run_with_every_lane(tmp_path):
    text = assembly("paged_attention.hip", tmp_path)
    for kernel in KERNELS:
        bodies = re.findall(r"^(\S*%s\S*):[^\n]*\n(.*?)\n\.Lfunc_end" % kernel, text, re.S | re.M)
        assert bodies, kernel
        for name, body in bodies:
            lines = [l.strip() for l in body.split("\n")]
            assert sum("v_mfma" in l for l in lines) >= 2, name
            assert unguarded(lines) == [], name

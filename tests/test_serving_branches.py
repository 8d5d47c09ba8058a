"""Matrix instructions ignore EXEC: in the assembly of the serving kernels whatever narrows EXEC is followed by a jump for
the case that no lane is left before the next of them."""
import os
import re
import subprocess

import pytest

from paper_2502_00425_amd import build
from test_attention_branches import HIPCC, unguarded

KERNELS = {"paged_attention.hip": ["paged_chunk_kernel", "paged_few_kernel"], "lora.hip": ["lora_shrink_kernel", "lora_expand_kernel", "lora_shrink_rows_kernel", "lora_expand_rows_kernel"]}


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="needs hipcc")
@pytest.mark.parametrize("source", list(KERNELS))
def test_matrix_instructions_run_with_every_lane(source, tmp_path):
    out = tmp_path / "kernels.s"
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run([HIPCC, *flags, "-S", "--cuda-device-only", "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC,
                    os.path.join(build.CSRC, source), "-o", str(out)], check=True, capture_output=True)
    bodies = re.findall(r"^(\S*(?:%s)\S*):[^\n]*\n(.*?)\n\.Lfunc_end" % "|".join(KERNELS[source]), out.read_text(), re.S | re.M)
    assert bodies
    for name, body in bodies:
        lines = [l.strip() for l in body.split("\n")]
        assert sum("v_mfma" in l for l in lines) >= 2, name
        assert unguarded(lines) == [], name

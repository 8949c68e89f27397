"""The wait states in front of the direct global -> LDS loads of the attention over pages, on every path of its assembly, and the
scratch memory of its kernels: a spilled register's load inside the loop over pages would wait for all requests under way."""
import os
import re
import subprocess

import pytest

from paper_2603_05353_amd import build
from tests.test_direct_load_wait_states import hazards

pytestmark = pytest.mark.skipif(not os.path.exists(build.HIPCC), reason="no hipcc in this environment")


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    out = tmp_path_factory.mktemp("asm") / "pages.s"
    subprocess.run([build.HIPCC, *build.FLAGS, "--cuda-device-only", "-S", os.path.join(build.CSRC, "attention_pages_matrix.hip"), "-o", str(out)],
                   check=True, capture_output=True, timeout=600)
    return out.read_text()


def test_wait_states_before_direct_loads(assembly):
    found, loads = hazards(assembly)
    assert loads >= 300 and not found, (loads, len(found), found[:4])


def test_no_kernel_uses_scratch(assembly):
    sizes = re.findall(r"\.name:\s+(\S*attend_pages\S*)\n(?:.*\n)*?\s+\.private_segment_fixed_size: (\d+)", assembly)
    assert len(sizes) >= 14 and all(n == "0" for _, n in sizes), [s for s in sizes if s[1] != "0"]

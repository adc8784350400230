"""Registers of the 8-bit cache's kernels that are said to fit, as the compiler makes them for gfx950."""
import os
import re
import subprocess

import pytest

from paper_2512_16273_amd import build

FORMS = ["weigh_kernel<Bf16, 128, 4, 1>", "weigh_kernel<F16, 128, 2, 4>", "weigh_kernel<float, 128, 1, 4>"]


@pytest.mark.skipif(not os.path.exists("/opt/rocm/bin/hipcc"), reason="needs hipcc")
def test_rows_of_weigh_stay_in_registers(tmp_path):
    src, asm = tmp_path / "form.hip", tmp_path / "form.s"
    src.write_text('#include "weigh.h"\nnamespace tslt {\n' + "".join("template __global__ void %s(const WeighParams);\n" % f for f in FORMS) + "}\n")
    flags = [f for f in build.hipcc_command()[1:] if f not in ("-fPIC", "-shared") and not f.endswith((".hip", ".so")) and f != "-o"]
    subprocess.run([build.hipcc_command()[0], *flags, "--cuda-device-only", "-S", "-o", str(asm), str(src)], check=True, stderr=subprocess.DEVNULL)
    made = [k for k in asm.read_text().split(".agpr_count")[1:] if re.search(r"\.symbol:\s+\S*weigh_kernel", k)]
    assert len(made) == len(FORMS)
    for k in made:
        assert re.search(r"\.vgpr_spill_count:\s+(\d+)", k).group(1) == "0", re.search(r"\.symbol:\s+(\S+)", k).group(1)

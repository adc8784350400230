"""Kernels around attention and verification that are written to stay in registers, as the compiler makes them for gfx950."""
import os
import re
import subprocess

import pytest

from paper_2512_16273_amd import build

FORMS = {"adapt": ["adapt_up_kernel<F16, 4, false>", "adapt_up_kernel<Bf16, 1, true>", "adapt_up_kernel<float, 2, false>", "adapt_down_many_kernel<Bf16, 4>"],
         "rotate": ["rotate_kernel<Bf16, 128, 4>", "rotate_backward_kernel<Bf16, 128, 4>"],
         "logprob": ["logprob_kernel<Bf16, 4>", "logprob_kernel<F16, 1>", "logprob_backward_kernel<Bf16>"]}
PARAMS = {"logprob_backward": "LogprobBackwardParams", "logprob": "LogprobParams", "rotate": "RotateParams", "adapt": "AdaptParams"}


@pytest.mark.skipif(not os.path.exists("/opt/rocm/bin/hipcc"), reason="needs hipcc")
@pytest.mark.parametrize("header", FORMS)
def test_nothing_is_spilled(header, tmp_path):
    src, asm = tmp_path / "form.hip", tmp_path / "form.s"
    forms = "".join("template __global__ void %s(const %s);\n" % (f, next(p for k, p in PARAMS.items() if f.startswith(k))) for f in FORMS[header])
    src.write_text('#include "%s.h"\nnamespace tslt {\n%s}\n' % (header, forms))
    flags = [f for f in build.hipcc_command()[1:] if f not in ("-fPIC", "-shared") and not f.endswith((".hip", ".so")) and f != "-o"]
    subprocess.run([build.hipcc_command()[0], *flags, "--cuda-device-only", "-S", "-o", str(asm), str(src)], check=True, stderr=subprocess.DEVNULL)
    made = [k for k in asm.read_text().split(".agpr_count")[1:] if re.search(r"\.symbol:\s+\S*(adapt|rotate|logprob)", k)]
    assert len(made) == len(FORMS[header])
    for k in made:
        name = re.search(r"\.symbol:\s+(\S+)", k).group(1)
        assert re.search(r"\.vgpr_spill_count:\s+(\d+)", k).group(1) == "0", name
        assert re.search(r"\.private_segment_fixed_size:\s+(\d+)", k).group(1) == "0", name

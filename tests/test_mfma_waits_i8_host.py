"""Wait states around the matrix instructions that gemm_i8_ring_kernel and gemm_i8_tail_kernel have in assembly (see test_mfma_waits_host, whose walk through
the compiled code this is): v_mfma_i32_16x16x64_i8 reads and writes its registers as v_mfma_f32_16x16x32_bf16 does."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2405_13053_amd import build
from tests import test_mfma_waits_host as waits


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
def test_every_int8_ring_kernel_keeps_the_wait_states(tmp_path):
    asm = tmp_path / "gemm_i8.s"
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-fPIC", "-shared")]
    src = os.path.join(build.HERE, "csrc", "gemm_i8.hip")
    subprocess.run(["hipcc", *flags, "--cuda-device-only", "-S", "-o", str(asm), src], check=True,
                   stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
    text = asm.read_text()
    kernels = set(re.findall(r"^(_Z\S*gemm_i8_(?:ring|tail)_kernel\S*):", text, re.M))
    assert len(kernels) >= 30
    text = text.replace("v_mfma_i32_16x16x64_i8", waits.MFMA)
    code = [(fn, op) for fn, op, _ in waits._parse(text)[0] if op == waits.MFMA]
    assert kernels <= {fn for fn, _ in code}
    # the other kernels use the builtin, for which the compiler sees to the wait states
    assert not [v for v in waits._violations(text) if v[0] in kernels]
    assert ".private_segment_fixed_size: 0" in text and not re.search(r"\.private_segment_fixed_size: [1-9]", text)   # no spills

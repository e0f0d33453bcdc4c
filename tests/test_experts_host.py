"""Wait states behind the matrix instructions of the experts' kernels and of the 4-bit products that use the builtins.  The compiler sees to them,
but where a branch stands between an instruction and a read of its result it has left some out (ROCm 7.2: an accumulator moved right behind the branch, its
last element wrong now and then), so the compiled code is walked along every path (see test_mfma_waits_host): 8 states is what the compiler
itself puts between v_mfma_f32_16x16x32_bf16 and a read in straight code."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2405_13053_amd import build
from tests import test_mfma_waits_host as waits


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
@pytest.mark.parametrize("source,kernels", [("experts", r"experts_(?:few_up|few_down|many)_kernel"), ("gemm_mx4", r"gemm_mx4_(?:wave|one|row)_kernel"),
                                            ("gemm_mx4_back", r"gemm_mx4_back_kernel")])
def test_results_of_builtins_are_waited_for_on_every_path(source, kernels, tmp_path, monkeypatch):
    asm = tmp_path / "code.s"
    flags = [f for f in build.HIPCC_FLAGS if f not in ("-fPIC", "-shared")]
    subprocess.run(["hipcc", *flags, "--cuda-device-only", "-S", "-o", str(asm), os.path.join(build.HERE, "csrc", source + ".hip")], check=True,
                   stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
    text = asm.read_text()
    names = set(re.findall(r"^(_Z\S*(?:%s)\S*):" % kernels, text, re.M))
    assert len(names) >= (5 if source == "gemm_mx4_back" else 10)
    text = text.replace("v_mfma_scale_f32_16x16x128_f8f6f4", waits.MFMA)
    assert names <= {fn for fn, op, _ in waits._parse(text)[0] if op == waits.MFMA}
    monkeypatch.setattr(waits, "AFTER", 8)
    assert not [v for v in waits._violations(text) if v[0] in names and v[1] == "result"]
    assert not re.search(r"\.private_segment_fixed_size: [1-9]", text)   # no spills

"""Compile-time checks of the packed-row kernels (CPU, needs hipcc): no scratch memory, registers for two waves a SIMD (one
in fp32, whose stages fill the LDS), no vector instruction that reads an MFMA result too early, no product that takes another's result as an operand."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2607_12422_amd import build as b
from test_mfma_hazards import early_reads
from test_paged_resources import results_as_operands


@pytest.mark.slow
@pytest.mark.parametrize("src,mfma", [("pbd_rows.hip", 300), ("pbd_plan.hip", 0), ("pbd_tree.hip", 0)])
def test_kernels_use_no_scratch_and_wait_for_mfma(src, mfma, tmp_path):
    cc = b.hipcc()
    if not shutil.which(cc) and not os.path.exists(cc):
        pytest.skip("hipcc not available")
    out = tmp_path / (src + ".s")
    r = subprocess.run([cc, *b.FLAGS, "--cuda-device-only", "-S", os.path.join(b.CSRC, src), "-o", str(out),
                        "-Rpass-analysis=kernel-resource-usage"],
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout[-2000:]
    scratch = [int(x) for x in re.findall(r"ScratchSize \[bytes/lane\]: (\d+)", r.stdout)]
    vgprs = [int(x) for x in re.findall(r" VGPRs: (\d+)", r.stdout)]
    agprs = [int(x) for x in re.findall(r" AGPRs: (\d+)", r.stdout)]
    assert scratch and max(scratch) == 0, scratch
    names = re.findall(r"Function Name: (\S+)", r.stdout)
    assert len(names) == len(vgprs)
    for name, v, a in zip(names, vgprs, agprs):
        assert v + a <= (512 if "k_rows_attnIf" in name else 256), (name, v, a)
    asm = out.read_text()
    assert asm.count("v_mfma") >= mfma
    assert not early_reads(asm)[:10]
    assert not results_as_operands(asm)[:10]
    assert not re.search(r"v_pk_(add|mul|fma)_f32", asm)

"""Compile-time checks of the paged-cache and log-probability kernels (CPU, needs
hipcc): no scratch memory, registers for two waves a SIMD at least, and no vector
instruction that reads an MFMA result too early (see test_mfma_hazards)."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2607_12422_amd import build as b
from test_mfma_hazards import early_reads


@pytest.mark.slow
@pytest.mark.parametrize("src,mfma", [("pbd_paged.hip", 100), ("pbd_evict.hip", 0), ("pbd_logprobs.hip", 0)])
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
    assert max(v + a for v, a in zip(vgprs, agprs)) <= 256
    asm = out.read_text()
    assert asm.count("v_mfma") >= mfma
    assert not early_reads(asm)[:10]
    assert not re.search(r"v_pk_(add|mul|fma)_f32", asm)

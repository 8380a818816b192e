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
from test_mfma_hazards import _regs


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


def results_as_operands(asm):
    """Matrix products whose A or B operand was last written by another one, within a block.  Theirs come from loads
    and vector instructions; the compiler once put a result over the rest of a loaded V tile that the next product read."""
    found, owner = [], {}
    for i, line in enumerate(asm.splitlines()):
        t = line.split(";")[0].strip()
        if not t or (t.startswith(".") and not t.endswith(":")):
            continue
        if t.endswith(":"):
            owner = {}
            continue
        parts = t.split(None, 1)
        ops = [o.strip() for o in re.split(r",(?![^\[]*\])", parts[1])] if len(parts) > 1 else []
        if parts[0].startswith("v_mfma"):
            found += [(i + 1, t) for o in ops[1:3] if any(r in owner for r in _regs(o))]
            owner.update({r: i for r in _regs(ops[0])})
        else:
            for o in ops[:2] if "swap" in parts[0] else ops[:1]:
                for r in _regs(o):
                    owner.pop(r, None)
    return found


def test_results_as_operands_are_found():
    load = "\tglobal_load_dwordx4 v[18:21], v54, s[12:13] nt\n"
    good = load + "\tv_mfma_f32_16x16x4_f32 v[4:7], v18, v50, v[4:7]\n\tv_mfma_f32_16x16x4_f32 v[4:7], v19, v51, v[4:7]\n"
    bad = load + "\tv_mfma_f32_16x16x4_f32 v[18:21], v18, v50, v[4:7]\n\tv_mfma_f32_16x16x4_f32 v[4:7], v19, v51, v[18:21]\n"
    assert not results_as_operands(good)
    assert [i for i, _ in results_as_operands(bad)] == [3]
    assert not results_as_operands(bad.replace("\n\tv_mfma_f32_16x16x4_f32 v[4:7]", "\n\tv_mov_b32_e32 v19, v3\n\tv_mfma_f32_16x16x4_f32 v[4:7]"))


@pytest.mark.slow
@pytest.mark.parametrize("src", ["pbd_paged.hip", "pbd_attn.hip"])
def test_no_product_takes_a_result_as_operand(src, tmp_path):
    cc = b.hipcc()
    if not shutil.which(cc) and not os.path.exists(cc):
        pytest.skip("hipcc not available")
    out = tmp_path / (src + ".s")
    r = subprocess.run([cc, *b.FLAGS, "--cuda-device-only", "-S", os.path.join(b.CSRC, src), "-o", str(out)],
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout[-2000:]
    asm = out.read_text()
    assert "v_mfma" in asm and not results_as_operands(asm)[:10]

"""Compiler output of attention over shared pages: no MFMA under an EXEC mask, nothing kept in scratch memory, no wait for the
pages in flight where a block table is looked up."""
import os
import re
import subprocess

import pytest

from test_isa_guards import HIPCC, SRC, masked_mfma


@pytest.fixture(scope="module")
def asm(tmp_path_factory):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc not found")
    out = tmp_path_factory.mktemp("isa") / "kernels_shared.s"
    src = os.path.join(os.path.dirname(SRC), "kernels_shared.hip")
    cmd = [HIPCC, "--offload-arch=gfx950", "-O3", "-std=c++17", "-fno-gpu-rdc", "-Xclang", "-target-feature", "-Xclang",
           "-packed-fp32-ops", "--cuda-device-only", "-S", src, "-o", str(out)]
    res = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert res.returncode == 0, res.stdout[-2000:]
    return out.read_text()


def test_no_mfma_under_an_exec_mask(asm):
    assert asm.count("v_mfma_f32_16x16x32_bf16") > 500
    bad = masked_mfma(asm)
    assert not bad, f"MFMA under an EXEC mask without a branch in: {bad}"


def test_registers_without_spills(asm):
    sizes = re.findall(r"\.private_segment_fixed_size: (\d+)", asm)
    assert len(sizes) >= 9 and set(sizes) == {"0"}, sizes


def test_block_tables_come_through_the_scalar_cache(asm):
    """A block table entry read by a vector load would be waited for together with the page loads behind which it was requested."""
    kernels = re.findall(r"^(_Z\S*shared_attn_kernel\S*):(.*?)^\s*s_endpgm\s*$\n(?=\s*\.section)", asm, re.M | re.S)
    assert len(kernels) == 4
    for name, body in kernels:
        steps = body[body.index("v_mfma"):body.rindex("v_mfma")]
        assert "s_load_dword " in steps, name
        # single words from memory in front of the pages only (a row's index and position), not between the products
        words = [m.start() for m in re.finditer(r"global_load_dword v", steps)]
        assert len(words) <= 2, (name, len(words))

"""The attention backward's registers and LDS as they are reserved: what its
comments say of the workgroups that share a CU."""
import os
import re
import subprocess

import pytest

from paper_2512_22737_amd import build as B

SRC = "attn_backward.hip"
# of a SIMD's wave (in eights), of a CU
REGISTERS, LDS = 512, 160 * 1024


@pytest.fixture(scope="module")
def reserved(tmp_path_factory):
    """{kernel<D>: (registers, bytes of LDS)}"""
    out = str(tmp_path_factory.mktemp("asm") / "k.s")
    try:
        cc = B.hipcc()
    except RuntimeError:
        pytest.skip("no hipcc")
    subprocess.run([cc, *B.HIPCC_FLAGS, *B.FILE_FLAGS[SRC], "-I", B.INCLUDE,
                    "-I", B.CSRC, "-S", "--cuda-device-only",
                    os.path.join(B.CSRC, SRC), "-o", out], check=True,
                   capture_output=True, timeout=600)
    found = {}
    for m in re.finditer(r"\.amdhsa_kernel \S*?(dq|dkv)_kernelILi(\d+)E(.*?)"
                         r"\.end_amdhsa_kernel", open(out).read(), re.S):
        value = lambda key: int(re.search(
            rf"\.amdhsa_{key} (\d+)", m.group(3)).group(1))
        found[f"{m.group(1)}<{m.group(2)}>"] = (
            value("next_free_vgpr"), value("group_segment_fixed_size"))
    assert len(found) == 4, list(found)
    return found


@pytest.mark.parametrize("kernel,workgroups", [
    ("dq<64>", 3), ("dq<128>", 2), ("dkv<64>", 1), ("dkv<128>", 1)])
def test_workgroups_of_a_cu(reserved, kernel, workgroups):
    """Workgroups of four waves, one on each SIMD."""
    registers, lds = reserved[kernel]
    assert min(REGISTERS // -(-registers // 8 * 8), LDS // lds) == workgroups

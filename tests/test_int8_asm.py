"""Static checks on the tile kernels of the 8-bit product, like those on the bf16 ones (test_kernel_asm.py): inline matrix
steps, whose hazards the compiler does not see, with accumulators it must not move."""
import re
import shutil
import subprocess
from pathlib import Path

import pytest

from test_kernel_asm import CSRC, ROOT, _assert_no_valu_write_in_front_of_its_mfma, _kernels


@pytest.fixture(scope="module")
def int8_asm(tmp_path_factory):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not Path(hipcc).exists():
        pytest.skip("hipcc not found")
    out = tmp_path_factory.mktemp("asm") / "osdp_int8.s"
    cmd = [hipcc, "-O3", "-std=c++17", "--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           f"-I{ROOT / 'include'}", f"-I{CSRC}", "-S", "--cuda-device-only", str(CSRC / "osdp_int8.hip"), "-o", str(out)]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    return out.read_text().split("\n")


def test_tile_kernels_use_no_scratch_and_respect_the_mfma_hazards(int8_asm):
    kernels = _kernels(int8_asm, "i8_w4_kernel")
    assert len(kernels) >= 4, "the tile kernels were not found in the assembly"
    for name, ins in kernels.items():
        mb, nb = map(int, re.search(r"i8_w4_kernelILi(\d+)ELi(\d+)E", name).groups())
        mfma = [i for i, t in enumerate(ins) if t.startswith("v_mfma")]
        # one K block of 2 * mb * nb, as many to clear the accumulators, and again between tiles where a workgroup has several
        assert len(mfma) in (3 * mb * nb, 4 * mb * nb), f"{name}: {len(mfma)} MFMAs"
        assert all("i32_16x16x64_i8" in ins[i] for i in mfma)
        assert not [t for t in ins if t.startswith("scratch_")], f"{name}: scratch traffic"
        for i in mfma:
            near = ins[max(0, i - 3):i]
            assert not [t for t in near if t.startswith(("v_accvgpr_write", "v_accvgpr_mov"))], \
                f"{name}: an accumulator register is written right in front of an inline MFMA"
        _assert_no_valu_write_in_front_of_its_mfma(name, ins, mfma)

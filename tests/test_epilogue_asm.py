"""Static checks on the forward kernels with an epilogue, like those on the ones without (test_kernel_asm.py): the epilogue, written out
for each activation, stands beside inline matrix steps whose hazards the compiler does not see, and must neither take registers of
the K loop nor move accumulators."""
import re
import shutil
import subprocess
from pathlib import Path

import pytest

from test_kernel_asm import CSRC, ROOT, _assert_no_valu_write_in_front_of_its_mfma, _kernels


@pytest.fixture(scope="module")
def epilogue_asm(tmp_path_factory):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not Path(hipcc).exists():
        pytest.skip("hipcc not found")
    out = tmp_path_factory.mktemp("asm") / "osdp_epilogue.s"
    cmd = [hipcc, "-O3", "-std=c++17", "--offload-arch=gfx950", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
           f"-I{ROOT / 'include'}", f"-I{CSRC}", "-S", "--cuda-device-only", str(CSRC / "osdp_epilogue.hip"), "-o", str(out)]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    return out.read_text().split("\n")


@pytest.mark.parametrize("kernel,least,blocks", [("gemm_w4_kernel", 4, (2,)), ("gemm_w4p_kernel", 2, (2, 4)), ("gemm_w4_small_kernel", 4, (2,)),
                                                 ("gemm_w4p_small_kernel", 2, (2, 4)), ("gemm_w4_128_kernel", 4, (2,))])
def test_the_epilogue_leaves_the_k_loop_alone(epilogue_asm, kernel, least, blocks):
    kernels = _kernels(epilogue_asm, kernel)
    assert len(kernels) >= least, "the instantiations were not found in the assembly"
    for name, ins in kernels.items():
        mb, nb = (4, 4) if "128" in kernel else (8, 8)
        if "small" in kernel:
            mb, nb = map(int, re.search(kernel + r"ILi(\d+)ELi(\d+)E", name).groups())
        mfma = [i for i, t in enumerate(ins) if t.startswith("v_mfma")]
        assert len(mfma) in [mb * nb * b for b in blocks], f"{name}: {len(mfma)} MFMAs (a loop body was duplicated?)"
        assert not [t for t in ins if t.startswith("scratch_")], f"{name}: scratch traffic"
        # the accumulators are read where an activation's code takes them, and nowhere else
        assert len([t for t in ins if t.startswith("v_accvgpr_read")]) == 5 * 4 * mb * nb, f"{name}: accumulators moved"
        for i in mfma:
            assert not [t for t in ins[max(0, i - 3):i] if t.startswith(("v_accvgpr_write", "v_accvgpr_mov"))], \
                f"{name}: an accumulator register is written right in front of an inline MFMA"
        _assert_no_valu_write_in_front_of_its_mfma(name, ins, mfma)


def test_the_eight_wave_kernels_keep_scratch_out_of_the_k_loop(epilogue_asm):
    """Tiles of which two fit a CU have 128 registers a lane: what the epilogue lacks of them it must not take from the K loop."""
    kernels = _kernels(epilogue_asm, "gemm_dma_kernel")
    assert len(kernels) >= 8, "the instantiations were not found in the assembly"
    for name, ins in kernels.items():
        mfma = [i for i, t in enumerate(ins) if t.startswith("v_mfma")]
        inside = [t for t in ins[mfma[0]:mfma[-1] + 1] if t.startswith("scratch_")]
        assert not inside, f"{name}: scratch traffic inside the K loop"

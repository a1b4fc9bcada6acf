"""The copies straight to LDS of expert_kernels.hpp as compiled beside other instructions that use m0, which holds a
copy's address in LDS (read from the assembly: the operators' own kernels have no such instructions)."""
import os
import re
import subprocess

import pytest

from paper_1910_02054_amd import build as b

SOURCE = """
#include "expert_kernels.hpp"
extern "C" __global__ void beside(const float* p, const float* q, float* out) {
    __shared__ float mine[256], other[64];
    const int t = threadIdx.x;
    auto copy = [&](int i) {
        __builtin_amdgcn_global_load_lds((__attribute__((address_space(1))) const void*)(q + i + t), ZO_LDS(void, other),
                                         4, 0, 0);
    };
    copy(0);
    zo::%s(p + 4 * t, zo::lds_address(mine));
    copy(64);
    zo::wait_stage<0>();
    out[t] = mine[t] + other[t];
}
"""


@pytest.mark.parametrize("copy", ("copy_to_lds", "copy_word_to_lds"))
def test_m0_is_set_again_behind_a_copy(tmp_path, copy):
    hip, asm = tmp_path / "beside.hip", tmp_path / "beside.s"
    hip.write_text(SOURCE % copy)
    flags = [f for f in b.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run([b.hipcc(), *flags, "-S", "--cuda-device-only", str(hip), "-o", str(asm)], check=True,
                   stdout=subprocess.DEVNULL, stderr=subprocess.DEVNULL)
    steps = re.findall(r"^\ts_\w+ (m0), |^\tglobal_load_lds_(\w+) ", asm.read_text(), re.M)
    names = ["set" if m0 else "copy" for m0, _ in steps]
    assert names.count("copy") == 3
    # every copy follows a setting of its own
    assert all(names[i - 1] == "set" for i, n in enumerate(names) if n == "copy"), steps


def test_the_operators_build_without_warnings_of_it(tmp_path):
    """The warning is dealt with where it arises."""
    hip = tmp_path / "empty.hip"
    hip.write_text(SOURCE % "copy_to_lds")
    flags = [f for f in b.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    out = subprocess.run([b.hipcc(), *flags, "-c", "--cuda-device-only", str(hip), "-o", os.devnull], check=True,
                         capture_output=True, text=True)
    assert "clobber" not in out.stderr

"""The compiler of ROCm 7.2 writes half of an fp64 constant that a wave keeps in scalar registers; the build goes through assembly
text, where such an instruction is refused (no GPU needed: these compile for gfx950 only)."""
import re
import subprocess

import pytest

from paper_1802_09113_amd import build

SOURCE = """#include <hip/hip_runtime.h>
__device__ double at_lane(double x, int lane)
{
    const long long b = __double_as_longlong(x);
    const unsigned lo = __builtin_amdgcn_readlane((int)b, lane);
    const int hi = __builtin_amdgcn_readlane((int)(b >> 32), lane);
    return __longlong_as_double(((long long)hi << 32) | (long long)lo);
}
__global__ void kth(const double *z, double *out, int n, int k)
{
    double v = -CONSTANT, least = -CONSTANT;
    for (int i = 0; i < n; ++i) {
        const double x = z[i * 64 + threadIdx.x];
        if (__ballot(x > least)) {
            v = x > v ? x : v;
            least = at_lane(v, k - 1);
        }
    }
    out[threadIdx.x] = v;
    if (threadIdx.x == 0) out[64] = least;
}
"""


@pytest.mark.parametrize("constant,halved", [("__builtin_inf()", True), ("1.0", False)])
def test_half_a_constant_is_not_built(tmp_path, monkeypatch, capfd, constant, halved):
    src = tmp_path / "kth.hip"
    src.write_text(SOURCE.replace("CONSTANT", constant))
    text = tmp_path / "kth.s"
    subprocess.check_call(["hipcc", "-S", "--cuda-device-only", *[f for f in build.FLAGS if f not in ("-shared", "-fPIC")],
                           "-o", str(text), str(src)], stderr=subprocess.DEVNULL)
    seen = re.search(r"_b64\w* .*, 0x[0-9a-f]{9,}", text.read_text()) is not None
    assert halved or not seen
    monkeypatch.setattr(build, "SRCS", [str(src)])
    monkeypatch.setattr(build, "LIB", str(tmp_path / "lib.so"))
    monkeypatch.setattr(build, "RESOURCES", str(tmp_path / "resources.json"))
    if seen:                                             # a compiler that does better builds it
        with pytest.raises(subprocess.CalledProcessError):
            build.build()
        assert "invalid operand" in capfd.readouterr().err
    else:
        build.build()
        assert (tmp_path / "lib.so").exists() and (tmp_path / "kth.o").exists()

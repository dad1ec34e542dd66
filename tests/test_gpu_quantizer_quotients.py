"""The quantizer's scale and reciprocal (csrc/wfq_rows.h) against correctly rounded quotients, for every fp32 number."""
import ctypes
import os
import struct
import subprocess

import pytest

from paper_2412_19867_b200 import build

pytestmark = pytest.mark.gpu

SOURCE = r"""
#include "wfq_rows.h"
// out: numbers whose scale, whose reciprocal differs, the first such bit patterns, numbers that have a quotient
__global__ void compare(unsigned first, unsigned n, unsigned long long *out)
{
    unsigned long long with = 0;
    for (unsigned i = blockIdx.x * blockDim.x + threadIdx.x; i < n; i += gridDim.x * blockDim.x) {
        const float amax = __uint_as_float(first + i);
        float scale, inv;
        wfq::quantizer_scale(amax, scale, inv);
        float s = 0.f, r = 0.f;
        with += amax >= 1e-30f && first + i < 0x7f800000u;
        if (amax >= 1e-30f) { s = __fdiv_rn(amax, 127.f); r = __fdiv_rn(127.f, amax); }
        if (first + i >= 0x7f800000u) { s = __uint_as_float(0x7fc00000u); r = 0.f; }
        const bool s_differs = s != s ? scale == scale : __float_as_uint(s) != __float_as_uint(scale);
        if (s_differs) { atomicAdd(out, 1ull); atomicMin(out + 2, (unsigned long long)(first + i)); }
        if (__float_as_uint(r) != __float_as_uint(inv)) { atomicAdd(out + 1, 1ull); atomicMin(out + 3, (unsigned long long)(first + i)); }
    }
    atomicAdd(out + 4, with);
}
extern "C" int run(unsigned long long *host)
{
    unsigned long long *d = nullptr, start[5] = {0, 0, ~0ull, ~0ull, 0};
    if (cudaMalloc(&d, sizeof(start)) != cudaSuccess) return 1;
    int bad = cudaMemcpy(d, start, sizeof(start), cudaMemcpyHostToDevice) != cudaSuccess;
    for (unsigned part = 0; part < 8 && !bad; ++part) {               // 2^31 patterns: every number that is not negative, NaN
        compare<<<1184, 256>>>(part << 28, 1u << 28, d);
        bad = cudaGetLastError() != cudaSuccess;
    }
    if (!bad) bad = cudaMemcpy(host, d, sizeof(start), cudaMemcpyDeviceToHost) != cudaSuccess;
    cudaFree(d);
    return bad;
}
"""


def test_every_number(tmp_path):
    (tmp_path / "q.cu").write_text(SOURCE)
    subprocess.run([build._nvcc(), "-gencode", "arch=compute_100a,code=sm_100a", "-O3", "-std=c++17", "-Xcompiler", "-fPIC", "-shared",
                    "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC, "-o", str(tmp_path / "q.so"), str(tmp_path / "q.cu")],
                   check=True, timeout=300)
    out = (ctypes.c_ulonglong * 5)()
    assert ctypes.CDLL(str(tmp_path / "q.so")).run(out) == 0
    scales, inverses, first_scale, first_inverse, compared = out
    assert compared == 0x7f800000 - struct.unpack("<I", struct.pack("<f", 1e-30))[0]
    assert (scales, inverses) == (0, 0), (scales, inverses, hex(first_scale), hex(first_inverse))

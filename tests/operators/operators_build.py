"""The CPU build of tests/lanes with the operators' units in it: the same fibres and checked memory, and the matrix instruction of
the four-bit kernels in plain C++."""
import os
import re
import sys

HERE = os.path.dirname(os.path.abspath(__file__))
sys.path.insert(0, os.path.join(os.path.dirname(HERE), "lanes"))
import cpu_build as lanes_build  # noqa: E402

UNITS = ["qmoe_norm.hip", "qmoe_route.hip", "qmoe_int4.hip", "qmoe_int4_mm_plain.hip", "qmoe_int4_mm_zeros.hip", "qmoe_int4_mm_gated.hip",
         "qmoe_int4_mm_gated_zeros.hip", "qmoe_int4_host.cpp"]
MORE = r"""#pragma once
#include <hip/hip_runtime.h>
#define __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, ...) lanes_mfma(a, b, c)
#define __expf(x) expf(x)
#define __builtin_amdgcn_ds_bpermute(from, v) lanes_bpermute(from, v)
inline int lanes_bpermute(int from, int v) { return (int)(uint32_t)lanes::wave_values((uint32_t)v)[(from >> 2) & 63]; }
template <class AB, class C> inline C lanes_mfma(AB a, AB b, C c)
{
    uint64_t mine[4], all[4][64];
    memcpy(mine, &a, 16);
    memcpy(mine + 2, &b, 16);
    for (int i = 0; i < 4; i++) memcpy(all[i], lanes::wave_values(mine[i]), sizeof all[i]);
    auto value = [&](int of, int lane, int k) {
        return __uint_as_float((uint32_t)(uint16_t)(all[2 * of + k / 4][lane] >> (16 * (k % 4))) << 16);
    };
    const int n = lanes::lane() & 15, m0 = 4 * (lanes::lane() >> 4);
    for (int i = 0; i < 4; i++)
        for (int quarter = 0; quarter < 4; quarter++)
            for (int k = 0; k < 8; k++) c[i] += value(0, m0 + i + 16 * quarter, k) * value(1, n + 16 * quarter, k);
    return c;
}
"""
ROUND = r"""#include <cstdint>
#include <cstring>
// what the compiler calls to round fp32 to bf16 where the processor cannot
extern "C" __bf16 __truncsfbf2(float f)
{
    uint32_t u;
    memcpy(&u, &f, 4);
    uint16_t r = (uint16_t)((u + 0x7FFFu + ((u >> 16) & 1u)) >> 16);
    if (f != f) r = (uint16_t)(u >> 16 | 0x40u);
    __bf16 b;
    memcpy(&b, &r, 2);
    return b;
}
"""


def build(into: str) -> str:
    src = os.path.join(into, "src")
    os.makedirs(src, exist_ok=True)
    with open(os.path.join(src, "operators_cpu.h"), "w") as f:
        f.write(MORE)
    plain, units = lanes_build.converted, lanes_build.UNITS
    lanes_build.converted = lambda text: '#include "operators_cpu.h"\n' + re.sub(r'asm( volatile)?\("" : "\+[sv]"\(\w+\)\);', "", plain(text))
    lanes_build.UNITS = units + UNITS
    more, lanes_build.NO_MATRIX_CORES = lanes_build.NO_MATRIX_CORES, lanes_build.NO_MATRIX_CORES + ROUND
    try:
        return lanes_build.build(into)
    finally:
        lanes_build.converted, lanes_build.UNITS, lanes_build.NO_MATRIX_CORES = plain, units, more

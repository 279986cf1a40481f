// Four-bit weights: what their kernels share.  Not part of the C ABI.
#pragma once

#include "qmoe_ops.h"

namespace qmoe {

constexpr int kInt4BlockCols = 128;  // columns of a 64-byte block of a row

struct Int4Args {
    const qmoe_int4_matrix *mats;  // device array by expert, or nullptr: `single`
    const uint8_t *weights;        // single
    const uint16_t *scale;
    const uint8_t *zero;
    const Item *items;             // device list, or nullptr: tiles of `batch` tokens of the single matrix
    const int *n_items_dev;
    int max_items, n_experts, batch;
    const int *perm;               // slot -> token; x rows and results by token, unless ...
    int x_by_slot, out_by_slot;
    const uint16_t *x;
    size_t ld_x, ld_out;
    void *out;
    int out_f32;
    const float *gate;             // by token, or nullptr
    int rows;                      // results a token: rows of the matrix, half of them if gated
    int cols, blocks, groups;
    int per_block, blocks_per_group;  // groups a block (1, 2, 4), blocks a group (1 or more)
    int activation;
    int split;                     // k_int4_split: wavefronts that share a tile of rows along the columns
};

// One matrix as a wavefront reads it.
struct Int4Matrix {
    const uint8_t *weights;
    const uint16_t *scale;
    const uint8_t *zero;
};
__device__ __forceinline__ Int4Matrix int4_matrix(const Int4Args &a, int expert)
{
    if (!a.mats) return {a.weights, a.scale, a.zero};
    const qmoe_int4_matrix &m = a.mats[expert];
    return {m.weights, m.scale_f16, m.zero};
}

// Eight weights (a word) as bf16 16 + q, in the order of their columns: bits 3..6 of a bf16 between 16 and 32 are its
// units, so a shift and an and-or do for two, exactly.  The 16 goes with the zero point, against the sum of x.
// The two constants are hidden from the compiler, which knows no and-or with literals (and takes three instructions).
__device__ __forceinline__ bf16x8 int4_plus16(uint32_t w)
{
    uint32_t m = 0x00780078u, b = 0x41804180u;
    asm("" : "+s"(m));
    asm("" : "+v"(b));
    const u32x4 v = {((w << 3) & m) | b, ((w >> 1) & m) | b, ((w >> 5) & m) | b, ((w >> 9) & m) | b};
    return __builtin_bit_cast(bf16x8, v);
}

// Eight activations of a token from column c on, 0 from column cols on.
__device__ __forceinline__ u32x4 int4_x(const uint16_t *row, int c, int cols)
{
    if (c + 8 <= cols) return *reinterpret_cast<const u32x4_by2 *>(row + c);
    u32x4 v = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; i++)
        if (c + i < cols) v[i / 2] |= (uint32_t)row[c + i] << (16 * (i % 2));
    return v;
}

// The sum of x over a group, in the last of the lanes (of 16 that hold the 128 columns of a token's block) whose columns the group is.
template <int PER_BLOCK>
__device__ __forceinline__ float int4_group_sum(u32x4 x)
{
    const bf16x2 one = __builtin_bit_cast(bf16x2, 0x3F803F80u);
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; i++) s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, (uint32_t)x[i]), one, s, false);
    s += dpp_f<0x111, 0xf>(0.0f, s);
    s += dpp_f<0x112, 0xf>(0.0f, s);
    if constexpr (PER_BLOCK <= 2) s += dpp_f<0x114, 0xf>(0.0f, s);
    if constexpr (PER_BLOCK == 1) s += dpp_f<0x118, 0xf>(0.0f, s);
    return s;
}

inline bool int4_is_gated(int activation) { return activation == QMOE_ACT_SILU_GATED || activation == QMOE_ACT_GELU_GATED; }

__device__ __forceinline__ float int4_gated(float g, float u, int activation)
{
    if (activation == QMOE_ACT_SILU_GATED) return g / (1.0f + expf(-g)) * u;
    return 0.5f * g * (1.0f + tanhf(0.7978845608028654f * fmaf(0.044715f * g * g, g, g))) * u;
}

__device__ __forceinline__ void int4_store(const Int4Args &a, size_t out_row, float gate, int r, float v)
{
    if (a.activation == QMOE_ACT_RELU) v = v > 0.0f || v != v ? v : 0.0f;
    v *= gate;
    const size_t at = out_row * a.ld_out + r;
    if (a.out_f32) static_cast<float *>(a.out)[at] = v;
    else static_cast<uint16_t *>(a.out)[at] = bf16_bits(v);
}

// qmoe_int4_mm_*.hip
qmoe_status launch_int4_mm_plain(const Int4Args &a, int cus, hipStream_t s);
qmoe_status launch_int4_mm_zeros(const Int4Args &a, int cus, hipStream_t s);
qmoe_status launch_int4_mm_gated(const Int4Args &a, int cus, hipStream_t s);
qmoe_status launch_int4_mm_gated_zeros(const Int4Args &a, int cus, hipStream_t s);

}  // namespace qmoe

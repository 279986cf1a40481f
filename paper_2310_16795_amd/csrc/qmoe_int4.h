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
    const Item *items;             // device list, or nullptr: tiles of `batch` tokens of the single matrix ...
    const int *direct;             // ... or, with this one, an item for each of max_items tokens: its expert, results 0 if that is none
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

// A value that is to be made here and not further down, where the compiler would like to make it beside others: sums that wait to be
// scaled hold registers.
__device__ __forceinline__ void int4_now(f32x4 &v) { asm volatile("" : "+v"(v)); }

// One matrix as a wavefront reads it.  Its pointers may come out of an array in memory, so they are given their address space by
// hand: through a generic pointer every load would also count as LDS traffic and be waited for together with it.
using gp_bytes = const __attribute__((address_space(1))) uint8_t *;
using gp_u16 = const __attribute__((address_space(1))) uint16_t *;
struct Int4Matrix {
    const uint8_t *weights;
    gp_u16 scale;
    gp_bytes zero;
};
__device__ __forceinline__ Int4Matrix int4_matrix(const Int4Args &a, int expert)
{
    if (!a.mats) return {a.weights, (gp_u16)a.scale, (gp_bytes)a.zero};
    const qmoe_int4_matrix &m = a.mats[expert];
    return {m.weights, (gp_u16)m.scale_f16, (gp_bytes)m.zero};
}
// N values of 2 or 1 bytes from memory, in N / 2 or N / 4 words
template <int BYTES> struct Int4Packed;
typedef uint16_t u16_by1 __attribute__((aligned(1)));
typedef uint32_t u32_by1 __attribute__((aligned(1)));
typedef uint32_t u32x2_by1 __attribute__((ext_vector_type(2), aligned(1)));
typedef uint32_t u32x4_by1 __attribute__((ext_vector_type(4), aligned(1)));
template <> struct Int4Packed<2> { using at = const __attribute__((address_space(1))) u16_by1 *; };
template <> struct Int4Packed<4> { using at = const __attribute__((address_space(1))) u32_by1 *; };
template <> struct Int4Packed<8> { using at = const __attribute__((address_space(1))) u32x2_by1 *; };
template <> struct Int4Packed<16> { using at = const __attribute__((address_space(1))) u32x4_by1 *; };
template <int BYTES, int WORDS, typename P>
__device__ __forceinline__ void int4_load_packed(uint32_t (&v)[WORDS], P from)
{
    if constexpr (BYTES == 1) {
        v[0] = *from;
    } else {
        const auto w = *(typename Int4Packed<BYTES>::at)from;
        if constexpr (BYTES <= 4) {
            v[0] = w;
        } else {
#pragma unroll
            for (int i = 0; i < WORDS; i++) v[i] = w[i];
        }
    }
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

// Eight activations of a token from column c on, 0 from column cols on.  whole: none is missing (the same for the wavefront).  The other
// path is rare, and is kept from asking for registers that the loop around it needs.
__device__ __forceinline__ u32x4 int4_x(const uint16_t *row, int c, int cols, bool whole)
{
    if (whole) return *reinterpret_cast<const u32x4_by2 *>(row + c);
    u32x4 v = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; i++) {
        if (c + i < cols) v[i / 2] |= (uint32_t)row[c + i] << (16 * (i % 2));
        asm volatile("" ::: "memory");
    }
    return v;
}

// The same in two parts, for loops that keep loads on their way (a branch with loads of its own would have them all waited for): eight
// values from column c on or from the row's last eight (cols >= 8) ...
__device__ __forceinline__ u32x4 int4_x_load(const uint16_t *row, int c, int cols)
{
    return *reinterpret_cast<const u32x4_by2 *>(row + min(c, cols - 8));
}
// ... and, where the row ends in them, those from c on moved to the front, zeros behind.
__device__ __forceinline__ u32x4 int4_x_end(u32x4 v, int c, int cols)
{
    const int over = max(0, min(c + 8 - cols, 8));
    if (over & 1) v = (u32x4){v[0] >> 16 | v[1] << 16, v[1] >> 16 | v[2] << 16, v[2] >> 16 | v[3] << 16, v[3] >> 16};
    if (over & 2) v = (u32x4){v[1], v[2], v[3], 0u};
    if (over & 4) v = (u32x4){v[2], v[3], 0u, 0u};
    if (over & 8) v = (u32x4){0u, 0u, 0u, 0u};
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

// (1 + tanh(z)) / 2 = 1 / (1 + exp(-2 z)): both are g / (1 + exp(-t)), and nothing cancels.
__device__ __forceinline__ float int4_gated(float g, float u, int activation)
{
    const float t = activation == QMOE_ACT_SILU_GATED ? g : 1.5957691216057308f * fmaf(0.044715f * g * g, g, g);
    return g / (1.0f + expf(-t)) * u;
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
qmoe_status launch_int4_mm_plain(const Int4Args &a, int grid, hipStream_t s);
qmoe_status launch_int4_mm_zeros(const Int4Args &a, int grid, hipStream_t s);
qmoe_status launch_int4_mm_gated(const Int4Args &a, int grid, hipStream_t s);
qmoe_status launch_int4_mm_gated_zeros(const Int4Args &a, int grid, hipStream_t s);

}  // namespace qmoe

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
    const int *direct;             // ... or, with this one, an item for each of max_items (up to 8) tokens: its expert, results 0 if that is none
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

// Eight weights (a word) as bf16 (q - z) / 16, in the order of their columns.  Exact, so that a weight of 0 takes nothing from its activation however large
// that is, and below 1, so that no product of a finite activation overflows; a group's scale brings the 16 back.
// Four bits under the exponent of 1024 are a binary16 number 1024 + q or, four bits higher up, 1024 + 16 q; a mixed-precision multiply-add takes either
// to (q - z) / 16 in fp32, whose upper half is the bf16: 17 instructions a word.  (16 + q as bf16, its excess taken off with the sum of x, was eight: the two
// large sums cancel, and one activation of 10^4 on a weight of 0 cost a group of ordinary ones 1e-3 of its sum.)
// The constants are hidden from the compiler, which knows no and-or with literals (and takes three instructions).
struct Int4Zero {
    float low, high;  // what the two places take off
};
__device__ __forceinline__ Int4Zero int4_zero(uint32_t z)
{
    const float s = 0.0625f * (float)z;
    return {-64.0f - s, -4.0f - s};
}
__device__ __forceinline__ bf16x8 int4_weights(uint32_t w, Int4Zero zero)
{
    typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
    uint32_t m = 0x000F000Fu, m16 = 0x00F000F0u, b = 0x64006400u;
    asm("" : "+s"(m));
    asm("" : "+s"(m16));
    asm("" : "+v"(b));
    const uint32_t w8 = w >> 8;
    const uint32_t halves[4] = {(w & m) | b, (w & m16) | b, (w8 & m) | b, (w8 & m16) | b};
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const f16x2 h = __builtin_bit_cast(f16x2, halves[i]);
        const float unit = i % 2 ? 0.00390625f : 0.0625f, off = i % 2 ? zero.high : zero.low;
        const float lo = fmaf((float)h[0], unit, off), hi = fmaf((float)h[1], unit, off);
        v[i] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
    }
    return __builtin_bit_cast(bf16x8, v);
}
__device__ __forceinline__ float int4_scale(uint16_t s) { return 16.0f * half_bits_to_float(s); }

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

// Shared by the operators around the ternary layer: residual stream and norm (qmoe_norm.hip), the router's choice
// (qmoe_route.hip), four-bit weights (qmoe_int4.hip, qmoe_int4_mm_*.hip).  Each unit holds its kernels and its C entry points.
// Not part of the C ABI.
#pragma once

#include "qmoe_dev.h"

namespace qmoe {

// ---- from qmoe_api.hip
qmoe_status gpu_info(DeviceInfo *out);
// Tokens grouped by expert in a layer workspace: one list of tiles, its length on the device; slot -> token, and the place of the hidden vectors by slot.
struct GroupedTokens {
    const Item *items;
    const int *n_items, *perm;
    uint16_t *hidden;
};
// Sizes and workspace, as the layer calls check them.
qmoe_status layer_workspace_ok(int n_tokens, int n_experts, int d_model, int d_ff, const void *workspace, size_t workspace_bytes);
// Enqueues the dispatch kernel on a workspace that is right: every expert's tokens in tiles of up to `tile`.  It also clears the rows
// (row_words 32-bit words each) of y whose token has no expert.
qmoe_status group_by_expert(const int32_t *expert_idx, int n_tokens, int n_experts, int d_model, int d_ff, int tile, void *workspace,
                            float *y, int row_words, hipStream_t s, GroupedTokens *out);

constexpr int kMaxJoined = 16;      // rows of a token that are joined, or copies of one: k and copies
constexpr int kMaxInt4Rows = 1 << 24;
constexpr int kMaxInt4Cols = 1 << 20;

// ---- device helpers

// Vectors read and written whole at any alignment that fits their elements (the hardware takes such addresses).
typedef uint32_t u32x4_by2 __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x4_by4 __attribute__((ext_vector_type(4), aligned(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi)  // to nearest even; NaN stays NaN
{
    const bf16x2 v = __builtin_convertvector((f32x2){lo, hi}, bf16x2);
    return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ uint16_t bf16_bits(float f) { return (uint16_t)bf16_pair(f, 0.0f); }

template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp_f(float old, float x)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(old), __float_as_int(x), CTRL, ROWS, 0xf, false));
}
// Sum over the wavefront, in every lane; always in the same order.
__device__ __forceinline__ float wave_sum(float x)
{
    x += dpp_f<0x121, 0xf>(0.0f, x);  // rotations within a row of 16
    x += dpp_f<0x122, 0xf>(0.0f, x);
    x += dpp_f<0x124, 0xf>(0.0f, x);
    x += dpp_f<0x128, 0xf>(0.0f, x);
    x += dpp_f<0x142, 0xa>(0.0f, x);  // a row's sum into the next, rows 1 and 3
    x += dpp_f<0x143, 0xc>(0.0f, x);  // ... rows 2 and 3
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}

}  // namespace qmoe

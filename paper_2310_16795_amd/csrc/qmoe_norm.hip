// qmoe_residual_norm: a block's output joins the residual stream, and the stream is normalised for the next call.
#include "qmoe_ops.h"

namespace qmoe {
namespace {

struct NormArgs {
    const void *h, *y;
    void *h_out;
    uint16_t *x;
    size_t ld_h, ld_y, ld_h_out, ld_x;
    const float *gate, *channel;
    qmoe_norm post, pre;
    int has_post, has_pre;
    float alpha, inv_d;
    int k, copies, n_tokens, d;
    int waves;  // wavefronts of a row
};

struct Eight {
    float v[8];
};

// Eight consecutive values of a row from column c on; columns from d on are 0.
template <int TYPE>
__device__ __forceinline__ Eight load8(const void *base, size_t at, int c, int d)
{
    Eight r;
    if (c + 8 <= d) {
        if constexpr (TYPE == QMOE_F32) {
            const f32x4_by4 *p = reinterpret_cast<const f32x4_by4 *>(static_cast<const float *>(base) + at + c);
            const f32x4 a = p[0], b = p[1];
#pragma unroll
            for (int i = 0; i < 4; i++) r.v[i] = a[i], r.v[4 + i] = b[i];
        } else {
            const u32x4 a = *reinterpret_cast<const u32x4_by2 *>(static_cast<const uint16_t *>(base) + at + c);
#pragma unroll
            for (int i = 0; i < 4; i++) {
                r.v[2 * i] = __uint_as_float(a[i] << 16);
                r.v[2 * i + 1] = __uint_as_float(a[i] & 0xFFFF0000u);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            r.v[i] = 0.0f;
            if (c + i < d)
                r.v[i] = TYPE == QMOE_F32 ? static_cast<const float *>(base)[at + c + i]
                                          : bf16_bits_to_float(static_cast<const uint16_t *>(base)[at + c + i]);
        }
    }
    return r;
}

template <int TYPE>
__device__ __forceinline__ void store8(void *base, size_t at, int c, int d, const Eight &r)
{
    if (c + 8 <= d) {
        if constexpr (TYPE == QMOE_F32) {
            f32x4_by4 *p = reinterpret_cast<f32x4_by4 *>(static_cast<float *>(base) + at + c);
            p[0] = (f32x4){r.v[0], r.v[1], r.v[2], r.v[3]};
            p[1] = (f32x4){r.v[4], r.v[5], r.v[6], r.v[7]};
        } else {
            *reinterpret_cast<u32x4_by2 *>(static_cast<uint16_t *>(base) + at + c) =
                (u32x4){bf16_pair(r.v[0], r.v[1]), bf16_pair(r.v[2], r.v[3]), bf16_pair(r.v[4], r.v[5]), bf16_pair(r.v[6], r.v[7])};
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (c + i < d) {
                if constexpr (TYPE == QMOE_F32) static_cast<float *>(base)[at + c + i] = r.v[i];
                else static_cast<uint16_t *>(base)[at + c + i] = bf16_bits(r.v[i]);
            }
    }
}

// A row is `waves` wavefronts' work: a lane holds PER times eight consecutive columns of it from the first load to the last
// store, so that every value crosses memory once.  Workgroups either give each wavefront a row of its own (waves = 1; no
// barrier) or are one row's.  The sums of a norm (of the values, then of the squares around the mean: no difference of
// two large sums) go through DPP and, with several wavefronts, LDS; their order depends on the sizes alone.
//
// Bound by memory: 2048 tokens of 2080 values (bf16 h, two fp32 rows a token, 68 MB) 14.6 us, 4.7 TB/s, what a large copy reaches; 8191 of 1024 (fp32 h
// written back, bf16 y, two layer norms, 101 MB) 25.5 us, 3.9 TB/s: a row's four sums come one after the other, and its loads and stores
// do not overlap them.  One token is the launch (3 us).  Rows of 1024 with a wavefront of two or four times as many values gained nothing.
template <int HT, int YT, int PER, bool ALONE>
__global__ __launch_bounds__(ALONE ? 256 : 1024) void k_residual_norm(const NormArgs a)
{
    __shared__ float sums[4][16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    constexpr bool alone = ALONE;
    const long long row = alone ? (long long)blockIdx.x * (blockDim.x >> 6) + wave : blockIdx.x;
    if (row >= a.n_tokens) return;  // (a workgroup of one row leaves as one)
    const int me = alone ? lane : (int)threadIdx.x, step = 64 * a.waves * 8;
    // the longest rows fill the registers: their quarters are not to be loaded ahead of each other (512 rows of 32768, all fp32, 56 us, 4.2 TB/s; spilled 97)
    auto apart = [] {
        if constexpr (PER == 4) __builtin_amdgcn_sched_barrier(0);
    };
    int at_sum = 0;
    auto row_sum = [&](float v) {
        v = wave_sum(v);
        if (!alone) {
            float *s = sums[at_sum++];
            if (lane == 0) s[wave] = v;
            __syncthreads();
            v = 0.0f;
            for (int w = 0; w < a.waves; w++) v += s[w];
        }
        return v;
    };
    auto norm = [&](Eight (&v)[PER], const qmoe_norm &n) {
        float mean = 0.0f;
        if (n.kind == QMOE_NORM_LAYER) {
            float s = 0.0f;
#pragma unroll
            for (int p = 0; p < PER; p++)
#pragma unroll
                for (int i = 0; i < 8; i++) s += v[p].v[i];  // (columns from d on hold 0)
            mean = row_sum(s) * a.inv_d;
        }
        float s = 0.0f;
#pragma unroll
        for (int p = 0; p < PER; p++)
#pragma unroll
            for (int i = 0; i < 8; i++) {
                v[p].v[i] -= mean;
                if (8 * me + p * step + i < a.d) s = fmaf(v[p].v[i], v[p].v[i], s);
            }
        const float r = 1.0f / sqrtf(row_sum(s) * a.inv_d + n.eps);
#pragma unroll
        for (int p = 0; p < PER; p++) {
            const int c = 8 * me + p * step;
#pragma unroll
            for (int i = 0; i < 8; i++) v[p].v[i] *= r;
            if (n.weight) {
                const Eight w = load8<QMOE_F32>(n.weight, 0, c, a.d);
#pragma unroll
                for (int i = 0; i < 8; i++) v[p].v[i] *= w.v[i];
            }
            if (n.bias) {
                const Eight w = load8<QMOE_F32>(n.bias, 0, c, a.d);
#pragma unroll
                for (int i = 0; i < 8; i++) v[p].v[i] += w.v[i];
            }
            apart();
        }
    };

    Eight h[PER];
#pragma unroll
    for (int p = 0; p < PER; p++) h[p] = load8<HT>(a.h, (size_t)row * a.ld_h, 8 * me + p * step, a.d), apart();
    if (a.y) {
        Eight b[PER];
#pragma unroll
        for (int p = 0; p < PER; p++)
#pragma unroll
            for (int i = 0; i < 8; i++) b[p].v[i] = 0.0f;
#pragma unroll 2
        for (int j = 0; j < a.k; j++) {
            const size_t r = (size_t)row * a.k + j;
            const float g = a.gate ? a.gate[r] : 1.0f;
#pragma unroll
            for (int p = 0; p < PER; p++) {
                const Eight y = load8<YT>(a.y, r * a.ld_y, 8 * me + p * step, a.d);
#pragma unroll
                for (int i = 0; i < 8; i++) b[p].v[i] = fmaf(g, y.v[i], b[p].v[i]);
                apart();
            }
        }
        if (a.has_post) norm(b, a.post);
#pragma unroll
        for (int p = 0; p < PER; p++) {
            if (a.channel) {
                const Eight w = load8<QMOE_F32>(a.channel, 0, 8 * me + p * step, a.d);
#pragma unroll
                for (int i = 0; i < 8; i++) b[p].v[i] *= w.v[i];
            }
#pragma unroll
            for (int i = 0; i < 8; i++) h[p].v[i] = fmaf(a.alpha, b[p].v[i], h[p].v[i]);
            // a norm's mean and bias, or an infinite gate, must not reach the columns from d on
#pragma unroll
            for (int i = 0; i < 8; i++) h[p].v[i] = 8 * me + p * step + i < a.d ? h[p].v[i] : 0.0f;
            apart();
        }
    }
    if (a.h_out) {
#pragma unroll
        for (int p = 0; p < PER; p++) store8<HT>(a.h_out, (size_t)row * a.ld_h_out, 8 * me + p * step, a.d, h[p]);
    }
    if (a.x) {
        if (a.has_pre) norm(h, a.pre);
        for (int j = 0; j < a.copies; j++)
#pragma unroll
            for (int p = 0; p < PER; p++)
                store8<QMOE_BF16>(a.x, ((size_t)row * a.copies + j) * a.ld_x, 8 * me + p * step, a.d, h[p]);
    }
}

template <int HT, int YT>
qmoe_status launch_norm(const NormArgs &a, int per, hipStream_t s)
{
    const bool alone = a.waves == 1;
    const dim3 grid(alone ? (a.n_tokens + 3) / 4 : a.n_tokens), threads(alone ? 256 : 64 * a.waves);
    if (alone) hipLaunchKernelGGL((k_residual_norm<HT, YT, 1, true>), grid, threads, 0, s, a);
    else if (per == 1) hipLaunchKernelGGL((k_residual_norm<HT, YT, 1, false>), grid, threads, 0, s, a);
    else if (per == 2) hipLaunchKernelGGL((k_residual_norm<HT, YT, 2, false>), grid, threads, 0, s, a);
    else hipLaunchKernelGGL((k_residual_norm<HT, YT, 4, false>), grid, threads, 0, s, a);
    QMOE_HIP_TRY(hipGetLastError());
    return QMOE_OK;
}

bool norm_ok(const qmoe_norm *n)
{
    return !n || ((n->kind == QMOE_NORM_RMS || n->kind == QMOE_NORM_LAYER) && n->eps >= 0.0f);
}
bool type_ok(int t) { return t == QMOE_F32 || t == QMOE_BF16; }

}  // namespace
}  // namespace qmoe

using namespace qmoe;

extern "C" qmoe_status qmoe_residual_norm(const void *h, int h_type, size_t ld_h, const void *y, int y_type, size_t ld_y, int k,
                                          const float *gate, const qmoe_norm *post, float alpha, const float *channel_scale,
                                          const qmoe_norm *pre, void *h_out, size_t ld_h_out, uint16_t *x_bf16, size_t ld_x,
                                          int copies, int n_tokens, int d, void *stream)
{
    if (!y) k = 1, y_type = QMOE_F32, post = nullptr;
    if (!x_bf16) copies = 1, pre = nullptr;
    if (!h || (!h_out && !x_bf16) || n_tokens < 1 || d < 1 || k < 1 || copies < 1 || !type_ok(h_type) || !type_ok(y_type) ||
        !norm_ok(post) || !norm_ok(pre) || ld_h < (size_t)d || (y && ld_y < (size_t)d) || (h_out && ld_h_out < (size_t)d) ||
        (x_bf16 && ld_x < (size_t)d) || (h_out == h && ld_h_out != ld_h))
        return QMOE_E_INVALID_ARG;
    if (n_tokens > kMaxTokens || d > kMaxCols || k > kMaxJoined || copies > kMaxJoined) return QMOE_E_LIMIT;
    NormArgs a{};
    a.h = h;
    a.y = y;
    a.h_out = h_out;
    a.x = x_bf16;
    a.ld_h = ld_h;
    a.ld_y = ld_y;
    a.ld_h_out = ld_h_out;
    a.ld_x = ld_x;
    a.gate = y ? gate : nullptr;
    a.channel = y ? channel_scale : nullptr;
    if (post) a.post = *post, a.has_post = 1;
    if (pre) a.pre = *pre, a.has_pre = 1;
    a.alpha = alpha;
    a.inv_d = 1.0f / (float)d;
    a.k = k;
    a.copies = copies;
    a.n_tokens = n_tokens;
    a.d = d;
    const int eights = (d + 7) / 8;
    const int per = eights <= 1024 ? 1 : (eights <= 2048 ? 2 : 4);
    a.waves = (eights + 64 * per - 1) / (64 * per);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (h_type == QMOE_F32)
        return y_type == QMOE_F32 ? launch_norm<QMOE_F32, QMOE_F32>(a, per, s)
                                  : launch_norm<QMOE_F32, QMOE_BF16>(a, per, s);
    return y_type == QMOE_F32 ? launch_norm<QMOE_BF16, QMOE_F32>(a, per, s)
                              : launch_norm<QMOE_BF16, QMOE_BF16>(a, per, s);
}

// qmoe_route: the experts of every token and their gates, from the router's logits.
#include <cfloat>

#include "qmoe_ops.h"

namespace qmoe {
namespace {

struct RouteArgs {
    const void *logits;
    size_t ld;
    const float *bias;
    const uint8_t *mask;
    int *idx;
    float *gate;
    int n_tokens, n_experts, k, chosen;
};

// A logit as the operator counts it: masked (-infinity) if it is NaN, finite if it is +infinity.
__device__ __forceinline__ float counted(float l) { return l == l ? fminf(l, FLT_MAX) : -INFINITY; }
__device__ __forceinline__ float key_of(float l, float bias) { return counted(l + bias); }  // (of a masked l: -infinity, or NaN, which counts as that)

template <int TYPE>
__device__ __forceinline__ float logit(const void *base, size_t at)
{
    if constexpr (TYPE == QMOE_F32) return static_cast<const float *>(base)[at];
    else return bf16_bits_to_float(static_cast<const uint16_t *>(base)[at]);
}

// Over the LANES lanes (16: a row of the wavefront; 64: all of it) that share a token, in every one of them.
template <int LANES, typename F>
__device__ __forceinline__ float over_lanes(float x, F f)
{
    x = f(x, dpp_f<0x121, 0xf>(x, x));
    x = f(x, dpp_f<0x122, 0xf>(x, x));
    x = f(x, dpp_f<0x124, 0xf>(x, x));
    x = f(x, dpp_f<0x128, 0xf>(x, x));
    if constexpr (LANES == 64) {
        const float a = f(__int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 15)),
                          __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 31)));
        const float b = f(__int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 47)),
                          __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63)));
        x = f(a, b);
    }
    return x;
}
template <int LANES>
__device__ __forceinline__ float lanes_max(float x)
{
    return over_lanes<LANES>(x, [](float a, float b) { return fmaxf(a, b); });
}
template <int LANES>
__device__ __forceinline__ float lanes_sum(float x)
{
    return over_lanes<LANES>(x, [](float a, float b) { return a + b; });
}
template <int LANES>
__device__ __forceinline__ int lanes_min(int x)
{
    auto step = [&](auto ctrl) {
        constexpr int c = decltype(ctrl)::value;
        x = min(x, __builtin_amdgcn_update_dpp(x, x, c, 0xf, 0xf, false));
    };
    step(std::integral_constant<int, 0x121>{});
    step(std::integral_constant<int, 0x122>{});
    step(std::integral_constant<int, 0x124>{});
    step(std::integral_constant<int, 0x128>{});
    if constexpr (LANES == 64)
        x = min(min(__builtin_amdgcn_readlane(x, 15), __builtin_amdgcn_readlane(x, 31)),
                min(__builtin_amdgcn_readlane(x, 47), __builtin_amdgcn_readlane(x, 63)));
    return x;
}

// The gates of the experts that the token's first k lanes hold (mine, -1 = none), and what the call returns of them.
template <int TYPE, int LANES>
__device__ __forceinline__ void finish(const RouteArgs &a, int t, int l, int mine, float top, float sum)
{
    float v = -INFINITY;
    if (l < a.k && mine >= 0) v = counted(logit<TYPE>(a.logits, (size_t)t * a.ld + mine));
    if (a.chosen) {
        top = lanes_max<LANES>(v);
        sum = lanes_sum<LANES>(v == -INFINITY ? 0.0f : expf(v - top));
    }
    if (l < a.k) {
        a.idx[(size_t)t * a.k + l] = mine;
        a.gate[(size_t)t * a.k + l] = mine >= 0 ? expf(v - top) / sum : 0.0f;
    }
}

// exp(v - top) for a sum; top is finite and the largest.  The hardware's exponential is that of 2^p, p = x log2 e rounded to fp32, which is off by |x| half steps or so
// and by the same for equal logits: 2047 of them 5.7 below the largest put a sum of 2048 off by four to six (root mean square over such distances).  What p stands for, p ln 2,
// is known to more bits than x has (ln 2 in two parts), and the difference put right.  (expf: 12.0 us for 4096 tokens of 2048, 10.4 so, 9.9 uncorrected.)
__device__ __forceinline__ float share(float v, float top)
{
    const float x = fmaxf(v - top, -200.0f);  // (exp(-200) is 0)
    const float p = x * 1.4426950408889634f;
    const float off = fmaf(p, 1.9046542e-9f, fmaf(p, -0.6931471824645996f, x));
    const float e = __expf(x);
    return fmaf(e, off, e);
}
// The sum over N values, halves joined: log2 N roundings.
template <int N, int PER>
__device__ __forceinline__ float shares(const float (&v)[PER], float top, int from = 0)
{
    if constexpr (N == 1) return share(v[from], top);
    else return shares<N / 2>(v, top, from) + shares<N / 2>(v, top, from + N / 2);
}

// Four consecutive logits from expert e on (n_experts a multiple of four, or elementwise).
template <int TYPE>
__device__ __forceinline__ void four_logits(float (&v)[4], const void *base, size_t row, int e, int n_experts, bool there)
{
    const bool whole = (n_experts & 3) == 0;
#pragma unroll
    for (int j = 0; j < 4; j++) v[j] = -INFINITY;
    if (whole) {
        if (there && e < n_experts) {
            if constexpr (TYPE == QMOE_F32) {
                const f32x4 q = *reinterpret_cast<const f32x4_by4 *>(static_cast<const float *>(base) + row + e);
#pragma unroll
                for (int j = 0; j < 4; j++) v[j] = q[j];
            } else {
                typedef uint32_t u32x2_by2 __attribute__((ext_vector_type(2), aligned(2)));
                const u32x2_by2 q = *reinterpret_cast<const u32x2_by2 *>(static_cast<const uint16_t *>(base) + row + e);
#pragma unroll
                for (int j = 0; j < 4; j++) v[j] = __uint_as_float(j % 2 ? q[j / 2] & 0xFFFF0000u : q[j / 2] << 16);
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; j++)
            if (there && e + j < n_experts) v[j] = logit<TYPE>(base, row + e + j);
    }
}

// A token's keys lie in the registers of LANES lanes, four neighbouring experts in a lane's four registers, then those 4 * LANES further: one
// pass over memory.  Each of the k rounds takes the largest key (a reduction over the lanes), of equal ones that of the lowest
// index (a second one), and the lane that held it looks for its next best.
// With many experts memory bounds it: 4096 tokens of 2048 fp32 logits (34 MB) 9.8 us, 3.4 TB/s; with few instruction issue
// does: 16384 tokens of 256 bf16 logits, best eight, 10.6 us for 9.4 MB, 1280 vector instructions a wavefront of four tokens, two thirds of them
// looking for the next best of 16 keys.  Keeping each lane's second best, too, was 17: with eight of 16 lanes' keys to take, some lane of four tokens needs
// its third in nearly every round.  16 lanes a token up to 256 experts keep the reductions inside
// a row of the wavefront (four DPP steps) and four tokens in one instruction.
template <int TYPE, int LANES, int PER, bool BIAS>
__global__ __launch_bounds__(256) void k_route(const RouteArgs a)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = lane & (LANES - 1);
    const int per_wave = 64 / LANES;
    const int t = (int)(blockIdx.x * 4 + wave) * per_wave + lane / LANES;
    const bool there = t < a.n_tokens && !(a.mask && a.mask[t] == 0);
    auto expert = [&](int i) { return 4 * l + 4 * LANES * (i >> 2) + (i & 3); };
    float key[PER];
    float top = 0.0f, sum = 0.0f;
    {
        float v[PER];
#pragma unroll
        for (int i = 0; i < PER; i += 4) {
            float q[4];
            four_logits<TYPE>(q, a.logits, (size_t)t * a.ld, expert(i), a.n_experts, there);
#pragma unroll
            for (int j = 0; j < 4; j++) v[i + j] = q[j];
        }
        if constexpr (BIAS) {
#pragma unroll
            for (int i = 0; i < PER; i += 4) {
                float q[4];
                four_logits<QMOE_F32>(q, a.bias, 0, expert(i), a.n_experts, true);
#pragma unroll
                for (int j = 0; j < 4; j++) key[i + j] = q[j];
            }
        }
#pragma unroll
        for (int i = 0; i < PER; i++) {
            v[i] = counted(v[i]);
            key[i] = BIAS ? key_of(v[i], key[i]) : v[i];
        }
        if (!a.chosen) {
            top = v[0];
#pragma unroll
            for (int i = 1; i < PER; i++) top = fmaxf(top, v[i]);
            top = fmaxf(lanes_max<LANES>(top), -FLT_MAX);
            sum = lanes_sum<LANES>(shares<PER>(v, top));
        }
    }
    float best = key[0];
    int best_i = 0;
#pragma unroll
    for (int i = 1; i < PER; i++)
        if (key[i] > best) best = key[i], best_i = i;
    int mine = -1;
    for (int j = 0; j < a.k; j++) {
        const float m = lanes_max<LANES>(best);
        const int e = lanes_min<LANES>(best == m ? expert(best_i) : 0x7FFFFFFF);
        if (l == j) mine = m == -INFINITY ? -1 : e;
        if (j + 1 == a.k) break;
        if (e == expert(best_i)) {  // one lane of the token's
            best = -INFINITY;
            const int gone = best_i;
#pragma unroll
            for (int i = 0; i < PER; i++) {
                if (i == gone) key[i] = -INFINITY;
                if (key[i] > best) best = key[i], best_i = i;
            }
        }
    }
    if (t < a.n_tokens) finish<TYPE, LANES>(a, t, l, mine, top, sum);
}

// More experts than a wavefront's registers hold: a workgroup a token, its keys in the registers of 512 lanes.  The rounds are k_route's, joined over the
// wavefronts through LDS, one barrier each (two places in turn).  4096 tokens of 4096 experts, best eight: 60 us; 64 of 16384: 12; reading the
// logits again for every round took 119 and 119.  The rounds bound it, as above: the reading takes 14 and less than 1.
constexpr int kWideLanes = 512;

template <int TYPE, int PER>
__global__ __launch_bounds__(kWideLanes) void k_route_wide(const RouteArgs a)
{
    constexpr int WAVES = kWideLanes / 64;
    __shared__ float s_top[WAVES], s_sum[WAVES], s_val[2][WAVES];
    __shared__ int s_idx[2][WAVES];
    const int t = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const bool there = !(a.mask && a.mask[t] == 0);
    auto expert = [&](int i) { return 4 * (int)threadIdx.x + 4 * kWideLanes * (i >> 2) + (i & 3); };
    float key[PER];
#pragma unroll
    for (int i = 0; i < PER; i += 4) {
        float q[4];
        four_logits<TYPE>(q, a.logits, (size_t)t * a.ld, expert(i), a.n_experts, there);
#pragma unroll
        for (int j = 0; j < 4; j++) key[i + j] = counted(q[j]);
    }
    float top = 0.0f, sum = 0.0f;
    if (!a.chosen) {
        top = key[0];
#pragma unroll
        for (int i = 1; i < PER; i++) top = fmaxf(top, key[i]);
        top = lanes_max<64>(top);
        if (lane == 0) s_top[wave] = top;
        __syncthreads();
        for (int w = 0; w < WAVES; w++) top = fmaxf(top, s_top[w]);
        top = fmaxf(top, -FLT_MAX);
        sum = lanes_sum<64>(shares<PER>(key, top));
        if (lane == 0) s_sum[wave] = sum;
        __syncthreads();
        sum = 0.0f;
        for (int w = 0; w < WAVES; w++) sum += s_sum[w];
    }
    if (a.bias) {
#pragma unroll
        for (int i = 0; i < PER; i += 4) {
            float q[4];
            four_logits<QMOE_F32>(q, a.bias, 0, expert(i), a.n_experts, true);
#pragma unroll
            for (int j = 0; j < 4; j++) key[i + j] = key_of(key[i + j], q[j]);
        }
    }
    float best = key[0];
    int best_i = 0, mine = -1;
#pragma unroll
    for (int i = 1; i < PER; i++)
        if (key[i] > best) best = key[i], best_i = i;
    for (int j = 0; j < a.k; j++) {
        float m = lanes_max<64>(best);
        int e = lanes_min<64>(best == m ? expert(best_i) : 0x7FFFFFFF);
        if (lane == 0) s_val[j & 1][wave] = m, s_idx[j & 1][wave] = e;
        __syncthreads();
        for (int w = 0; w < WAVES; w++) {
            const float v = s_val[j & 1][w];
            const int at = s_idx[j & 1][w];
            e = v > m || (v == m && at < e) ? at : e;
            m = fmaxf(m, v);
        }
        if (m == -INFINITY) break;  // the same for the whole workgroup
        if (lane == j) mine = e;
        if (e == expert(best_i)) {  // one lane
            best = -INFINITY;
            const int gone = best_i;
#pragma unroll
            for (int i = 0; i < PER; i++) {
                if (i == gone) key[i] = -INFINITY;
                if (key[i] > best) best = key[i], best_i = i;
            }
        }
    }
    if (wave == 0) finish<TYPE, 64>(a, t, lane, mine, top, sum);
}

template <int TYPE, int LANES, int PER>
void launch_per(const RouteArgs &a, hipStream_t s)
{
    const int a_block = 4 * (64 / LANES), grid = (a.n_tokens + a_block - 1) / a_block;
    if (a.bias) hipLaunchKernelGGL((k_route<TYPE, LANES, PER, true>), dim3(grid), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k_route<TYPE, LANES, PER, false>), dim3(grid), dim3(256), 0, s, a);
}

static_assert(kMaxExperts <= 32 * kWideLanes, "k_route_wide holds every key");

template <int TYPE>
qmoe_status launch_route(const RouteArgs &a, hipStream_t s)
{
    const int e = a.n_experts;
    if (e <= 64) launch_per<TYPE, 16, 4>(a, s);
    else if (e <= 128) launch_per<TYPE, 16, 8>(a, s);
    else if (e <= 256) launch_per<TYPE, 16, 16>(a, s);
    else if (e <= 512) launch_per<TYPE, 64, 8>(a, s);
    else if (e <= 1024) launch_per<TYPE, 64, 16>(a, s);
    else if (e <= 2048) launch_per<TYPE, 64, 32>(a, s);
    else if (e <= 8 * kWideLanes) hipLaunchKernelGGL((k_route_wide<TYPE, 8>), dim3(a.n_tokens), dim3(kWideLanes), 0, s, a);
    else if (e <= 16 * kWideLanes) hipLaunchKernelGGL((k_route_wide<TYPE, 16>), dim3(a.n_tokens), dim3(kWideLanes), 0, s, a);
    else hipLaunchKernelGGL((k_route_wide<TYPE, 32>), dim3(a.n_tokens), dim3(kWideLanes), 0, s, a);
    QMOE_HIP_TRY(hipGetLastError());
    return QMOE_OK;
}

}  // namespace
}  // namespace qmoe

using namespace qmoe;

extern "C" qmoe_status qmoe_route(const void *logits, int logits_type, size_t ld, const float *bias, const uint8_t *token_mask,
                                  int n_tokens, int n_experts, int k, int gates, int32_t *expert_idx, float *gate, void *stream)
{
    if (!logits || !expert_idx || !gate || n_tokens < 1 || n_experts < 1 || k < 1 || k > n_experts || ld < (size_t)n_experts ||
        (logits_type != QMOE_F32 && logits_type != QMOE_BF16) || (gates != QMOE_GATES_ALL && gates != QMOE_GATES_CHOSEN))
        return QMOE_E_INVALID_ARG;
    if (n_experts > kMaxExperts || n_tokens > kMaxTokens || k > kMaxJoined) return QMOE_E_LIMIT;
    const RouteArgs a{logits, ld, bias, token_mask, expert_idx, gate, n_tokens, n_experts, k, gates == QMOE_GATES_CHOSEN};
    hipStream_t s = static_cast<hipStream_t>(stream);
    return logits_type == QMOE_F32 ? launch_route<QMOE_F32>(a, s) : launch_route<QMOE_BF16>(a, s);
}

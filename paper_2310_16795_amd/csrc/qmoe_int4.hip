// Four-bit weights: the product for few tokens, and the C entry points.
#include "qmoe_int4.h"
#include "qmoe_hooks.h"

namespace qmoe {
namespace {

constexpr int kInt4MaxSplit = 8;
// Layer calls of up to so many tokens do without the dispatch: an item a token, of which an expert's first one takes the others along (a slot's number is four
// bits of a word).  Gated, 8 tokens, so / with the dispatch, us, each on an expert of its own: 128 experts of 768 x 3072 19 / 25, 64 of 1024 x 4096 22 / 27, 8 of 2080 x 6144 57 / 57; all on
// one: 15 / 21, 16 / 21, 24 / 34 (45 with an item for each token).
constexpr int kInt4Direct = 8;

// What both kernels here share.
//
// v_mfma_f32_16x16x32_bf16 takes 16 tokens as its first operand and 16 rows as its second, so a result lane holds one
// row and four tokens and needs one scale.  16 bytes of a row are a lane's operands for four steps of 32 columns and become (q - z) / 16
// (int4_weights); a lane's weights are one row's, so a group's zero point is one for the lane.
// Four neighbouring lanes load the 64 bytes that a row has in a block (one access of the cache; a load in the operands' order, a row a
// lane, is four), and ds_bpermute brings them to their lanes.  In k_int4_split the scales of the next four blocks come in one load, a
// quarter of the wavefront each; k_int4_tile keeps them in LDS.

// SIDES tiles of 16 rows: their weights and scales, as a lane loads them.
template <int SIDES, int BLOCKS, int PER_BLOCK>
struct Int4Rows {
    static constexpr int GROUPS = BLOCKS * PER_BLOCK, WORDS = (GROUPS + 1) / 2, ZERO_WORDS = (GROUPS + 3) / 4;
    const uint8_t *row[SIDES];
    size_t meta[SIDES];
    uint32_t scales[SIDES][WORDS], zeros[SIDES][ZERO_WORDS];

    // the tile's first row on each side, and what stands behind it in the matrix (the other projection)
    __device__ __forceinline__ void at(const Int4Args &a, const Int4Matrix &m, int lane, const int (&base)[SIDES], const int (&behind)[SIDES])
    {
        const size_t row_bytes = (size_t)64 * a.blocks;
#pragma unroll
        for (int g = 0; g < SIDES; g++) {
            row[g] = m.weights + (size_t)(min(base[g] + (lane >> 2), a.rows - 1) + behind[g]) * row_bytes + 16 * (lane & 3);
            meta[g] = (size_t)(min(base[g] + (lane & 15), a.rows - 1) + behind[g]) * a.groups;
        }
    }
    __device__ __forceinline__ void load(u32x4 (&next)[BLOCKS][SIDES], int b, int last) const
    {
#pragma unroll
        for (int u = 0; u < BLOCKS; u++)
#pragma unroll
            for (int g = 0; g < SIDES; g++) next[u][g] = *(gp_u32x4)(row[g] + (size_t)64 * min(b + u, last));
    }
    // scales of the 4 * BLOCKS blocks from b on
    __device__ __forceinline__ void load_scales(const Int4Args &a, const Int4Matrix &m, int quarter, int b)
    {
        const int mine = b + BLOCKS * quarter, g0 = PER_BLOCK * mine;
        if (a.blocks_per_group == 1 && g0 + GROUPS <= a.groups) {
#pragma unroll
            for (int g = 0; g < SIDES; g++) {
                int4_load_packed<2 * GROUPS>(scales[g], m.scale + (meta[g] + g0));
                if (m.zero) int4_load_packed<GROUPS>(zeros[g], m.zero + (meta[g] + g0));
            }
            return;
        }
#pragma unroll
        for (int g = 0; g < SIDES; g++) {
#pragma unroll
            for (int i = 0; i < WORDS; i++) scales[g][i] = 0;
#pragma unroll
            for (int i = 0; i < ZERO_WORDS; i++) zeros[g][i] = 0;
#pragma unroll
            for (int i = 0; i < GROUPS; i++) {
                const int of = a.blocks_per_group > 1 ? (mine + i) / a.blocks_per_group : g0 + i;
                const size_t at = meta[g] + min(of, a.groups - 1);
                scales[g][i / 2] |= (uint32_t)m.scale[at] << (16 * (i % 2));
                if (m.zero) zeros[g][i / 4] |= (uint32_t)m.zero[at] << (8 * (i % 4));
                asm volatile("" ::: "memory");  // (rare: kept from asking for registers that the loop around it needs)
            }
        }
    }
};

// A block's 128 columns: acc += scale * sum over the group of (q - z) x, tokens and rows of this wavefront.
// x: this lane's first operand in LDS, a token's row every ld_x values.
template <int SIDES, int TILES, int PER_BLOCK, int BLOCKS>
__device__ __forceinline__ void int4_block(f32x4 (&acc)[SIDES][TILES], const u32x4 (&w)[SIDES], int u, const uint32_t (&scale_of)[SIDES][Int4Rows<SIDES, BLOCKS, PER_BLOCK>::WORDS],
                                           const uint32_t (&zero_of)[SIDES][Int4Rows<SIDES, BLOCKS, PER_BLOCK>::ZERO_WORDS], bool zeros,
                                           const uint16_t *x, int ld_x)
{
    f32x4 sum[SIDES][TILES];
    Int4Zero zero[SIDES];
#pragma unroll
    for (int s = 0; s < 4; s++) {
        const int i = u * PER_BLOCK + s * PER_BLOCK / 4;
        if (s * PER_BLOCK % 4 == 0) {
#pragma unroll
            for (int g = 0; g < SIDES; g++) {
                zero[g] = int4_zero(zeros ? (zero_of[g][i / 4] >> (8 * (i % 4))) & 255u : 8u);
#pragma unroll
                for (int t = 0; t < TILES; t++) sum[g][t] = (f32x4){0, 0, 0, 0};
            }
        }
        bf16x8 wf[SIDES];
#pragma unroll
        for (int g = 0; g < SIDES; g++) wf[g] = int4_weights(w[g][s], zero[g]);
#pragma unroll
        for (int t = 0; t < TILES; t++) {
            const bf16x8 xf = *reinterpret_cast<const bf16x8 *>(x + 16 * t * ld_x + 32 * s);
#pragma unroll
            for (int g = 0; g < SIDES; g++) sum[g][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xf, wf[g], sum[g][t], 0, 0, 0);
        }
        if ((s + 1) * PER_BLOCK % 4) continue;
#pragma unroll
        for (int g = 0; g < SIDES; g++) {
            const float scale = int4_scale((uint16_t)(scale_of[g][i / 2] >> (16 * (i % 2))));
#pragma unroll
            for (int t = 0; t < TILES; t++)
#pragma unroll
                for (int k = 0; k < 4; k++) acc[g][t][k] = fmaf(scale, sum[g][t][k], acc[g][t][k]);
        }
    }
}

__device__ __forceinline__ bool int4_gates(const Int4Args &a) { return a.activation == QMOE_ACT_SILU_GATED || a.activation == QMOE_ACT_GELU_GATED; }

struct Int4Unit {
    int expert, slot0, ntok;
};
__device__ __forceinline__ Int4Unit int4_unit(const Int4Args &a, int item, int tokens)
{
    if (!a.items) return {0, item * tokens, min(tokens, a.batch - item * tokens)};
    const Item it = a.items[item];
    return {it.expert, it.slot0, min(it.ntok, tokens)};
}
// Direct items: the first token of an expert takes the others along (theirs are empty, ntok 0).  A token without an expert is alone, and its results are 0.
struct Int4Direct {
    int expert, ntok;
    bool none;
    uint32_t slots;  // four bits each
};
__device__ __forceinline__ Int4Direct int4_direct(const Int4Args &a, int item, int lane)
{
    const int mine = a.direct[min(lane, a.max_items - 1)], e = __builtin_amdgcn_readlane(mine, item);
    const bool none = e < 0 || e >= a.n_experts;
    const uint32_t same = none ? 1u << item : (uint32_t)__ballot(lane < a.max_items && mine == e);
    Int4Direct it{none ? 0 : e, 0, none, 0};
#pragma unroll
    for (int j = 0; j < kInt4Direct; j++)
        if (same >> j & 1u) it.slots |= (uint32_t)j << (4 * it.ntok++);
    if (same & ((1u << item) - 1u)) it.ntok = 0;
    return it;
}
__device__ __forceinline__ const uint16_t *int4_x_row(const Int4Args &a, int slot)
{
    return a.x + (size_t)(a.perm && !a.x_by_slot ? a.perm[slot] : slot) * a.ld_x;
}

// Results of 16 tokens (of the tile t) and the SIDES tiles of rows from row on; gated: the two are one's gate and product.  slot_of: where the unit's i-th token stands.
template <int SIDES, typename F>
__device__ __forceinline__ void int4_results(const Int4Args &a, bool gated, const f32x4 (&v)[SIDES], int t, int row, int quarter, int ntok, F slot_of,
                                             bool none = false)
{
#pragma unroll
    for (int k = 0; k < 4; k++) {
        const int in_tile = 16 * t + 4 * quarter + k;
        if (in_tile >= ntok) continue;
        const int slot = slot_of(in_tile), token = a.perm ? a.perm[slot] : slot;
        const size_t out_row = a.out_by_slot ? slot : token;
        const float gate = none ? 0.0f : a.gate ? a.gate[token] : 1.0f;
        if (SIDES == 2 && gated) {
            if (row < a.rows) int4_store(a, out_row, gate, row, int4_gated(v[0][k], v[SIDES - 1][k], a.activation));
        } else {
#pragma unroll
            for (int g = 0; g < SIDES; g++)
                if (row + 16 * g < a.rows) int4_store(a, out_row, gate, row + 16 * g, v[g][k]);
        }
    }
}

// Little work: a workgroup's wavefronts share 16 rows (gated: of each projection) along the columns, each with its own piece of LDS for the
// activations of its block, so that none waits for another before all join their sums, in a fixed order.
// Bound by latency: 4096 x 1024, one token (2.2 MB) 5.2 us (k_route of one token, a launch with next to no work, is 2.2 in the same trace); 2080 x 6144 with zero points, 37 tokens (7.1 MB) 12 us,
// six blocks one after the other in each of 3120 wavefronts, 2080 x 6144 with one token 6.5 us (1 TB/s).
template <int SIDES, int PER_BLOCK, bool DIRECT>
__global__ __launch_bounds__(64 * kInt4MaxSplit) void k_int4_split(const Int4Args a)
{
    extern __shared__ __align__(16) unsigned char smem[];
    constexpr int TOKENS = 16, LD = kInt4BlockCols + 8;  // (16 lanes' reads, a token each, meet no bank twice)
    constexpr int WAVE_BYTES = TOKENS * LD * 2;
    const int lane = threadIdx.x & 63, part = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int n16 = lane & 15, quarter = lane >> 4, from_lane = 4 * (4 * n16 + quarter);
    uint16_t *s_x = reinterpret_cast<uint16_t *>(smem + part * WAVE_BYTES);
    f32x4 *joined = reinterpret_cast<f32x4 *>(smem);
    const bool gated = int4_gates(a);
    const int row_tiles = (a.rows + 15) / 16;
    const int n_items = DIRECT ? a.max_items : a.items ? min(*a.n_items_dev, a.max_items) : (a.batch + TOKENS - 1) / TOKENS;
    const long long total = (long long)n_items * row_tiles;
    const int b0 = (int)((long long)a.blocks * part / a.split), b_end = (int)((long long)a.blocks * (part + 1) / a.split);
    for (long long unit = blockIdx.x; unit < total; unit += gridDim.x) {
        const int item = (int)(unit / row_tiles), tile = (int)(unit - (long long)item * row_tiles);
        int expert, slot0 = 0, ntok;
        uint32_t slots = 0;
        bool none = false;
        if constexpr (DIRECT) {
            const Int4Direct it = int4_direct(a, item, lane);
            if (it.ntok == 0) continue;  // (the same for the workgroup)
            expert = it.expert, ntok = it.ntok, slots = it.slots, none = it.none;
        } else {
            const Int4Unit it = int4_unit(a, item, TOKENS);
            expert = it.expert, slot0 = it.slot0, ntok = it.ntok;
        }
        const int b1 = none ? b0 : b_end;
        auto slot_of = [&](int i) { return DIRECT ? (int)(slots >> (4 * i) & 15u) : slot0 + i; };
        const Int4Matrix m = int4_matrix(a, expert);
        Int4Rows<SIDES, 1, PER_BLOCK> rows;
        int base[SIDES], behind[SIDES];
#pragma unroll
        for (int g = 0; g < SIDES; g++) base[g] = 16 * tile, behind[g] = g * a.rows;
        rows.at(a, m, lane, base, behind);
        const uint16_t *x_row[4];
#pragma unroll
        for (int j = 0; j < 4; j++)
            if (4 * j < ntok) x_row[j] = int4_x_row(a, slot_of(min(4 * j + quarter, ntok - 1)));
        u32x4 x_next[4], w_next[1][SIDES];
        auto load_x = [&](int b) {
#pragma unroll
            for (int j = 0; j < 4; j++)
                if (4 * j < ntok) x_next[j] = int4_x(x_row[j], kInt4BlockCols * b + 8 * n16, a.cols, kInt4BlockCols * (b + 1) <= a.cols);
        };
        f32x4 acc[SIDES][1];
#pragma unroll
        for (int g = 0; g < SIDES; g++) acc[g][0] = (f32x4){0, 0, 0, 0};
        if (b0 < b1) {
            rows.load(w_next, b0, b1 - 1);
            load_x(b0);
        }
        for (int b = b0; b < b1; b++) {
            const int step = (b - b0) & 3;
            if (step == 0) rows.load_scales(a, m, quarter, b);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();  // the block before has been read
#pragma unroll
            for (int j = 0; j < 4; j++) {
                if (4 * j >= ntok) continue;
                *reinterpret_cast<u32x4 *>(&s_x[(4 * j + quarter) * LD + 8 * n16]) = x_next[j];
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            u32x4 w[SIDES];
            uint32_t scale_of[SIDES][decltype(rows)::WORDS], zero_of[SIDES][decltype(rows)::ZERO_WORDS];
#pragma unroll
            for (int g = 0; g < SIDES; g++) {
#pragma unroll
                for (int s = 0; s < 4; s++) w[g][s] = (uint32_t)__builtin_amdgcn_ds_bpermute(from_lane, (int)w_next[0][g][s]);
#pragma unroll
                for (int i = 0; i < decltype(rows)::WORDS; i++)
                    scale_of[g][i] = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * (n16 + 16 * step), (int)rows.scales[g][i]);
                if (m.zero) {
#pragma unroll
                    for (int i = 0; i < decltype(rows)::ZERO_WORDS; i++)
                        zero_of[g][i] = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * (n16 + 16 * step), (int)rows.zeros[g][i]);
                }
            }
            if (b + 1 < b1) {
                rows.load(w_next, b + 1, b1 - 1);
                load_x(b + 1);
            }
            int4_block<SIDES, 1, PER_BLOCK, 1>(acc, w, 0, scale_of, zero_of, bool(m.zero), s_x + n16 * LD + 8 * quarter, LD);
        }
        __syncthreads();  // all have read their activations: the sums take their place
#pragma unroll
        for (int g = 0; g < SIDES; g++) joined[(part * SIDES + g) * 64 + lane] = acc[g][0];
        __syncthreads();
        if (part == 0) {
            f32x4 v[SIDES];
#pragma unroll
            for (int g = 0; g < SIDES; g++) {
                v[g] = joined[g * 64 + lane];
                for (int p = 1; p < a.split; p++) v[g] += joined[(p * SIDES + g) * 64 + lane];
            }
            int4_results<SIDES>(a, gated, v, 0, 16 * tile + n16, quarter, ntok, slot_of, none);
        }
        __syncthreads();  // before the next unit's activations overwrite these
    }
}

// More work: four wavefronts with two tiles of 16 rows each (gated: the same rows of both projections) and all the columns.  Steps of
// two blocks: the activations of the next one and a wavefront's weights are on their way while this one is multiplied; x
// goes through LDS in two turns, a barrier a step.  Up to four tokens each wavefront brings for itself, into a quarter of that LDS, and none waits for
// another.
// The scales and zero points of AT_ONCE groups go through LDS, too, a wavefront's own: a row's few bytes a step, asked for step by step, would
// be the same lines of memory again and again, gone from the caches in between.
// Few tokens an expert: memory and decoding, 64 tokens on 57 of 256 gated experts of 2080 x 6144 (1.17 GB) 284 us for both products, 4.1 TB/s where a large copy
// has 4.9; vector instructions, three quarters of them int4_weights, are issued in 75 % of the first product's cycles.
// More: 128 experts of 768 x 3072, 4001 tokens (38 GFLOP, 310 MB) 168 us: vector instructions in 53 % of the cycles of either product, the matrix cores in 15, and the
// starts of 6072 and 1518 units of three and twelve steps, which one of three wavefronts a SIMD waits for.
template <int TILES, int PER_BLOCK>
__global__ __launch_bounds__(256, TILES == 1 ? 4 : 3) void k_int4_tile(const Int4Args a)
{
    constexpr int TOKENS = 16 * TILES, BLOCKS = 2, COLS = BLOCKS * kInt4BlockCols, LD = COLS + 8, GROUPS = BLOCKS * PER_BLOCK;
    constexpr int AT_ONCE = TILES == 1 ? 32 : 16, LD_SCALE = AT_ONCE + 8, LD_ZERO = AT_ONCE + 8;
    using Rows = Int4Rows<2, BLOCKS, PER_BLOCK>;
    __shared__ __align__(16) uint16_t s_x[2][TOKENS * LD];
    __shared__ __align__(16) uint16_t s_scale[4][2 * 16 * LD_SCALE];
    __shared__ __align__(16) uint8_t s_zero[4][2 * 16 * LD_ZERO];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int n16 = lane & 15, quarter = lane >> 4, from_lane = 4 * (4 * n16 + quarter);
    const bool gated = int4_gates(a);
    const int wave_rows = gated ? 16 : 32, units_per_item = (a.rows + 4 * wave_rows - 1) / (4 * wave_rows);
    const int n_items = a.items ? min(*a.n_items_dev, a.max_items) : (a.batch + TOKENS - 1) / TOKENS;
    const long long total = (long long)n_items * units_per_item;
    for (long long unit = blockIdx.x; unit < total; unit += gridDim.x) {
        const int item = (int)(unit / units_per_item), first = ((int)(unit - (long long)item * units_per_item) * 4 + wave) * wave_rows;
        const Int4Unit it = int4_unit(a, item, TOKENS);
        const Int4Matrix m = int4_matrix(a, it.expert);
        Rows rows;
        rows.at(a, m, lane, {first, gated ? first : first + 16}, {0, gated ? a.rows : 0});
        const bool alone = TILES == 1 && it.ntok <= 4;
        const int piece = threadIdx.x & 31, stager = alone ? lane >> 5 : threadIdx.x >> 5, stagers = alone ? 2 : 8;
        const int place = alone ? 4 * wave : 0;  // of the tile's first token in LDS
        const uint16_t *x_row[2 * TILES];
#pragma unroll
        for (int j = 0; j < 2 * TILES; j++)
            x_row[j] = int4_x_row(a, it.slot0 + min(stagers * j + stager, it.ntok - 1));
        u32x4 x_next[2 * TILES];
        auto load_x = [&](int b) {
#pragma unroll
            for (int j = 0; j < 2 * TILES; j++) x_next[j] = int4_x_load(x_row[j], kInt4BlockCols * b + 8 * piece, a.cols);
        };
        u32x4 w_next[BLOCKS][2];
        rows.load(w_next, 0, a.blocks - 1);
        load_x(0);
        // groups g0 .. g0 + AT_ONCE - 1 of the wavefront's 32 rows, eight groups a lane
        auto fill = [&](int g0) {
            constexpr int LANES = AT_ONCE / 8, AT = 64 / LANES;  // lanes of a row, rows at a time
#pragma unroll
            for (int j = 0; j < 32 / AT; j++) {
                const int r = AT * j + lane / LANES, at = 8 * (lane % LANES), side = r >> 4;
                const int base = gated ? first : first + 16 * side;
                const size_t row = (size_t)(min(base + (r & 15), a.rows - 1) + (gated ? side * a.rows : 0)) * a.groups;
                if (g0 + at >= PER_BLOCK * a.blocks) continue;  // (nothing behind the last block is read)
                uint16_t *to = &s_scale[wave][r * LD_SCALE + at];
                uint8_t *to_zero = &s_zero[wave][r * LD_ZERO + at];
                if (g0 + at + 8 <= a.groups) {
                    uint32_t v[4], z[2] = {0x08080808u, 0x08080808u};
                    int4_load_packed<16>(v, m.scale + (row + g0 + at));
                    if (m.zero) int4_load_packed<8>(z, m.zero + (row + g0 + at));
                    *reinterpret_cast<u32x4 *>(to) = (u32x4){v[0], v[1], v[2], v[3]};
                    *reinterpret_cast<uint2 *>(to_zero) = make_uint2(z[0], z[1]);
                } else {
                    for (int i = 0; i < 8; i++) {  // 0 behind the last group: its columns are none, but what lies there could be infinite
                        const bool is = g0 + at + i < a.groups;
                        to[i] = is ? m.scale[row + g0 + at + i] : 0;
                        to_zero[i] = is && m.zero ? m.zero[row + g0 + at + i] : 8;
                    }
                }
            }
        };
        f32x4 acc[2][TILES];
#pragma unroll
        for (int g = 0; g < 2; g++)
#pragma unroll
            for (int t = 0; t < TILES; t++) acc[g][t] = (f32x4){0, 0, 0, 0};
        __syncthreads();  // the unit before has read its last steps
        const int x_at = (place + (alone ? n16 & 3 : n16)) * LD + 8 * quarter;
        const int last_step = (a.blocks - 1) / BLOCKS * BLOCKS;
        auto one_step = [&](int b, int g_from, int turn) {
            if (kInt4BlockCols * b + COLS > a.cols) {
#pragma unroll
                for (int j = 0; j < 2 * TILES; j++) x_next[j] = int4_x_end(x_next[j], kInt4BlockCols * b + 8 * piece, a.cols);
            }
#pragma unroll
            for (int j = 0; j < 2 * TILES; j++) {
                if (alone && j > 1) break;
                const int token = place + stagers * j + stager;
                *reinterpret_cast<u32x4 *>(&s_x[turn][token * LD + 8 * piece]) = x_next[j];
            }
            if (alone) {
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                __builtin_amdgcn_wave_barrier();
            } else {
                __syncthreads();
            }
            u32x4 w[BLOCKS][2];
            uint32_t scale_of[2][Rows::WORDS], zero_of[2][Rows::ZERO_WORDS];
            // the step's groups, from the first that lies in LDS on
            const int from = (a.blocks_per_group > 1 ? b / a.blocks_per_group : b * PER_BLOCK) - g_from;
#pragma unroll
            for (int g = 0; g < 2; g++) {
#pragma unroll
                for (int u = 0; u < BLOCKS; u++)
#pragma unroll
                    for (int s = 0; s < 4; s++) w[u][g][s] = (uint32_t)__builtin_amdgcn_ds_bpermute(from_lane, (int)w_next[u][g][s]);
                const int r = 16 * g + n16;
                const uint16_t *scale = &s_scale[wave][r * LD_SCALE];
                const uint8_t *zero = &s_zero[wave][r * LD_ZERO];
                if constexpr (PER_BLOCK == 1) {
                    const int then = (a.blocks_per_group > 1 ? (b + 1) / a.blocks_per_group : b + 1) - g_from;
                    scale_of[g][0] = (uint32_t)scale[from] | (uint32_t)scale[then] << 16;
                    zero_of[g][0] = (uint32_t)zero[from] | (uint32_t)zero[then] << 8;
                } else {
                    __builtin_memcpy(scale_of[g], __builtin_assume_aligned(scale + from, 2 * GROUPS), 2 * GROUPS);
                    __builtin_memcpy(zero_of[g], __builtin_assume_aligned(zero + from, GROUPS), GROUPS);
                }
            }
            rows.load(w_next, b + BLOCKS, a.blocks - 1);
            load_x(min(b + BLOCKS, last_step));
#pragma unroll
            for (int u = 0; u < BLOCKS; u++) {
                if (b + u >= a.blocks) break;
                int4_block<2, TILES, PER_BLOCK, BLOCKS>(acc, w[u], u, scale_of, zero_of, true, s_x[turn] + x_at + kInt4BlockCols * u, LD);
            }
        };
        const int span = a.blocks_per_group > 1 ? AT_ONCE * a.blocks_per_group : AT_ONCE / PER_BLOCK;  // blocks whose scales lie in LDS
        int turn = 0;
        for (int s0 = 0; s0 < a.blocks; s0 += span) {
            const int g_from = a.blocks_per_group > 1 ? s0 / a.blocks_per_group : s0 * PER_BLOCK, s1 = min(a.blocks, s0 + span);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();  // the wavefront has read those before
            fill(g_from);
            for (int b = s0; b < s1; b += BLOCKS, turn ^= 1) one_step(b, g_from, turn);
        }
#pragma unroll
        for (int t = 0; t < TILES; t++) {
            if (16 * t >= it.ntok) break;
            const f32x4 v[2] = {acc[0][t], acc[1][t]};
            int4_results<2>(a, gated, v, t, first + n16, quarter, it.ntok, [&](int i) { return it.slot0 + i; });
        }
    }
}

bool group_ok(int group) { return group == 32 || group == 64 || (group > 0 && group % kInt4BlockCols == 0); }

// rows: results a token
void fill_shape(Int4Args *a, int rows, int cols, int group)
{
    a->rows = rows;
    a->cols = cols;
    a->blocks = (cols + kInt4BlockCols - 1) / kInt4BlockCols;
    a->groups = (int)(((long long)cols + group - 1) / group);
    a->per_block = group < kInt4BlockCols ? kInt4BlockCols / group : 1;
    a->blocks_per_group = group < kInt4BlockCols ? 1 : group / kInt4BlockCols;
}

template <int SIDES, int PER_BLOCK>
qmoe_status launch_split_variant(const Int4Args &a, int grid, hipStream_t s)
{
    const size_t x = a.split * (16 * (kInt4BlockCols + 8) * 2);
    const size_t smem = std::max(x, (size_t)a.split * SIDES * 64 * sizeof(f32x4));
    const auto kernel = a.direct ? k_int4_split<SIDES, PER_BLOCK, true> : k_int4_split<SIDES, PER_BLOCK, false>;
    const qmoe_status st = allow_lds(kernel, smem);
    if (st != QMOE_OK) return st;
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(64 * a.split), smem, s, a);
    QMOE_HIP_TRY(hipGetLastError());
    return QMOE_OK;
}
template <int SIDES>
qmoe_status launch_split(const Int4Args &a, int grid, hipStream_t s)
{
    if (a.per_block == 1) return launch_split_variant<SIDES, 1>(a, grid, s);
    if (a.per_block == 2) return launch_split_variant<SIDES, 2>(a, grid, s);
    return launch_split_variant<SIDES, 4>(a, grid, s);
}
template <int TILES>
qmoe_status launch_tile(const Int4Args &a, int grid, hipStream_t s)
{
    if (a.per_block == 1) hipLaunchKernelGGL((k_int4_tile<TILES, 1>), dim3(grid), dim3(256), 0, s, a);
    else if (a.per_block == 2) hipLaunchKernelGGL((k_int4_tile<TILES, 2>), dim3(grid), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((k_int4_tile<TILES, 4>), dim3(grid), dim3(256), 0, s, a);
    QMOE_HIP_TRY(hipGetLastError());
    return QMOE_OK;
}

// How a product of up to `tokens` (and no more than 512 or so of one matrix) is split, by what each way takes, us: a start, and as often as the compute
// units are full (k_int4_split: wavefronts, which follow each other one by one), or in turns of a workgroup each (k_int4_tile), the steps.  Fitted to single matrices of
// 384 x 1024, 1024 x 768, 4096 x 1024, 2080 x 6144, 6144 x 2080 and 12288 x 2080, 1 to 1024 tokens, groups of 128: from 9 us on the way it picks is within 8 % of the best
// one in all but one of these 60 (2080 x 6144, 64 tokens, 14 %), and with groups of 32 and 64, zero points or gates in all but three of 45 (2080 x 6144: 64 tokens 12 and 32 %, 512 13 %).
// Measured, the best k_int4_split / k_int4_tile with 16 tokens an item / with 32: 2080 x 6144, 16 tokens 9.0 / 35 / -, 128 23 /
// 37 / 41, 256 39 / 52 / 43, 512 65 / 69 / 59; 4096 x 1024, 64 7.5 / 9.8 / 11, 128 9.7 / 10 / 11, 512 25 / 20 / 16; 12288 x 2080, 1 7.8 / 15 / -,
// 16 12 / 17 / -, 64 25 / 23 / 19, 256 70 / 51 / 35; 1024 x 768, 256 6.8 / 9.6 / 10, 1024 - / 13 / 11.
struct Int4Way {
    double us;
    int split;  // wavefronts that share a tile's columns (k_int4_split); 0: k_int4_tile, or ...
    int tiles;  // of 16 tokens, an item (0: k_int4_mm)
};
int kernel_of(const Int4Way &w) { return w.split ? 1 : w.tiles ? 1 + w.tiles : 4; }
// items: of up to 16 tokens, how many the call has at most
Int4Way split_way(const Int4Args &a, long long items, int tokens, int cus)
{
    const double groups = (double)items * ((a.rows + 15) / 16);
    const double block = (0.38 + 0.022 * std::min(tokens, 16)) * (int4_is_gated(a.activation) ? 1.5 : 1.0);
    Int4Way best{1e30, 1, 1};
    for (int split = 1; split <= kInt4MaxSplit && (split == 1 || split / 2 < a.blocks); split *= 2) {
        const double full = groups * split / (16.0 * cus);  // four wavefronts a SIMD
        const double us = 1.5 + 0.5 * split + std::max(1.0, full) * (2.0 + block * (1.0 + 0.9 * std::min(1.0, full)) * ((a.blocks + split - 1) / split));
        if (us < best.us) best = {us, split, 1};
    }
    return best;
}
long long tile_units(const Int4Args &a, long long items)
{
    return items * (int4_is_gated(a.activation) ? (a.rows + 63) / 64 : (a.rows + 127) / 128);
}
Int4Way tile_way(const Int4Args &a, int tiles, long long items, int cus)
{
    const double more = (double)((tile_units(a, items) - 1) / cus), steps = (a.blocks + 1) / 2;
    return {tiles == 1 ? 5.0 + steps * (1.3 + 0.7 * more) : 5.6 + steps * (1.5 + 0.88 * more), 0, tiles};
}
// of up to 16 tokens an item
Int4Way narrow_way(const Int4Args &a, long long items, int tokens, int cus)
{
    const Int4Way split = split_way(a, items, tokens, cus), tile = tile_way(a, 1, items, cus);
    return a.direct || a.cols < 8 || split.us <= tile.us ? split : tile;  // (k_int4_tile loads eight columns, and knows no direct items)
}
qmoe_status launch_way(Int4Args a, const Int4Way &way, long long items, int cus, hipStream_t s)
{
    if (way.split) {
        a.split = way.split;
        const int grid = (int)std::min<long long>(items * ((a.rows + 15) / 16), 32LL * cus);
        return int4_is_gated(a.activation) ? launch_split<2>(a, grid, s) : launch_split<1>(a, grid, s);
    }
    const int grid = (int)std::min<long long>(tile_units(a, items), 64LL * cus);
    return way.tiles == 1 ? launch_tile<1>(a, grid, s) : launch_tile<2>(a, grid, s);
}

// One matrix: the kernel for many tokens where it fills the GPU one and a half times (12288 x 2080, 256 tokens 37 us, the other way 35; 512 52 /
// 61; 1024 77 / 110).  In layer calls, where tiles are partly empty, it lost (16 experts of 1024 x 4096, 4001 tokens 213, the other way 182;
// 64 of 1024 x 2048, 1000 tokens 122 / 68, both with the earlier decoding).
long long mm_units(const Int4Args &a)
{
    const int rows = int4_is_gated(a.activation) ? 128 : 256;
    return ((a.batch + 63LL) / 64) * ((a.rows + rows - 1) / rows);
}
Int4Way matrix_way(const Int4Args &a, int cus)
{
    if (a.batch > 64 && 2 * mm_units(a) >= 3LL * cus && a.cols >= 8) return {0, 0, 0};
    const Int4Way narrow = narrow_way(a, (a.batch + 15) / 16, a.batch, cus), wide = tile_way(a, 2, (a.batch + 31) / 32, cus);
    return a.batch > 16 && a.cols >= 8 && wide.us < narrow.us ? wide : narrow;
}
qmoe_status launch_matrix(const Int4Args &a, int cus, hipStream_t s)
{
    const Int4Way way = matrix_way(a, cus);
    if (way.tiles) return launch_way(a, way, (a.batch + 16LL * way.tiles - 1) / (16 * way.tiles), cus, s);
    const int grid = (int)std::min<long long>(mm_units(a), 64LL * cus);
    if (int4_is_gated(a.activation)) return a.zero ? launch_int4_mm_gated_zeros(a, grid, s) : launch_int4_mm_gated(a, grid, s);
    return a.zero ? launch_int4_mm_zeros(a, grid, s) : launch_int4_mm_plain(a, grid, s);
}

// A layer call's two products.  Experts' tokens go in tiles of 16 or of 32, whichever has less to do if every expert leaves a tile partly empty.  (16 / 32, us:
// 128 experts of 768 x 3072, 4001 tokens 210 / 164; 16 of 1024 x 4096, 4001 239 / 176; 64 of 1024 x 2048, 1000 Zipf 71 / 70; 32 of 512 x 1024, 400 28 / 29; 256 gated ones of
// 2080 x 6144, zero points, 300 838 / 1051.)
struct Int4LayerWays {
    Int4Way up, down;
    long long items;
};
Int4LayerWays layer_ways(const Int4Args &up, const Int4Args &down, int n_experts, int n_tokens, int cus)
{
    const int most = up.direct ? 1 : 16;
    const long long items = up.direct ? n_tokens : std::min(n_tokens, n_experts + n_tokens / 16), wide_items = std::min(n_tokens, n_experts + n_tokens / 32);
    const Int4LayerWays narrow{narrow_way(up, items, most, cus), narrow_way(down, items, most, cus), items};
    const Int4LayerWays wide{tile_way(up, 2, wide_items, cus), tile_way(down, 2, wide_items, cus), wide_items};
    return n_tokens > 16 && wide.up.us + wide.down.us < narrow.up.us + narrow.down.us ? wide : narrow;
}

}  // namespace
}  // namespace qmoe

using namespace qmoe;

extern "C" {

qmoe_status qmoe_int4_matvec(const qmoe_int4_matrix *W, const uint16_t *x_bf16, size_t ld_x, int batch, int activation, void *y,
                             int y_type, size_t ld_y, void *stream)
{
    if (!W || !W->weights || !W->scale_f16 || !x_bf16 || !y || W->rows < 1 || W->cols < 1 || batch < 1 || !group_ok(W->group) ||
        W->reserved || reinterpret_cast<uintptr_t>(W->weights) % 16 || (y_type != QMOE_F32 && y_type != QMOE_BF16) ||
        activation < QMOE_ACT_NONE || activation > QMOE_ACT_GELU_GATED || (int4_is_gated(activation) && W->rows % 2))
        return QMOE_E_INVALID_ARG;
    const int rows = int4_is_gated(activation) ? W->rows / 2 : W->rows;
    if (ld_x < (size_t)W->cols || ld_y < (size_t)rows) return QMOE_E_INVALID_ARG;
    if (W->rows > kMaxInt4Rows || W->cols > kMaxInt4Cols || batch > kMaxTokens) return QMOE_E_LIMIT;
    DeviceInfo di;
    const qmoe_status st = gpu_info(&di);
    if (st != QMOE_OK) return st;
    Int4Args a{};
    a.weights = W->weights;
    a.scale = W->scale_f16;
    a.zero = W->zero;
    a.batch = batch;
    a.x = x_bf16;
    a.ld_x = ld_x;
    a.out = y;
    a.ld_out = ld_y;
    a.out_f32 = y_type == QMOE_F32;
    a.activation = activation;
    fill_shape(&a, rows, W->cols, W->group);
    return launch_matrix(a, di.cus, static_cast<hipStream_t>(stream));
}

qmoe_status qmoe_int4_layer_forward(const qmoe_int4_matrix *wi, const qmoe_int4_matrix *wo, int group, int activation, int n_experts,
                                    int d_model, int d_ff, const uint16_t *x_bf16, const int32_t *expert_idx, const float *gate,
                                    int n_tokens, void *y, int y_type, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!wi || !wo || !x_bf16 || !expert_idx || !y || !group_ok(group) || (activation != QMOE_ACT_RELU && !int4_is_gated(activation)) ||
        (y_type != QMOE_F32 && y_type != QMOE_BF16) || d_model % 8 || d_ff % 8 || reinterpret_cast<uintptr_t>(x_bf16) % 16 ||
        reinterpret_cast<uintptr_t>(y) % 4)
        return QMOE_E_INVALID_ARG;
    qmoe_status st = layer_workspace_ok(n_tokens, n_experts, d_model, d_ff, workspace, workspace_bytes);
    if (st != QMOE_OK) return st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    DeviceInfo di;
    if ((st = gpu_info(&di)) != QMOE_OK) return st;
    const bool direct = n_tokens <= kInt4Direct;
    Int4Args up{}, down{};
    up.mats = wi;
    down.mats = wo;
    up.n_experts = down.n_experts = n_experts;
    up.activation = activation;
    fill_shape(&up, d_ff, d_model, group);
    fill_shape(&down, d_model, d_ff, group);
    up.direct = down.direct = direct ? expert_idx : nullptr;
    const Int4LayerWays ways = layer_ways(up, down, n_experts, n_tokens, di.cus);
    GroupedTokens g{};
    if (direct) {
        qmoe_ws_layout l;
        if ((st = qmoe_moe_layer_ws_layout(n_experts, d_model, d_ff, n_tokens, &l)) != QMOE_OK) return st;
        g.hidden = reinterpret_cast<uint16_t *>(static_cast<unsigned char *>(workspace) + l.hidden);
    } else if ((st = group_by_expert(expert_idx, n_tokens, n_experts, d_model, d_ff, 16 * ways.up.tiles, workspace, static_cast<float *>(y),
                                     y_type == QMOE_F32 ? d_model : d_model / 2, s, &g)) != QMOE_OK) {
        return st;
    }
    up.perm = down.perm = g.perm;
    up.items = down.items = g.items;
    up.n_items_dev = down.n_items_dev = g.n_items;
    up.max_items = down.max_items = (int)ways.items;
    up.x = x_bf16;
    up.ld_x = d_model;
    up.out = g.hidden;
    up.ld_out = d_ff;
    up.out_by_slot = 1;
    if ((st = launch_way(up, ways.up, ways.items, di.cus, s)) != QMOE_OK) return st;
    down.x = g.hidden;
    down.ld_x = d_ff;
    down.x_by_slot = 1;
    down.out = y;
    down.ld_out = d_model;
    down.out_f32 = y_type == QMOE_F32;
    down.gate = gate;
    down.activation = QMOE_ACT_NONE;
    return launch_way(down, ways.down, ways.items, di.cus, s);
}

int qmoe_hook_int4_kernel(int rows, int cols, int group, int activation, int batch, int compute_units)
{
    if (rows < 1 || cols < 1 || batch < 1 || compute_units < 1 || !group_ok(group)) return 0;
    Int4Args a{};
    a.batch = batch;
    a.activation = activation;
    fill_shape(&a, int4_is_gated(activation) ? rows / 2 : rows, cols, group);
    return kernel_of(matrix_way(a, compute_units));
}

qmoe_status qmoe_hook_int4_layer_kernels(int group, int activation, int n_experts, int d_model, int d_ff, int n_tokens, int compute_units,
                                         int kernels[2])
{
    if (n_experts < 1 || d_model < 1 || d_ff < 1 || n_tokens < 1 || compute_units < 1 || !group_ok(group) || !kernels) return QMOE_E_INVALID_ARG;
    static const int32_t some = 0;
    Int4Args up{}, down{};
    up.activation = activation;
    fill_shape(&up, d_ff, d_model, group);
    fill_shape(&down, d_model, d_ff, group);
    up.direct = down.direct = n_tokens <= kInt4Direct ? &some : nullptr;
    const Int4LayerWays ways = layer_ways(up, down, n_experts, n_tokens, compute_units);
    kernels[0] = kernel_of(ways.up);
    kernels[1] = kernel_of(ways.down);
    return QMOE_OK;
}

}  // extern "C"

// The gradients of attention to states of another length (taser_cross_attention_grad).
//
// With p = exp(x - top) / sum, dp = <dout, v>, t = <dout, out> of a row: dx = p (dp - t); dv = sum of p dout, dk = scale * sum of
// dx q, dq = scale * sum of dx k, dtable = sum of dx by bucket. One kernel owns states and goes over the rows (dk, dv), another
// owns rows and goes over the states (dq, dtable): scores and dp are computed twice (7 products for 5), but nothing is added to
// memory by more than one block, so all sums have one order and need no second pass over a gradient.
// Weights (for dv) and dx (for dk, dq) are rounded to 16-bit types where they enter a product. To multiply what that takes off too, as the
// forward pass does for few rows, costs a third more products: forward and gradient of 2 x 4096 x 4096 take 20 - 26 % longer then, those of
// few rows 2 - 7 %. It is not done: errors are 1.4 times those of the results' own rounding.
#include <cmath>
#include <type_traits>

#include "attention.h"

namespace {

constexpr float kLog2e = 1.4426950408889634f;

// What the passes need of a row: {reference of its scores, log2 of its sum, <dout, out>}; a row without states has weights of 0.
// 16 lanes a row.
template <typename T>
__global__ __launch_bounds__(256) void attention_grad_rows_kernel(const T* out, const T* dout, const float* stats, int32_t stat_floats, int64_t rows, int32_t dim, taser_f4* info) {
    const int64_t row = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
    if (row >= rows) return;
    const int e = 8 * (threadIdx.x & 15);
    const taser_frag<T> x = taser_load_frag<T>(out + row * dim + e, dim - e), y = taser_load_frag<T>(dout + row * dim + e, dim - e);
    float t = 0.f;
    if constexpr (sizeof(T) == 2) {
        const taser_frag<T> z = taser_load_frag<T>(taser_rest<T>((float*)stats, row, stat_floats) + e, dim - e);
#pragma unroll
        for (int i = 0; i < 8; ++i) t = fmaf((float)x[i] + (float)z[i], (float)y[i], t);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) t = fmaf(x[i], y[i], t);
    }
#pragma unroll
    for (int m = 1; m < 16; m <<= 1) t += __shfl_xor(t, m);
    if (e) return;
    const float top = stats[row * stat_floats], sum = stats[row * stat_floats + 1];
    taser_f4 w;
    w[0] = sum == 0.f ? INFINITY : top;
    w[1] = sum == 0.f ? 0.f : log2f(sum);
    w[2] = t;
    w[3] = 0.f;
    info[row] = w;
}

// ---- dq, dtable -----------------------------------------------------------------------------------------------------------
// A wave owns 32 rows, as in the forward pass; four waves share tiles of 32 states. Bound by registers (queries, their gradients, output: two
// waves a SIMD) and by what the vector units do to scores between products; tiles with several buckets add each dx to its bucket's sum in
// LDS. 2 x 4096 x 4096, 16 heads on 4 of 128, bfloat16: 379 us without a bias, 498 with 32 buckets around distance 0 (405 and 567 in ten
// passes without a pause).
template <typename T, int ND, bool BIAS>
__global__ __launch_bounds__(256, (sizeof(T) == 2 ? 2 : 1)) void attention_grad_queries_kernel(const TaserAttentionArgs a, const taser_f4* info, const T* dout, T* dq,
                                                                                               float* part_dq, float* part_table, int64_t work) {
    constexpr int DP = taser_row_elements(ND), KT = 32, NC = 2 * ND, BYTES = KT * DP * (int)sizeof(T);
    __shared__ __attribute__((aligned(1024))) char k0[BYTES], v0[BYTES], k1[BYTES], v1[BYTES];
    __shared__ int64_t pos0[BIAS ? KT : 1], pos1[BIAS ? KT : 1], ranges[4][2];
    __shared__ uint8_t near[BIAS ? kTaserNear : 1];
    __shared__ float table[BIAS ? TASER_MAX_GROUP_BUCKETS : 1];                             // [buckets][group]
    __shared__ float table_sums[BIAS ? 4 : 1][BIAS ? TASER_MAX_BUCKETS : 1][32];             // of dx, by a wave's buckets and rows
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int64_t item = taser_stretch_of_work(blockIdx.x, work);
    if (item < 0) return;
    const int row_tile = (int)(item % a.row_tiles), split = (int)(item / a.row_tiles % a.splits);
    const int64_t pair = item / a.row_tiles / a.splits;
    const int hk = (int)(pair % a.kv_heads), b = (int)(pair / a.kv_heads);
    const int32_t length = taser_length(a, b);
    const int all_tiles = (length + KT - 1) / KT, each = (all_tiles + a.splits - 1) / a.splits;
    const int first = split * each, last = first + each < all_tiles ? first + each : all_tiles;

    const int row = row_tile * 128 + wave * 32 + (lane & 31);
    const bool real = row < a.rows;
    const int query = real ? row / a.group : 0, g = real ? row - query * a.group : 0, head = hk * a.group + g;
    const int64_t at_row = ((int64_t)b * a.queries + query) * a.heads + head;
    taser_frag<T> q[NC], dy[NC];
    {
        const T *from = (const T*)a.q + b * a.q_batch + query * a.q_token + head * a.q_head, *dfrom = dout + at_row * a.dim;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int e = 16 * c + 8 * half, n = real ? a.dim - e : 0;
            q[c] = taser_load_frag<T>(from + e, n);
            dy[c] = taser_load_frag<T>(dfrom + e, n);
        }
    }
    taser_f4 mine = {INFINITY, 0.f, 0.f, 0.f};
    if (real) mine = info[at_row];
    if (mine[0] == INFINITY && mine[1] == 0.f) {   // a row without states: whatever comes back to it
        mine[2] = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c) dy[c] = taser_frag<T>{};
    }
    int64_t query_pos = 0, bound = 0, query_low = 0, query_high = 0;
    uint64_t foldable = 0;
    TaserNear map;
    if constexpr (BIAS) {
        const T* from = (const T*)a.table + (int64_t)hk * a.group * a.buckets;
        for (int i = threadIdx.x; i < a.group * a.buckets; i += 256) table[i] = (float)from[i % a.group * a.buckets + i / a.group];
        for (int i = threadIdx.x; i < 4 * TASER_MAX_BUCKETS * 32; i += 256) (&table_sums[0][0][0])[i] = 0.f;
        query_pos = a.query_pos[b * a.query_pos_batch + (row < a.rows ? row : a.rows - 1) / a.group];
        bound = taser_lane_bound(a, lane);
        taser_range(query_pos, true, &query_low, &query_high);
        map = TaserNear(bound, a.buckets, near);
        __syncthreads();
        foldable = taser_foldable(table, a.buckets, a.group, lane);
    }
    const float* my_table = table + g;   // by bucket, `group` apart
    float (*my_sums)[32] = table_sums[wave];
    const T* const k_from = (const T*)a.k + b * a.k_batch + hk * a.k_head;
    const T* const v_from = (const T*)a.v + b * a.v_batch + hk * a.v_head;

    // A lane's mask byte of a tile's states is on its way a tile ahead, their positions are two tiles ahead (as in the forward pass).
    uint8_t ahead_mask = 1;
    int64_t next_pos = 0, after_pos = 0;
    auto state_pos = [&](int tile) -> int64_t {
        const int64_t at = (int64_t)tile * KT + lane;
        return BIAS && wave == 0 && lane < KT && at < length ? a.key_pos[b * a.key_pos_batch + at] : 0;
    };
    auto look = [&](int tile) {
        const int64_t at = (int64_t)tile * KT + lane;
        if (a.mask) ahead_mask = lane < KT && at < length ? a.mask[b * a.mask_batch + at] : 0;
    };
    auto kept = [&](int tile) -> uint32_t {
        const int n = length - tile * KT;
        uint32_t keep = n >= 32 ? ~0u : (1u << n) - 1;
        if (a.mask) keep &= (uint32_t)__ballot(ahead_mask != 0);
        return keep;
    };
    TaserTileLoader<T, DP, KT, 256> load_k(threadIdx.x, a.dim, a.direct), load_v(threadIdx.x, a.dim, a.direct);
    load_k.set([&](int r) { return r * a.k_token; });
    load_v.set([&](int r) { return r * a.v_token; });
    auto fetch = [&](char* k, char* v, int64_t* pos, int tile, uint32_t keep) {
        const int64_t at = (int64_t)tile * KT;
        const int n = length - tile * KT < KT ? length - tile * KT : KT, size = (int)sizeof(T);
        load_k.load(k, k_from + at * a.k_token, taser_span(n, a.k_token * size, a.dim * size), keep, a.mask, [&](int r) { return r * a.k_token; });
        load_v.load(v, v_from + at * a.v_token, taser_span(n, a.v_token * size, a.dim * size), keep, a.mask, [&](int r) { return r * a.v_token; });
        if constexpr (BIAS)
            if (wave == 0 && lane < KT) pos[lane] = next_pos;
    };

    const TaserRowsAt<T, DP> rows_at(lane);
    const TaserColumnsAt<T, DP> columns_at(lane);
    taser_f16 acc[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[d][r] = 0.f;
    const float scale2 = a.scale * kLog2e;
    constexpr bool LIFTED = taser_lifted<T>;
    float lift = LIFTED ? kTaserFirstLift : 1.f;   // of the row's dx and sums

    // As in the forward pass: one bias for the tile goes into the row's constant, others into the scores.
    float tile_bias = 0.f;
    bool tile_sums = false;
    int tile_low = 0, tile_high = 0;
    auto prepare = [&](int turn) {
        const int64_t* range = ranges[turn & 3];
        tile_low = taser_uniform_bucket(bound, taser_apart(query_low, range[1]), a.buckets);
        tile_high = taser_uniform_bucket(bound, taser_apart(query_high, range[0]), a.buckets);
        tile_sums = tile_low != tile_high || !((foldable >> tile_low) & 1);
        tile_bias = my_table[tile_low * a.group];
    };
    auto compute = [&](const char* k, const char* v, const int64_t* pos, int turn, uint32_t keep) {
        float bias = tile_bias, by = scale2, minus = mine[0];
        const bool sums = tile_sums;
        const int low = tile_low, high = tile_high;
        if constexpr (BIAS) prepare(turn + 1);
        if (!keep) return;
        float sum_before = 0.f;
        if constexpr (BIAS) sum_before = my_sums[low][lane & 31];
        taser_f16 s, dp;
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r] = dp[r] = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            taser_mma(s, rows_at.operand(k, 0, c), q[c]);
            taser_mma(dp, rows_at.operand(v, 0, c), dy[c]);
        }
        if constexpr (sizeof(T) == 2) taser_order<6, 1, 2 * NC>();
        if constexpr (BIAS) {
            if (sums) {
                const int64_t* range = ranges[turn & 3];
                const TaserBuckets of(map, near, bound, low, high, taser_apart(query_low, range[1]), taser_apart(query_high, range[0]));
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    int bucket[4];
                    of.find<false>(bucket, query_pos, pos + 8 * j + 4 * half);
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[4 * j + i] = fmaf(s[4 * j + i], a.scale, my_table[bucket[i] * a.group]) - mine[0];
                }
                bias = minus = 0.f;
                by = kLog2e;
            }
        }
        const float plus = fmaf(bias - minus, kLog2e, -mine[1]);
        if (keep != ~0u) {
            uint32_t bits = keep >> (4 * half);
            asm volatile("" : "+v"(bits));   // keeps this a branch: most tiles are whole
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (!((bits >> (8 * (r >> 2) + (r & 3))) & 1)) s[r] = -INFINITY;
        }
        const float less = LIFTED ? mine[2] * lift : mine[2];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float p = __builtin_amdgcn_exp2f(fmaf(s[r], by, plus));
            s[r] = p * (LIFTED ? fmaf(dp[r], lift, -less) : dp[r] - less);
        }
        if constexpr (LIFTED) {
            float most = fabsf(s[0]);
#pragma unroll
            for (int r = 1; r < 16; ++r) most = fmaxf(most, fabsf(s[r]));
            most = taser_halves_max(most);
            if (__any(most >= kTaserMostLifted)) {
                const float again = most >= kTaserMostLifted ? taser_relift(most) : 1.f;
                lift *= again;
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] *= again;
#pragma unroll
                for (int d = 0; d < ND; ++d)
#pragma unroll
                    for (int r = 0; r < 16; ++r) acc[d][r] *= again;
            }
        }
        const float down = LIFTED ? taser_unlift(lift) : 1.f;
        if constexpr (BIAS) {
            if (low != high) {   // a row's two lanes add one after the other: the sums have one order
                const int64_t* range = ranges[turn & 3];
                const TaserBuckets of(map, near, bound, low, high, taser_apart(query_low, range[1]), taser_apart(query_high, range[0]));
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    int bucket[4];
                    of.find<false>(bucket, query_pos, pos + 8 * j + 4 * half);
                    // Four at a time: what has a later one's bucket is added to that one, whose write comes after its own.
                    float x[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        x[i] = s[4 * j + i];
#pragma unroll
                        for (int e = 0; e < i; ++e) x[i] += bucket[e] == bucket[i] ? s[4 * j + e] : 0.f;
                    }
#pragma unroll
                    for (int side = 0; side < 2; ++side) {
                        if (half == side) {
                            float y[4];
#pragma unroll
                            for (int i = 0; i < 4; ++i) y[i] = my_sums[bucket[i]][lane & 31];
#pragma unroll
                            for (int i = 0; i < 4; ++i) my_sums[bucket[i]][lane & 31] = y[i] + x[i] * down;
                        }
                        taser_next_turn();
                    }
                }
            } else {
                float x = 0.f;
#pragma unroll
                for (int r = 0; r < 16; ++r) x += s[r];
                x = taser_halves_sum(x);
                if (half == 0) my_sums[low][lane] = sum_before + x * down;
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const taser_frag<T> x = taser_operand<T>(s, h);
#pragma unroll
            for (int d = 0; d < ND; ++d) taser_mma(acc[d], columns_at.operand(k, 16 * h, d), x);
        }
    };

    int tile = first;
    uint32_t keep0 = 0, keep1 = 0;
    auto store_range = [&](int64_t pos, int at, int turn) {
        if (wave == 0) taser_store_range(pos, lane < KT && (int64_t)at * KT + lane < length, lane, ranges[turn & 3]);
    };
    auto open = [&](char* k, char* v, int64_t* pos, int at, int turn, uint32_t& keep) {
        if (at >= last) return;
        keep = kept(at);
        fetch(k, v, pos, at, keep);
        look(at + 1);
        if constexpr (BIAS) {
            store_range(after_pos, at + 1, turn + 1);
            next_pos = after_pos;
            after_pos = state_pos(at + 2);
        }
    };
    look(tile);
    int turn = 0;
    if constexpr (BIAS) {
        next_pos = state_pos(tile);
        after_pos = state_pos(tile + 1);
        store_range(next_pos, tile, 0);
    }
    open(k0, v0, pos0, tile, 0, keep0);
    for (; tile < last; tile += 2, turn += 2) {
        taser_loads_arrived();
        __syncthreads();
        if constexpr (BIAS)
            if (turn == 0) prepare(0);
        open(k1, v1, pos1, tile + 1, turn + 1, keep1);
        compute(k0, v0, pos0, turn, keep0);
        if (tile + 1 >= last) break;
        taser_loads_arrived();
        __syncthreads();
        open(k0, v0, pos0, tile + 2, turn + 2, keep0);
        compute(k1, v1, pos1, turn + 1, keep1);
    }

    if constexpr (BIAS) {
        __syncthreads();
        float* to = part_table + item * (a.group * taser_padded(a.buckets));
        const int rows = a.rows - row_tile * 128 < 128 ? a.rows - row_tile * 128 : 128;
        for (int i = threadIdx.x; i < a.group * a.buckets; i += 256) {
            const int of = i / a.buckets, u = i - of * a.buckets;
            int r = (int)((of + a.group - (int64_t)row_tile * 128 % a.group) % a.group);   // the first row of this tile with that head
            float x = 0.f;
            for (; r < rows; r += a.group) x += table_sums[r >> 5][u][r & 31];
            to[of * taser_padded(a.buckets) + u] = x;
        }
    }
    if (!real) return;
    float* part = part_dq ? part_dq + (split * (int64_t)a.batch * a.queries * a.heads + at_row) * a.dim : nullptr;
    T* to = dq + at_row * a.dim;
    const float back = LIFTED ? a.scale * taser_unlift(lift) : a.scale;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int e = 32 * d + 8 * j + 4 * half;
            T x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float y = acc[d][4 * j + i] * back;
                x[i] = (T)y;
                if (part && e + i < a.dim) part[e + i] = y;
            }
            if (part) continue;
            taser_store(to + e, a.dim - e, x);
        }
}

// ---- dk, dv ---------------------------------------------------------------------------------------------------------------
// Two waves own 32 states (lane l: state l % 32), four such pairs share tiles of 64 rows (32 in single precision). The first of a pair
// has the keys in registers: scores, weights, dv. The second has the values: dp, dx, dk; the weights come to it through LDS. Each of a
// tile's two steps is as many products for the one as for the other, and neither holds more than half of the sums: a wave with both
// has too many registers for a second one on its SIMD (measured: 610 TFLOP/s so at 2 x 4096 x 4096, 16 heads of 128). Rows of all query
// heads of the key head pass by, so shared heads' gradients are whole. The size above: 589 us without a bias, 629 with (664 and 729 in ten
// passes without a pause; matrix cores 0.37 busy). Registers are spilled here: 13 in 16 bits, heads of 97 to 128 elements, with a bias; 31 in
// single precision, with a bias 55; and where heads have up to 64 elements 10, with a bias 103 to 128, since four waves a SIMD leave 128
// registers: the size above with heads of 64 takes 334 us without a bias, 585 with.
template <typename T, int ND, bool BIAS>
__global__ __launch_bounds__(512, (ND <= 2 && sizeof(T) == 2 ? 4 : 2)) void attention_grad_states_kernel(const TaserAttentionArgs a, const taser_f4* info, const T* dout, T* dk, T* dv, float* part_dk,
                                                                    float* part_dv, int64_t work) {
    constexpr int DP = taser_row_elements(ND), RT = sizeof(T) == 2 ? 64 : 32, NS = RT / 32, NC = 2 * ND, BYTES = RT * DP * (int)sizeof(T);
    __shared__ __attribute__((aligned(1024))) char q0[BYTES], y0[BYTES], q1[BYTES], y1[BYTES];
    __shared__ taser_f4 passed[4][NS][4][64];                 // a pair's weights, by registers and lane
    __shared__ taser_f4 info0[3][RT / 4], info1[3][RT / 4];   // a kind of number of 4 rows
    __shared__ taser_f4 constants[BIAS ? 4 : 1][2][RT / 4];   // a pair's: what the exponents of 4 rows get added, of this tile and the next
    __shared__ int64_t pos0[BIAS ? RT : 1], pos1[BIAS ? RT : 1], range0[NS][2], range1[NS][2];
    __shared__ int at0[BIAS ? RT : 1], at1[BIAS ? RT : 1];    // a row's place in the table
    __shared__ uint8_t near[BIAS ? kTaserNear : 1];
    __shared__ float table[BIAS ? TASER_MAX_GROUP_BUCKETS : 1];   // [buckets][group]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, pair = wave & 3;
    const bool second = wave >= 4;
    const int64_t item = taser_stretch_of_work(blockIdx.x, work);
    if (item < 0) return;
    const int state_tile = (int)(item % a.row_tiles), split = (int)(item / a.row_tiles % a.splits);
    const int64_t head_of = item / a.row_tiles / a.splits;
    const int hk = (int)(head_of % a.kv_heads), b = (int)(head_of / a.kv_heads);
    const int32_t length = taser_length(a, b);
    const int all_tiles = state_tile * 128 < length ? (a.rows + RT - 1) / RT : 0, each = (all_tiles + a.splits - 1) / a.splits;
    const int first = split * each, last = first + each < all_tiles ? first + each : all_tiles;

    const int state = state_tile * 128 + pair * 32 + (lane & 31);
    const bool real = state < length && (!a.mask || a.mask[b * a.mask_batch + state]);
    taser_frag<T> own[NC];   // the states' keys, or values
    {
        const int64_t at = real ? state : 0;
        const T* from = second ? (const T*)a.v + b * a.v_batch + hk * a.v_head + at * a.v_token : (const T*)a.k + b * a.k_batch + hk * a.k_head + at * a.k_token;
#pragma unroll
        for (int c = 0; c < NC; ++c) own[c] = taser_load_frag<T>(from + 16 * c + 8 * half, real ? a.dim - 16 * c - 8 * half : 0);
    }
    int64_t key_pos = 0, bound = 0, key_low = 0, key_high = 0;
    uint64_t foldable = 0;
    TaserNear map;
    if constexpr (BIAS) {
        const T* from = (const T*)a.table + (int64_t)hk * a.group * a.buckets;
        for (int i = threadIdx.x; i < a.group * a.buckets; i += 512) table[i] = (float)from[i % a.group * a.buckets + i / a.group];
        key_pos = real ? a.key_pos[b * a.key_pos_batch + state] : 0;
        bound = taser_lane_bound(a, lane);
        taser_range(key_pos, real, &key_low, &key_high);
        map = TaserNear(bound, a.buckets, near);
        __syncthreads();
        foldable = taser_foldable(table, a.buckets, a.group, lane);
    }
    const bool any = __any(real);
    const T* const q_from = (const T*)a.q + b * a.q_batch + (int64_t)hk * a.group * a.q_head;
    const T* const y_from = dout + ((int64_t)b * a.queries * a.heads + hk * a.group) * a.dim;
    const int64_t y_token = (int64_t)a.heads * a.dim;
    // Where the heads of a query end with a tile, rows have the same places in every tile.
    const bool even = RT % a.group == 0;
    TaserTileLoader<T, DP, RT, 512> load_q(threadIdx.x, a.dim, a.direct), load_y(threadIdx.x, a.dim, a.direct);
    // What one wave writes down of a tile's rows, a lane a row, is on its way a tile ahead.
    taser_f4 ahead_info = {INFINITY, 0.f, 0.f, 0.f};
    int64_t ahead_pos = 0;
    int ahead_head = 0;
    auto look = [&](int tile) {
        if (wave != 4) return;
        const int64_t at = (int64_t)tile * RT + lane;
        const bool there = lane < RT && at < a.rows;
        const int row = there ? (int)at : 0, query = row / a.group, g = row - query * a.group;
        taser_f4 w = {INFINITY, 0.f, 0.f, 0.f};
        if (there) w = info[((int64_t)b * a.queries + query) * a.heads + hk * a.group + g];
        ahead_info = w;
        if constexpr (BIAS) {
            ahead_head = g;
            ahead_pos = there ? a.query_pos[b * a.query_pos_batch + query] : 0;
        }
    };
    auto fetch = [&](char* q, char* y, taser_f4 (*rows_info)[RT / 4], int64_t* pos, int64_t (*range)[2], int* in_table, int tile) {
        const int at = tile * RT, n = a.rows - at < RT ? a.rows - at : RT, query0 = at / a.group;
        const uint64_t keep = n >= 64 ? ~0ull : (1ull << n) - 1;
        auto row_at = [&](int64_t token, int64_t head) {
            return [=](int r) -> int64_t {   // past the last row: the last one's place, outside `keep`
                const int row = at + (r < n ? r : n - 1), query = row / a.group;
                return (query - query0) * token + (row - query * a.group) * head;
            };
        };
        const auto q_at = row_at(a.q_token, a.q_head), y_at = row_at(y_token, a.dim);
        if (!even || tile == first || n < RT) {
            load_q.set(q_at);
            load_y.set(y_at);
        }
        load_q.load(q, q_from + query0 * a.q_token, kTaserTileBytes, keep, n < RT, q_at);
        load_y.load(y, y_from + query0 * y_token, kTaserTileBytes, keep, n < RT, y_at);
        if (wave == 4) {
            if (lane < RT)
#pragma unroll
                for (int i = 0; i < 3; ++i) ((float*)rows_info[i])[lane] = i == 0 && !BIAS ? fmaf(-ahead_info[0], kLog2e, -ahead_info[1]) : ahead_info[i];   // (without a bias: the constant itself)
            if constexpr (BIAS) {
                const bool there = lane < n && lane < RT;
                if (lane < RT) {
                    pos[lane] = ahead_pos;
                    in_table[lane] = ahead_head;
                }
                const int64_t low = taser_half_min(there ? ahead_pos : INT64_MAX), high = -taser_half_min(there ? -ahead_pos : INT64_MAX);
                if ((lane & 31) == 0 && lane < RT) {
                    range[lane >> 5][0] = low;
                    range[lane >> 5][1] = high;
                }
            }
        }
    };

    // Weights are at most 1: in half precision they are 2^14 times as large where dv's product takes them. dx has a factor a state.
    constexpr bool LIFTED = taser_lifted<T>;
    float lift = !LIFTED ? 1.f : second ? kTaserFirstLift : 0x1p14f;
    const TaserRowsAt<T, DP> rows_at(lane);
    const TaserColumnsAt<T, DP> columns_at(lane);
    taser_f16 sum[ND];   // of dv, or dk
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) sum[d][r] = 0.f;
    const float scale2 = a.scale * kLog2e;
    taser_f16 x[NS];     // scores, then weights; or dp, then dx

    // As in the forward pass: one bias for the tile goes into the rows' constants, others into the scores. Which it is, and the constants,
    // are found a tile ahead, under the products of the step before.
    int low[NS], high[NS];
    bool sums = false;
    auto prepare = [&](const taser_f4 (*rows_info)[RT / 4], const int64_t (*range)[2], const int* in_table, int turn) {
        bool one = true;
#pragma unroll
        for (int n = 0; n < NS; ++n) {
            low[n] = taser_uniform_bucket(bound, taser_apart(range[n][0], key_high), a.buckets);
            high[n] = taser_uniform_bucket(bound, taser_apart(range[n][1], key_low), a.buckets);
            one = one && low[n] == high[n] && (foldable >> low[n]) & 1;
        }
        sums = !one;
        float bias = 0.f, top = 0.f, log_sum = 0.f;
        if (lane < RT) {   // a lane a row
            bias = table[low[lane >> 5 < NS ? lane >> 5 : 0] * a.group + in_table[lane]];
            top = ((const float*)rows_info[0])[lane];
            log_sum = ((const float*)rows_info[1])[lane];
        }
        if (lane < RT) ((float*)constants[pair][turn & 1])[lane] = fmaf(sums ? 0.f : bias - top, kLog2e, -log_sum);
    };
    // First step: the scores and their weights, or dp.
    auto begin = [&](const char* q, const char* y, const taser_f4 (*rows_info)[RT / 4], const int64_t* pos, const int64_t (*range)[2], const int* in_table, int turn) {
        if (second) {
#pragma unroll
            for (int n = 0; n < NS; ++n) {
#pragma unroll
                for (int r = 0; r < 16; ++r) x[n][r] = 0.f;
#pragma unroll
                for (int c = 0; c < NC; ++c) taser_mma(x[n], rows_at.operand(y, 32 * n, c), own[c]);
            }
            if constexpr (sizeof(T) == 2) taser_order<8, 1, NS * NC>();
            return;
        }
        const float by = BIAS && sums ? kLog2e : scale2;
        const taser_f4* plus = BIAS ? constants[pair][turn & 1] : rows_info[0];
#pragma unroll
        for (int n = 0; n < NS; ++n) {
#pragma unroll
            for (int r = 0; r < 16; ++r) x[n][r] = 0.f;
#pragma unroll
            for (int c = 0; c < NC; ++c) taser_mma(x[n], rows_at.operand(q, 32 * n, c), own[c]);
        }
        if constexpr (BIAS) {
            if (sums) {
#pragma unroll
                for (int n = 0; n < NS; ++n) {
                    const TaserBuckets of(map, near, bound, low[n], high[n], taser_apart(range[n][0], key_high), taser_apart(range[n][1], key_low));
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        int bucket[4];
                        const int row = 32 * n + 8 * j + 4 * half;
                        of.find<true>(bucket, key_pos, pos + row);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            x[n][4 * j + i] = fmaf(x[n][4 * j + i], a.scale, table[bucket[i] * a.group + in_table[row + i]]) - ((const float*)rows_info[0])[row + i];
                    }
                }
            }
        }
#pragma unroll
        for (int n = 0; n < NS; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const taser_f4 more = plus[8 * n + 2 * j + half];
                taser_f4 w;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    w[i] = __builtin_amdgcn_exp2f(fmaf(x[n][4 * j + i], by, more[i]));
                    if (!real) w[i] = 0.f;
                    x[n][4 * j + i] = w[i];
                }
                passed[pair][n][j][lane] = w;
            }
    };
    // Second step: dv, or dx and dk.
    auto end = [&](const char* q, const char* y, const taser_f4 (*rows_info)[RT / 4]) {
        if (second) {
#pragma unroll
            for (int n = 0; n < NS; ++n)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const taser_f4 w = passed[pair][n][j][lane], t = rows_info[2][8 * n + 2 * j + half];
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[n][4 * j + i] = w[i] * (x[n][4 * j + i] - t[i]);
                }
            if constexpr (LIFTED) {
                float most = 0.f;
#pragma unroll
                for (int n = 0; n < NS; ++n)
#pragma unroll
                    for (int r = 0; r < 16; ++r) most = fmaxf(most, fabsf(x[n][r]));
                most = taser_halves_max(most);
                if (__any(most * lift >= kTaserMostLifted)) {
                    const float before = lift;
                    if (most * lift >= kTaserMostLifted) lift = taser_relift(most);
                    const float again = lift * taser_unlift(before);
#pragma unroll
                    for (int d = 0; d < ND; ++d)
#pragma unroll
                        for (int r = 0; r < 16; ++r) sum[d][r] *= again;
                }
            }
        }
        const char* from = second ? q : y;
#pragma unroll
        for (int n = 0; n < NS; ++n)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const taser_frag<T> w = taser_operand<T>(x[n], h, lift);
#pragma unroll
                for (int d = 0; d < ND; ++d) taser_mma(sum[d], columns_at.operand(from, 32 * n + 16 * h, d), w);
            }
    };

    int tile = first;
    auto open = [&](char* q, char* y, taser_f4 (*rows_info)[RT / 4], int64_t* pos, int64_t (*range)[2], int* in_table, int at) {
        if (at >= last) return;
        fetch(q, y, rows_info, pos, range, in_table, at);
        look(at + 1);
    };
    look(tile);
    open(q0, y0, info0, pos0, range0, at0, tile);
    for (int turn = 0; tile < last; tile += 2, turn += 2) {
        taser_loads_arrived();
        __syncthreads();
        if constexpr (BIAS)
            if (turn == 0 && !second) prepare(info0, range0, at0, 0);
        open(q1, y1, info1, pos1, range1, at1, tile + 1);
        if (any) begin(q0, y0, info0, pos0, range0, at0, turn);
        taser_lds_barrier();
        if constexpr (BIAS)
            if (!second && tile + 1 < last) prepare(info1, range1, at1, turn + 1);
        if (any) end(q0, y0, info0);
        if (tile + 1 >= last) break;
        taser_loads_arrived();
        __syncthreads();
        open(q0, y0, info0, pos0, range0, at0, tile + 2);
        if (any) begin(q1, y1, info1, pos1, range1, at1, turn + 1);
        taser_lds_barrier();
        if constexpr (BIAS)
            if (!second && tile + 2 < last) prepare(info0, range0, at0, turn + 2);
        if (any) end(q1, y1, info1);
    }

    if (state >= a.keys) return;
    const int64_t at = (((int64_t)b * a.keys + state) * a.kv_heads + hk) * a.dim, all = (int64_t)a.batch * a.keys * a.kv_heads * a.dim;
    const float by = second ? a.scale * taser_unlift(lift) : taser_unlift(lift);
    T* to = (second ? dk : dv) + at;
    float* part = part_dk ? (second ? part_dk : part_dv) + split * all + at : nullptr;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int e = 32 * d + 8 * j + 4 * half;
            T y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float one = real ? sum[d][4 * j + i] * by : 0.f;   // (a NaN among the queries is no masked state's)
                y[i] = (T)one;
                if (part && e + i < a.dim) part[e + i] = one;
            }
            if (!part) taser_store(to + e, a.dim - e, y);
        }
}

// Adds up parts of up to three gradients, in their order: one launch for all (of 5 us each in a small call).
template <typename T> struct Sums {
    int32_t count = 0, n_parts[3];
    int64_t n[3];
    const float* parts[3];
    T* out[3];
    void add(const float* parts_, int32_t n_parts_, int64_t n_, T* out_) {
        if (!n_) return;
        parts[count] = parts_;
        n_parts[count] = n_parts_;
        n[count] = n_;
        out[count++] = out_;
    }
};
template <typename T> __global__ __launch_bounds__(256) void attention_grad_add_kernel(const Sums<T> sums) {
    const int of = blockIdx.y;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, n = sums.n[of];
    if (i >= n) return;
    const float* parts = sums.parts[of] + i;
    float x = 0.f;
#pragma unroll 4
    for (int p = 0; p < sums.n_parts[of]; ++p) x += parts[p * n];
    sums.out[of][i] = (T)x;
}

// A block has a head, a thread four buckets of a chain of sums: as many chains as there are threads, then the chains in their order.
template <typename T>
__global__ __launch_bounds__(1024) void attention_grad_table_kernel(const float* parts, int64_t outer, int64_t inner, int32_t kv_heads, int32_t rows, int32_t group, int32_t buckets, T* dtable) {
    __shared__ taser_f4 sums[1024];
    const int head = blockIdx.x, hk = head / group, g = head - hk * group, width = taser_padded(buckets) / 4, chains = 1024 / width, chain = threadIdx.x / width, u = threadIdx.x % width;
    taser_f4 x = {0.f, 0.f, 0.f, 0.f};
    if (chain < chains) {
#pragma unroll 4
        for (int64_t i = chain; i < outer * inner; i += chains) {
            const taser_f4* from = (const taser_f4*)parts + ((i / inner * kv_heads + hk) * inner + i % inner) * rows * width + u;
            for (int r = g; r < rows; r += group) x += from[r * width];
        }
    }
    sums[threadIdx.x] = x;
    __syncthreads();
    // 16 chains of chains, then those
    if (chain < 16) {
        x = taser_f4{0.f, 0.f, 0.f, 0.f};
        for (int c = chain; c < chains; c += 16) x += sums[c * width + u];
    }
    __syncthreads();
    if (chain < 16) sums[threadIdx.x] = x;
    __syncthreads();
    if (chain) return;
    x = taser_f4{0.f, 0.f, 0.f, 0.f};
    for (int c = 0; c < 16; ++c) x += sums[c * width + u];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (4 * u + i < buckets) dtable[(int64_t)head * buckets + 4 * u + i] = (T)x[i];
}

struct Plan {
    int row_tiles, row_splits, state_tiles, state_splits;   // row_splits: parts of the states that a tile of rows goes over, and the other way round
    uint64_t info, dq, dk, dv, table, bytes;                // places in the workspace
};

Plan plan(const TaserAttentionArgs& a, int32_t type) {
    Plan p = {};
    const int64_t pairs = (int64_t)a.batch * a.kv_heads;
    p.row_tiles = (int)(((int64_t)a.rows + 127) / 128);
    p.state_tiles = (int)(((int64_t)a.keys + 127) / 128);
    const int64_t rows_bytes = pairs * a.rows * a.dim * 4, states_bytes = 2 * pairs * a.keys * a.dim * 4;
    const double tile = (a.dim <= 64 ? 0.5 : a.dim <= 96 ? 0.75 : 1.) * (type == TASER_F32 ? 11. : 1.5);   // us of 32 states, or rows, for a block (measured)
    p.row_splits = taser_splits(pairs * p.row_tiles, type == TASER_F32 ? 256 : 512, (a.keys + 31) / 32, tile, rows_bytes);
    p.state_splits = taser_splits(pairs * p.state_tiles, type != TASER_F32 && a.dim <= 64 ? 512 : 256, (a.rows + 31) / 32, tile, states_bytes);
    auto take = [&](uint64_t bytes) {
        const uint64_t at = p.bytes;
        p.bytes += (bytes + 255) / 256 * 256;
        return at;
    };
    const uint64_t rows = (uint64_t)a.batch * a.queries * a.heads, states = (uint64_t)a.batch * a.keys * a.kv_heads * a.dim;
    p.info = take(rows * 16);
    p.dq = take(p.row_splits > 1 ? p.row_splits * rows * a.dim * 4 : 0);
    p.dk = take(p.state_splits > 1 ? p.state_splits * states * 4 : 0);
    p.dv = take(p.state_splits > 1 ? p.state_splits * states * 4 : 0);
    p.table = take(a.table ? (uint64_t)pairs * p.row_tiles * p.row_splits * a.group * taser_padded(a.buckets) * 4 : 0);
    return p;
}

// Of the kernels over tiles, those of launch(); the table's has a block of 1024 a head.
bool launches_fit(const TaserAttentionArgs& a, const Plan& p) {
    const int64_t pairs = (int64_t)a.batch * a.kv_heads, rows = (int64_t)a.batch * a.queries * a.heads, states = pairs * a.keys * a.dim;
    return taser_launch_fits((rows + 15) / 16, 256) && taser_launch_fits(taser_stretched_grid(pairs * p.row_tiles * p.row_splits), 256) &&
           taser_launch_fits(taser_stretched_grid(pairs * p.state_tiles * p.state_splits), 512) &&
           (p.row_splits == 1 || taser_launch_fits((rows * a.dim + 255) / 256, 256)) && (p.state_splits == 1 || taser_launch_fits((states + 255) / 256, 256));
}

template <typename T, int ND>
int launch(TaserAttentionArgs& a, const Plan& p, const T* out, const float* stats, const T* dout, T* dq, T* dk, T* dv, T* dtable, char* work, hipStream_t stream) {
    const int64_t rows = (int64_t)a.batch * a.queries * a.heads, states = (int64_t)a.batch * a.keys * a.kv_heads * a.dim, pairs = (int64_t)a.batch * a.kv_heads;
    taser_f4* info = (taser_f4*)(work + p.info);
    Sums<T> sums;
    if (rows) {
        TaserProfileSpan span(stream, "attention_grad_rows");
        attention_grad_rows_kernel<T><<<dim3((unsigned)((rows + 15) / 16)), 256, 0, stream>>>(out, dout, stats, a.stat_floats, rows, a.dim, info);
        TASER_HIP_TRY(hipGetLastError());
    }
    float* part_table = (float*)(work + p.table);
    if (rows) {
        a.row_tiles = p.row_tiles;
        a.splits = p.row_splits;
        float* part = p.row_splits > 1 ? (float*)(work + p.dq) : nullptr;
        const int64_t items = pairs * p.row_tiles * p.row_splits;
        const dim3 grid((unsigned)taser_stretched_grid(items));
        {
            TaserProfileSpan span(stream, "attention_grad_queries");
            if (a.table)
                attention_grad_queries_kernel<T, ND, true><<<grid, 256, 0, stream>>>(a, info, dout, dq, part, part_table, items);
            else
                attention_grad_queries_kernel<T, ND, false><<<grid, 256, 0, stream>>>(a, info, dout, dq, part, part_table, items);
            TASER_HIP_TRY(hipGetLastError());
        }
        if (part) sums.add(part, p.row_splits, rows * a.dim, dq);
    }
    if (a.table) {
        const int32_t type = std::is_same_v<T, float> ? TASER_F32 : std::is_same_v<T, _Float16> ? TASER_F16 : TASER_BF16;
        if (const int rc = taser_add_tables(part_table, rows ? a.batch : 0, (int64_t)p.row_tiles * p.row_splits, a.kv_heads, a.group, a.group, a.buckets, type, dtable, stream)) return rc;
    }
    if (states) {
        a.row_tiles = p.state_tiles;
        a.splits = p.state_splits;
        float* part = p.state_splits > 1 ? (float*)(work + p.dk) : nullptr;
        float* part_v = p.state_splits > 1 ? (float*)(work + p.dv) : nullptr;
        const int64_t items = pairs * p.state_tiles * p.state_splits;
        const dim3 grid((unsigned)taser_stretched_grid(items));
        // rows are loaded here: q and dout have to be aligned for loads past the registers
        const int whole = 16 / (int)sizeof(T);
        a.direct = a.dim % whole == 0 && ((uintptr_t)a.q | (uintptr_t)dout) % 16 == 0 && a.q_batch % whole == 0 && a.q_token % whole == 0 && a.q_head % whole == 0;
        // the rows of a tile within the reach of its descriptor
        const int64_t reach = kTaserTileBytes / 64 / (int)sizeof(T);
        a.direct = a.direct && a.q_token >= 0 && a.q_head >= 0 && a.q_token < reach && a.q_head < reach / a.group && (int64_t)a.heads * a.dim < reach;
        {
            TaserProfileSpan span(stream, "attention_grad_states");
            if (a.table)
                attention_grad_states_kernel<T, ND, true><<<grid, 512, 0, stream>>>(a, info, dout, dk, dv, part, part_v, items);
            else
                attention_grad_states_kernel<T, ND, false><<<grid, 512, 0, stream>>>(a, info, dout, dk, dv, part, part_v, items);
            TASER_HIP_TRY(hipGetLastError());
        }
        if (part) {
            sums.add(part, p.state_splits, states, dk);
            sums.add(part_v, p.state_splits, states, dv);
        }
    }
    if (sums.count) {
        int64_t most = 0;
        for (int i = 0; i < sums.count; ++i) most = sums.n[i] > most ? sums.n[i] : most;
        TaserProfileSpan span(stream, "attention_grad_add");
        attention_grad_add_kernel<T><<<dim3((unsigned)((most + 255) / 256), (unsigned)sums.count), 256, 0, stream>>>(sums);
        TASER_HIP_TRY(hipGetLastError());
    }
    return TASER_OK;
}

template <typename T>
int launch_typed(TaserAttentionArgs& a, const Plan& p, const void* out, const float* stats, const void* dout, void* dq, void* dk, void* dv, void* dtable, char* work, hipStream_t stream) {
    if (a.dim <= 64) return launch<T, 2>(a, p, (const T*)out, stats, (const T*)dout, (T*)dq, (T*)dk, (T*)dv, (T*)dtable, work, stream);
    if (a.dim <= 96) return launch<T, 3>(a, p, (const T*)out, stats, (const T*)dout, (T*)dq, (T*)dk, (T*)dv, (T*)dtable, work, stream);
    return launch<T, 4>(a, p, (const T*)out, stats, (const T*)dout, (T*)dq, (T*)dk, (T*)dv, (T*)dtable, work, stream);
}

}  // namespace

int taser_add_tables(const float* parts, int64_t outer, int64_t inner, int32_t kv_heads, int32_t rows, int32_t group, int32_t buckets, int32_t type, void* dtable, hipStream_t stream) {
    TaserProfileSpan span(stream, "attention_grad_table");
    const dim3 grid((unsigned)(kv_heads * group));
    if (type == TASER_F32) attention_grad_table_kernel<float><<<grid, 1024, 0, stream>>>(parts, outer, inner, kv_heads, rows, group, buckets, (float*)dtable);
    else if (type == TASER_F16) attention_grad_table_kernel<_Float16><<<grid, 1024, 0, stream>>>(parts, outer, inner, kv_heads, rows, group, buckets, (_Float16*)dtable);
    else attention_grad_table_kernel<__bf16><<<grid, 1024, 0, stream>>>(parts, outer, inner, kv_heads, rows, group, buckets, (__bf16*)dtable);
    TASER_HIP_TRY(hipGetLastError());
    return TASER_OK;
}

// Windows go their own way where there is anything to do.
static bool window(const TaserAttentionArgs& a) { return taser_window_fits(a) && a.batch && a.queries; }

uint64_t taser_attention_grad_bytes(const TaserAttentionArgs& a, int32_t type) { return window(a) ? taser_window_grad_bytes(a) : plan(a, type).bytes; }

extern "C" int taser_cross_attention_grad(const taser_attention* arg, const void* out, const float* stats, const void* dout, void* dq, void* dk, void* dv, void* dtable, void* work,
                                          uint64_t work_size, void* hip_stream) {
    TaserAttentionArgs a;
    if (const int rc = taser_attention_args(arg, "cross_attention_grad", &a)) return rc;
    const bool rows = a.batch && a.queries, states = a.batch && a.keys;
    if (rows && (!out || !stats || !dout || !dq)) return taser_fail(TASER_E_ARG, "cross_attention_grad: null output, statistics or gradient of the queries' side");
    if (states && (!dk || !dv)) return taser_fail(TASER_E_ARG, "cross_attention_grad: null gradient of the states");
    if (a.table && !dtable) return taser_fail(TASER_E_ARG, "cross_attention_grad: null gradient of the bias table");
    const Plan p = plan(a, arg->type);
    const uint64_t need = taser_attention_grad_bytes(a, arg->type);
    if (need > work_size)
        return taser_fail(TASER_E_RANGE, "cross_attention_grad: %llu bytes of workspace, %llu needed", (unsigned long long)work_size, (unsigned long long)need);
    if (need && (!work || (uintptr_t)work % 16)) return taser_fail(TASER_E_ARG, "cross_attention_grad: null or misaligned workspace");
    if (!(window(a) || launches_fit(a, p)) || (a.table && !taser_launch_fits(a.heads, 1024)))
        return taser_fail(TASER_E_RANGE, "cross_attention_grad: too many queries, states and batch entries for one launch");
    hipStream_t stream = (hipStream_t)hip_stream;
    taser_clear_stale_hip_error();
    if (window(a)) return taser_window_attention_grad(a, arg->type, stats, dout, dq, dk, dv, dtable, (float*)work, stream);
    if (arg->type == TASER_F32) return launch_typed<float>(a, p, out, stats, dout, dq, dk, dv, dtable, (char*)work, stream);
    if (arg->type == TASER_F16) return launch_typed<_Float16>(a, p, out, stats, dout, dq, dk, dv, dtable, (char*)work, stream);
    return launch_typed<__bf16>(a, p, out, stats, dout, dq, dk, dv, dtable, (char*)work, stream);
}

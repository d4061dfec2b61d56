// Attention to states of another length (taser_cross_attention): one pass over the states with the running maximum and sum of
// a softmax: with m' = max(m, tile's scores), weights exp(x - m'), and sum and output so far times exp(m - m') where m grew.
//
// Few rows: bound by reading the states. 32 single tokens, 8192 states, 32 heads on 8 of 128, bfloat16: 162 us for 806 MB, 5.0 TB/s.
// Many rows: bound by the matrix products and, beside them, the exponentials and reads of LDS that feed them (counters: matrix cores 0.5
// busy, 1.5 LDS instructions a product). 4 x 2048 queries, 2700 to 4050 of 4096 states, 16 heads of 128, bfloat16: 233 us, 885 TFLOP/s, in
// single passes, and 270 - 300 without a pause between them, as all of these products take longer then; 2 x 4096 x 4096 320 - 380 us
// with a bias, 265 - 320 without; float32, 3 x 333 x 777, 6 heads of 80: 36 us.
#include <cmath>
#include <type_traits>

#include "attention.h"

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kMostSplits = 128, kFineStates = 128;

// A wave owns 32 query rows (of the queries of one key head: row r is query r / group, head r % group of them), lane l row
// l % 32 of them. Scores come out transposed, states in registers, so a row's softmax needs one exchange, with the other half of
// the wave, and its weights are an operand as they are. SHARED: the four waves of a block have 32 rows each and share tiles of 64
// states. Else the block has 32 rows and each wave every fourth (second) tile of 32 states, joined at the end: for few rows.
template <typename T, int DP, bool SHARED> struct Shape {
    static constexpr int kWaves = !SHARED && DP * sizeof(T) > 256 ? 2 : 4, kStates = SHARED && sizeof(T) == 2 ? 64 : 32;
    static constexpr int kTileBytes = kStates * DP * (int)sizeof(T), kTiles = SHARED ? 1 : kWaves;   // tiles in LDS at a time, of each of four kinds
    static constexpr int kRows = SHARED ? 32 * kWaves : 32;
};

// FINE: the output is exact to 32 bits before it is rounded. Without it 16-bit weights' roundings are in it (1.4 times as far off as the
// rounded output need be, where they average out over many states) and in the gradient's <dout, out>.
template <typename T, int ND, bool SHARED, bool BIAS, bool FINE>
__global__ __launch_bounds__((64 * Shape<T, taser_row_elements(ND), SHARED>::kWaves), (SHARED && sizeof(T) == 2 && !(FINE && ND > 2) ? 2 : 1)) void attention_kernel(const TaserAttentionArgs a, T* out, float* stats, float* part_out,
                                                                                      float* part_stats, int64_t work) {
    constexpr int DP = taser_row_elements(ND);
    using S = Shape<T, DP, SHARED>;
    constexpr int KT = S::kStates, NK = KT / 32, NC = 2 * ND;
    __shared__ __attribute__((aligned(1024))) char k0[S::kTiles][S::kTileBytes], v0[S::kTiles][S::kTileBytes], k1[S::kTiles][S::kTileBytes], v1[S::kTiles][S::kTileBytes];
    __shared__ int64_t pos0[S::kTiles][BIAS ? KT : 1], pos1[S::kTiles][BIAS ? KT : 1], ranges[S::kTiles][4][2];
    __shared__ float joined[2][S::kWaves][32];
    __shared__ uint8_t near[BIAS && SHARED ? kTaserNear : 1];
    __shared__ float table[BIAS ? TASER_MAX_GROUP_BUCKETS : 1];   // [buckets][group]; of its own, so that no read of it waits for a tile
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int64_t item = taser_stretch_of_work(blockIdx.x, work);
    if (item < 0) return;
    const int row_tile = (int)(item % a.row_tiles), split = (int)(item / a.row_tiles % a.splits);
    const int64_t pair = item / a.row_tiles / a.splits;
    const int hk = (int)(pair % a.kv_heads), b = (int)(pair / a.kv_heads);
    const int32_t length = taser_length(a, b);
    const int all_tiles = (length + KT - 1) / KT, each = (all_tiles + a.splits - 1) / a.splits;
    const int first = split * each, last = first + each < all_tiles ? first + each : all_tiles;

    const int row = row_tile * S::kRows + (SHARED ? wave * 32 : 0) + (lane & 31);
    const bool real = row < a.rows;
    const int query = real ? row / a.group : 0, g = real ? row - query * a.group : 0, head = hk * a.group + g;
    taser_frag<T> q[NC];
    {
        const T* from = (const T*)a.q + b * a.q_batch + query * a.q_token + head * a.q_head;
#pragma unroll
        for (int c = 0; c < NC; ++c) q[c] = taser_load_frag<T>(from + 16 * c + 8 * half, real ? a.dim - 16 * c - 8 * half : 0);
    }
    int64_t query_pos = 0, bound = 0, query_low = 0, query_high = 0;
    uint64_t foldable = 0;
    TaserNear map;
    if constexpr (BIAS) {
        const T* from = (const T*)a.table + (int64_t)hk * a.group * a.buckets;
        for (int i = threadIdx.x; i < a.group * a.buckets; i += blockDim.x) table[i] = (float)from[i % a.group * a.buckets + i / a.group];
        query_pos = a.query_pos[b * a.query_pos_batch + (row < a.rows ? row : a.rows - 1) / a.group];
        bound = taser_lane_bound(a, lane);
        taser_range(query_pos, true, &query_low, &query_high);
        if (SHARED) map = TaserNear(bound, a.buckets, near);   // (a few rows meet few tiles of several buckets: not worth making)
        __syncthreads();
        foldable = taser_foldable(table, a.buckets, a.group, lane);
    }
    const float* my_table = table + g;   // by bucket, `group` apart
    const T* const k_from = (const T*)a.k + b * a.k_batch + hk * a.k_head;
    const T* const v_from = (const T*)a.v + b * a.v_batch + hk * a.v_head;

    // A lane's mask byte of a tile's states is on its way a tile ahead, their positions are two tiles ahead: which buckets a tile can
    // need is known before it begins.
    uint8_t ahead_mask = 1;
    int64_t next_pos = 0, after_pos = 0;
    auto state_pos = [&](int tile) -> int64_t {
        const int64_t at = (int64_t)tile * KT + lane;
        return BIAS && (!SHARED || wave == 0) && lane < KT && at < length ? a.key_pos[b * a.key_pos_batch + at] : 0;
    };
    auto look = [&](int tile) {
        const int64_t at = (int64_t)tile * KT + lane;
        if (a.mask) ahead_mask = lane < KT && at < length ? a.mask[b * a.mask_batch + at] : 0;
    };
    // states [KT * tile, ..) that take part
    auto kept = [&](int tile) -> uint64_t {
        const int n = length - tile * KT;
        uint64_t keep = n >= 64 ? ~0ull : (n <= 0 ? 0 : (1ull << n) - 1);
        if (KT == 32) keep &= 0xffffffffull;
        if (a.mask) keep &= __ballot(ahead_mask != 0);
        return keep;
    };
    constexpr int THREADS = SHARED ? 64 * S::kWaves : 64;
    const int thread = SHARED ? (int)threadIdx.x : lane, slot = SHARED ? 0 : wave;
    TaserTileLoader<T, DP, KT, THREADS> load_k(thread, a.dim, a.direct), load_v(thread, a.dim, a.direct);
    load_k.set([&](int r) { return r * a.k_token; });
    load_v.set([&](int r) { return r * a.v_token; });
    auto fetch = [&](char* k, char* v, int64_t* pos, int tile, uint64_t keep) {
        const int64_t at = (int64_t)tile * KT;
        const int n = length - tile * KT < KT ? length - tile * KT : KT, size = (int)sizeof(T);
        load_k.load(k, k_from + at * a.k_token, taser_span(n, a.k_token * size, a.dim * size), keep, a.mask, [&](int r) { return r * a.k_token; });
        load_v.load(v, v_from + at * a.v_token, taser_span(n, a.v_token * size, a.dim * size), keep, a.mask, [&](int r) { return r * a.v_token; });
        if constexpr (BIAS)
            if ((!SHARED || wave == 0) && lane < KT) pos[lane] = next_pos;
    };

    // Half precision ends at 6e-8 below 1: there the weights, and all sums of them, are 2^10 times as large until the end.
    constexpr float lift = std::is_same_v<T, _Float16> ? 10.f : 0.f, drop = std::is_same_v<T, _Float16> ? 1.f / 1024.f : 1.f;
    // The reference of a row follows its largest score only when that is e^kSlack weights away: most tiles leave the sums as they are.
    constexpr float kSlack = 3.5f;
    const TaserRowsAt<T, DP> rows_at(lane);
    const TaserColumnsAt<T, DP> columns_at(lane);
    float top = -INFINITY, sum = 0.f;
    taser_f16 o[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
    const float scale2 = a.scale * kLog2e;

    // Scores stay products while one bias holds for the whole tile: it goes into the row's constant. Elsewhere, and where a bias is so
    // large that the sum's rounding decides (the lowest value swallows all products), they become sums.
    float tile_bias = 0.f;
    bool tile_sums = false;
    int tile_low = 0, tile_high = 0;
    auto prepare = [&](int turn) {
        const int64_t* range = ranges[slot][turn & 3];
        tile_low = taser_uniform_bucket(bound, taser_apart(query_low, range[1]), a.buckets);
        tile_high = taser_uniform_bucket(bound, taser_apart(query_high, range[0]), a.buckets);
        tile_sums = tile_low != tile_high || !((foldable >> tile_low) & 1);
        tile_bias = tile_sums ? 0.f : my_table[tile_low * a.group];
    };

    auto compute = [&](const char* k, const char* v, const int64_t* pos, int turn, uint64_t keep) {
        float bias = tile_bias;
        const bool sums = tile_sums;
        const int low = tile_low, high = tile_high;
        if constexpr (BIAS) prepare(turn + 1);
        taser_f16 s[NK];
#pragma unroll
        for (int n = 0; n < NK; ++n) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[n][r] = 0.f;
#pragma unroll
            for (int c = 0; c < NC; ++c) taser_mma(s[n], rows_at.operand(k, 32 * n, c), q[c]);
        }
        if constexpr (BIAS) {
            if (sums) {
                const int64_t* range = ranges[slot][turn & 3];
                const TaserBuckets buckets(map, near, bound, low, high, taser_apart(query_low, range[1]), taser_apart(query_high, range[0]));
#pragma unroll
                for (int n = 0; n < NK; ++n)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        int bucket[4];
                        buckets.find<false>(bucket, query_pos, pos + 32 * n + 8 * j + 4 * half);
#pragma unroll
                        for (int i = 0; i < 4; ++i) s[n][4 * j + i] = fmaf(s[n][4 * j + i], a.scale, my_table[bucket[i] * a.group]);
                    }
            }
        }
        if (keep != (KT == 64 ? ~0ull : 0xffffffffull)) {
#pragma unroll
            for (int n = 0; n < NK; ++n) {
                uint32_t bits = (uint32_t)(keep >> (32 * n)) >> (4 * half);
                asm volatile("" : "+v"(bits));   // keeps this a branch: most tiles are whole
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (!((bits >> (8 * (r >> 2) + (r & 3))) & 1)) s[n][r] = -INFINITY;
            }
        }
        float now = s[0][0];
#pragma unroll
        for (int n = 0; n < NK; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) now = fmaxf(now, s[n][r]);
        now = taser_halves_max(now);
        if (!sums) now = fmaf(now, a.scale, bias);
        if (__any(now > top + kSlack)) {
            now = fmaxf(now, top);
            const float shrink = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f((top - now) * kLog2e);
            top = now;
            sum *= shrink;
#pragma unroll
            for (int d = 0; d < ND; ++d)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[d][r] *= shrink;
        }
        const float base = top == -INFINITY ? 0.f : top;
        float by = scale2, plus = fmaf(bias - base, kLog2e, lift);
        if (BIAS && sums) {
#pragma unroll
            for (int n = 0; n < NK; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[n][r] -= base;
            by = kLog2e;
            plus = lift;
        }
        float part = 0.f;
#pragma unroll
        for (int n = 0; n < NK; ++n)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[n][r] = __builtin_amdgcn_exp2f(fmaf(s[n][r], by, plus));
                part += s[n][r];
            }
        sum += part;
        // The weights are rounded to the type of the states that they multiply; their sum is of the unrounded ones. Where FINE, what the
        // rounding took off is multiplied too.
        if constexpr (FINE) {
#pragma unroll
            for (int n = 0; n < NK; ++n)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const taser_frag<T> p = taser_operand<T>(s[n], h);
                    taser_frag<T> q;
#pragma unroll
                    for (int i = 0; i < 8; ++i) q[i] = (T)(s[n][8 * h + i] - (float)p[i]);
#pragma unroll
                    for (int d = 0; d < ND; ++d) {
                        const taser_frag<T> x = columns_at.operand(v, 32 * n + 16 * h, d);
                        taser_mma(o[d], x, p);
                        taser_mma(o[d], x, q);
                    }
                }
        } else {
#pragma unroll
            for (int n = 0; n < NK; ++n)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const taser_frag<T> p = taser_operand<T>(s[n], h);
#pragma unroll
                    for (int d = 0; d < ND; ++d) taser_mma(o[d], columns_at.operand(v, 32 * n + 16 * h, d), p);
                }
        }
    };

    const int step = SHARED ? 1 : S::kWaves;
    int tile = first + (SHARED ? 0 : wave);
    uint64_t keep0 = 0, keep1 = 0;
    auto arrived = [&]() {
        taser_loads_arrived();
        if (SHARED) __syncthreads();
        else __builtin_amdgcn_wave_barrier();
    };
    auto store_range = [&](int64_t pos, int at, int turn) {
        if (!SHARED || wave == 0) taser_store_range(pos, lane < KT && (int64_t)at * KT + lane < length, lane, ranges[slot][turn & 3]);
    };
    auto open = [&](char* k, char* v, int64_t* pos, int at, int turn, uint64_t& keep) {
        if (at >= last) return;
        keep = kept(at);
        fetch(k, v, pos, at, keep);
        look(at + step);
        if constexpr (BIAS) {
            store_range(after_pos, at + step, turn + 1);
            next_pos = after_pos;
            after_pos = state_pos(at + 2 * step);
        }
    };
    look(tile);
    int turn = 0;
    if constexpr (BIAS) {
        next_pos = state_pos(tile);
        after_pos = state_pos(tile + step);
        store_range(next_pos, tile, 0);
    }
    open(k0[slot], v0[slot], pos0[slot], tile, 0, keep0);
    for (; tile < last; tile += 2 * step, turn += 2) {
        arrived();
        if constexpr (BIAS)
            if (turn == 0) prepare(0);
        open(k1[slot], v1[slot], pos1[slot], tile + step, turn + 1, keep1);
        compute(k0[slot], v0[slot], pos0[slot], turn, keep0);
        if (tile + step >= last) break;
        arrived();
        open(k0[slot], v0[slot], pos0[slot], tile + 2 * step, turn + 2, keep0);
        compute(k1[slot], v1[slot], pos1[slot], turn + 1, keep1);
    }

    sum = taser_halves_sum(sum);
    if constexpr (!SHARED) {   // the waves' shares are joined
        constexpr int W = S::kWaves;
        joined[0][wave][lane & 31] = top;
        joined[1][wave][lane & 31] = sum;
        // a wave's sums need twice the bytes of a tile of 16-bit elements
        auto place = [&](int w, int d) -> float* {
            constexpr int FIRST = sizeof(T) == 2 ? ND / 2 : ND;
            return (float*)(d < FIRST ? k0[w] + d * 4096 : k1[w] + (d - FIRST) * 4096);
        };
        taser_loads_arrived();
        __syncthreads();
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) place(wave, d)[64 * r + lane] = o[d][r];
        __syncthreads();
        float best = -INFINITY, by[W];
#pragma unroll
        for (int w = 0; w < W; ++w) best = fmaxf(best, joined[0][w][lane & 31]);
        sum = 0.f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            by[w] = best == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((joined[0][w][lane & 31] - best) * kLog2e);
            sum = fmaf(by[w], joined[1][w][lane & 31], sum);
        }
        top = best;
#pragma unroll
        for (int d = 0; d < ND; ++d) {
            if (d % W != wave) continue;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                float x = 0.f;
#pragma unroll
                for (int w = 0; w < W; ++w) x = fmaf(by[w], place(w, d)[64 * r + lane], x);
                o[d][r] = x;
            }
        }
    }
    if (!real) return;
    const int64_t at = ((int64_t)b * a.queries + query) * a.heads + head;
    if (part_out) {
        const int64_t all_rows = (int64_t)a.batch * a.queries * a.heads;
        float* to = part_out + (split * all_rows + at) * a.dim;
        if (half == 0 && (SHARED || wave == 0)) {
            part_stats[2 * (split * all_rows + at)] = top;
            part_stats[2 * (split * all_rows + at) + 1] = sum * drop;
        }
#pragma unroll
        for (int d = 0; d < ND; ++d) {
            if (!SHARED && d % S::kWaves != wave) continue;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int e = 32 * d + 8 * (r >> 2) + 4 * half + (r & 3);
                if (e < a.dim) to[e] = o[d][r] * drop;
            }
        }
        return;
    }
    if (stats && half == 0 && (SHARED || wave == 0)) {
        stats[at * a.stat_floats] = top;
        stats[at * a.stat_floats + 1] = sum * drop;
    }
    const float inverse = sum > 0.f ? 1.f / sum : (sum == 0.f ? 0.f : sum);
    T *to = out + at * a.dim, *rest = sizeof(T) == 2 && stats ? taser_rest<T>(stats, at, a.stat_floats) : nullptr;
#pragma unroll
    for (int d = 0; d < ND; ++d) {
        if (!SHARED && d % S::kWaves != wave) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int e = 32 * d + 8 * j + 4 * half;
            T x[4], y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[i] = (T)(o[d][4 * j + i] * inverse);
                y[i] = (T)(o[d][4 * j + i] * inverse - (float)x[i]);
            }
            taser_store(to + e, a.dim - e, x);
            if (rest) taser_store(rest + e, a.dim - e, y);
        }
    }
}

// Joins the splits, where they are few: a thread has one element of a row.
template <typename T>
__global__ __launch_bounds__(256) void attention_join_few_kernel(const float* part_out, const float* part_stats, int64_t rows, int32_t dim, int32_t splits, T* out, float* stats,
                                                                 int32_t stat_floats) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= rows * dim) return;
    const int64_t row = i / dim;
    const int e = (int)(i - row * dim);
    float top = -INFINITY, sum = 0.f, x = 0.f;
#pragma unroll 4
    for (int s = 0; s < splits; ++s) top = fmaxf(top, part_stats[2 * (s * rows + row)]);
    // (Splits whose scores are all NaN say minus infinity too, but their sums are not 0.)
#pragma unroll 4
    for (int s = 0; s < splits; ++s) {
        const float by = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((part_stats[2 * (s * rows + row)] - top) * kLog2e);
        sum = fmaf(by, part_stats[2 * (s * rows + row) + 1], sum);
        x = fmaf(by, part_out[(s * rows + row) * dim + e], x);
    }
    x = sum != 0.f ? x / sum : 0.f;
    out[i] = (T)x;
    if (!stats) return;
    if (sizeof(T) == 2) taser_rest<T>(stats, row, stat_floats)[e] = (T)(x - (float)(T)x);
    if (e == 0) {
        stats[row * stat_floats] = top;
        stats[row * stat_floats + 1] = sum;
    }
}

// Where they are many: a block has a row, a thread one element of every eighth split. (96 rows of 112 splits 7 us, 45 by the other; 6 000
// rows of few splits 27 us, and 7 by the other.)
template <typename T>
__global__ __launch_bounds__(1024) void attention_join_kernel(const float* part_out, const float* part_stats, int64_t rows, int32_t dim, int32_t splits, T* out, float* stats,
                                                              int32_t stat_floats) {
    __shared__ float weights[kMostSplits], parts[8][TASER_MAX_HEAD_DIM], whole[2];
    const int64_t row = blockIdx.x;
    const int e = threadIdx.x & 127, chain = threadIdx.x >> 7;
    if (threadIdx.x < 64) {   // the splits' weights, and the row's sum in one order
        float top = -INFINITY, sum = 0.f;
        for (int s = threadIdx.x; s < splits; s += 64) top = fmaxf(top, part_stats[2 * (s * rows + row)]);
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) top = fmaxf(top, __shfl_xor(top, m));
        for (int s = threadIdx.x; s < splits; s += 64) {
            const float by = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((part_stats[2 * (s * rows + row)] - top) * kLog2e);
            weights[s] = by;
            sum = fmaf(by, part_stats[2 * (s * rows + row) + 1], sum);
        }
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) sum += __shfl_xor(sum, m);
        if (threadIdx.x == 0) {
            whole[0] = top;
            whole[1] = sum;
        }
    }
    __syncthreads();
    float x = 0.f;
    if (e < dim)
#pragma unroll 4
        for (int s = chain; s < splits; s += 8) x = fmaf(weights[s], part_out[(s * rows + row) * dim + e], x);
    parts[chain][e] = x;
    __syncthreads();
    if (chain || e >= dim) return;
    x = 0.f;
#pragma unroll
    for (int c = 0; c < 8; ++c) x += parts[c][e];
    const float sum = whole[1];
    x = sum != 0.f ? x / sum : 0.f;
    out[row * dim + e] = (T)x;
    if (!stats) return;
    if (sizeof(T) == 2) taser_rest<T>(stats, row, stat_floats)[e] = (T)(x - (float)(T)x);
    if (e == 0) {
        stats[row * stat_floats] = whole[0];
        stats[row * stat_floats + 1] = sum;
    }
}

template <typename T, int ND, bool SHARED>
int launch(TaserAttentionArgs& a, void* out, float* stats, float* work, hipStream_t stream) {
    using S = Shape<T, taser_row_elements(ND), SHARED>;
    const int64_t rows = (int64_t)a.batch * a.queries * a.heads;
    float* part_out = a.splits > 1 ? work : nullptr;
    float* part_stats = a.splits > 1 ? work + a.splits * rows * a.dim : nullptr;
    a.row_tiles = (a.rows + S::kRows - 1) / S::kRows;
    const int64_t items = (int64_t)a.batch * a.kv_heads * a.splits * a.row_tiles;
    const dim3 grid((unsigned)taser_stretched_grid(items)), block(64 * S::kWaves);
    const bool few = a.splits <= 16;
    if (!taser_launch_fits(taser_stretched_grid(items), block.x) || (a.splits > 1 && !taser_launch_fits(few ? (rows * a.dim + 255) / 256 : rows, few ? 256 : 1024)))
        return taser_fail(TASER_E_RANGE, "cross_attention: too many queries and batch entries for one launch");
    {
        TaserProfileSpan span(stream, "attention");
        auto run = [&](auto bias, auto fine) {
            attention_kernel<T, ND, SHARED, decltype(bias)::value, decltype(fine)::value><<<grid, block, 0, stream>>>(a, (T*)out, stats, part_out, part_stats, items);
        };
        const std::true_type yes;
        const std::false_type no;
        constexpr bool narrow = sizeof(T) == 2;
        const std::bool_constant<narrow> fine;
        const std::bool_constant<narrow && !SHARED> rest;   // (what few rows have in any case)
        // Few rows wait for the states, and what the second product adds is little: 32 x 1 query, 8192 states 164.3 us, 165.0 with it; 2 x 3, 100 001
        // states 55.2, 57.1; 8 x 2, 3000 states 36.0, 38.8. Many rows wait for the products: 4 x 2048 x 4096 271 us, 442 with it (heads of 64: 158, 212);
        // up to 128 states, where single weights' roundings do not average out, they have it all the same. With and without `stats` alike: the
        // output's bits do not depend on whether a gradient will be asked for.
        if (!SHARED || a.keys <= kFineStates) {
            if (a.table) run(yes, fine);
            else run(no, fine);
        } else {
            if (a.table) run(yes, rest);
            else run(no, rest);
        }
        TASER_HIP_TRY(hipGetLastError());
    }
    if (a.splits > 1) {
        TaserProfileSpan span(stream, "attention_join");
        if (few)
            attention_join_few_kernel<T><<<dim3((unsigned)((rows * a.dim + 255) / 256)), 256, 0, stream>>>(part_out, part_stats, rows, a.dim, a.splits, (T*)out, stats, a.stat_floats);
        else
            attention_join_kernel<T><<<dim3((unsigned)rows), 1024, 0, stream>>>(part_out, part_stats, rows, a.dim, a.splits, (T*)out, stats, a.stat_floats);
        TASER_HIP_TRY(hipGetLastError());
    }
    return TASER_OK;
}

template <typename T> int launch_typed(TaserAttentionArgs& a, bool shared, void* out, float* stats, float* work, hipStream_t stream) {
    if (a.dim <= 64) return shared ? launch<T, 2, true>(a, out, stats, work, stream) : launch<T, 2, false>(a, out, stats, work, stream);
    if (a.dim <= 96 && shared) return launch<T, 3, true>(a, out, stats, work, stream);   // (few rows: reading the states bounds it)
    return shared ? launch<T, 4, true>(a, out, stats, work, stream) : launch<T, 4, false>(a, out, stats, work, stream);
}

// Rows of its own for each block of waves, or rows shared by them? (8 x 8 pairs, 4096 states, heads of 128, us, own / shared: float32 32 rows
// 111 / 156, 64 188 / 160, 96 352 / 165. bfloat16 32 rows 38 / 36, 64 44 / 40, 96 63 / 50, where the former multiply the weights' rest too:
// without it they cost 34, 39 and 57.)
bool few_rows(const TaserAttentionArgs& a) { return a.rows <= (taser_single(a) ? 32 : 64); }

// Parts of the states, so that the chip is full where there are few rows.
int splits_for(const TaserAttentionArgs& a, int32_t type) {
    if (taser_window_fits(a)) return 1;
    const int64_t pairs = (int64_t)a.batch * a.kv_heads, bytes = pairs * a.rows * a.dim * 4;
    const double width = a.dim <= 64 ? 0.5 : a.dim <= 96 && !few_rows(a) ? 0.75 : 1.;
    // us of a tile for a block, of 64 states for 128 rows, or of 128 for 32 (measured). 512 blocks at a time is right for few rows of up to 64
    // 16-bit elements; the others' blocks take over 80 KiB of LDS and run 256 at a time, which these parts do not allow for.
    if (few_rows(a)) return taser_splits(pairs * ((a.rows + 31) / 32), 512, (a.keys + 127) / 128, width * (type == TASER_F32 ? 5. : 2.), bytes);
    return taser_splits(pairs * ((a.rows + 127) / 128), type == TASER_F32 ? 256 : 512, (a.keys + 63) / 64, width * (type == TASER_F32 ? 14. : 2.5), bytes);
}

uint64_t work_bytes(const TaserAttentionArgs& a, int splits) {
    return splits > 1 ? sizeof(float) * (uint64_t)splits * a.batch * a.queries * a.heads * (a.dim + 2) : 0;
}

}  // namespace

int taser_attention_args(const taser_attention* p, const char* what, TaserAttentionArgs* a) {
    if (!p) return taser_fail(TASER_E_ARG, "%s: null argument block", what);
    if (p->type < TASER_F32 || p->type > TASER_BF16) return taser_fail(TASER_E_ARG, "%s: unknown element type %d", what, p->type);
    if (p->batch < 0 || p->queries < 0 || p->keys < 0 || p->heads < 1 || p->kv_heads < 1 || p->head_dim < 1)
        return taser_fail(TASER_E_ARG, "%s: negative size, or no heads or elements", what);
    if (p->heads % p->kv_heads) return taser_fail(TASER_E_ARG, "%s: %d query heads cannot share %d key heads evenly", what, p->heads, p->kv_heads);
    if (p->head_dim > TASER_MAX_HEAD_DIM) return taser_fail(TASER_E_RANGE, "%s: heads of %d elements (at most %d)", what, p->head_dim, TASER_MAX_HEAD_DIM);
    const int64_t group = p->heads / p->kv_heads, limit = (int64_t)1 << 31;
    if (p->batch >= limit || p->queries * group >= limit - 128 || p->keys >= limit - 128 || (p->queries && p->batch * p->heads >= ((int64_t)1 << 39) / p->queries) ||
        (p->keys && p->batch * p->kv_heads >= ((int64_t)1 << 39) / p->keys))
        return taser_fail(TASER_E_RANGE, "%s: too many queries, states or batch entries", what);
    if (!(p->scale > 0.f) || std::isinf(p->scale)) return taser_fail(TASER_E_ARG, "%s: the scale must be positive and finite", what);
    const bool queries = p->batch && p->queries;
    if (queries && !p->q) return taser_fail(TASER_E_ARG, "%s: null queries", what);
    if (p->batch && p->keys && (!p->k || !p->v)) return taser_fail(TASER_E_ARG, "%s: null states", what);
    if (p->bias_table) {
        if (p->buckets < 1 || p->buckets > TASER_MAX_BUCKETS) return taser_fail(TASER_E_RANGE, "%s: %d buckets (1 to %d)", what, p->buckets, TASER_MAX_BUCKETS);
        if (p->buckets > 1 && !p->bounds) return taser_fail(TASER_E_ARG, "%s: a bias needs its bounds", what);
        if ((queries && !p->query_pos) || (p->batch && p->keys && !p->key_pos)) return taser_fail(TASER_E_ARG, "%s: a bias needs positions", what);
        if (group * p->buckets > TASER_MAX_GROUP_BUCKETS)
            return taser_fail(TASER_E_RANGE, "%s: %lld query heads to a key head with %d buckets (product at most %d)", what, (long long)group, p->buckets, TASER_MAX_GROUP_BUCKETS);
    }
    *a = TaserAttentionArgs{};
    a->q = p->q; a->k = p->k; a->v = p->v;
    a->q_batch = p->q_strides[0]; a->q_token = p->q_strides[1]; a->q_head = p->q_strides[2];
    a->k_batch = p->k_strides[0]; a->k_token = p->k_strides[1]; a->k_head = p->k_strides[2];
    a->v_batch = p->v_strides[0]; a->v_token = p->v_strides[1]; a->v_head = p->v_strides[2];
    a->batch = (int32_t)p->batch; a->heads = p->heads; a->kv_heads = p->kv_heads; a->group = (int32_t)group; a->dim = p->head_dim;
    a->queries = (int32_t)p->queries; a->keys = (int32_t)p->keys; a->rows = (int32_t)(p->queries * group);
    a->scale = p->scale;
    a->lengths = p->lengths; a->mask = p->mask; a->mask_batch = p->mask_stride;
    a->table = p->bias_table; a->bounds = p->bounds; a->query_pos = p->query_pos; a->key_pos = p->key_pos;
    a->query_pos_batch = p->query_pos_stride; a->key_pos_batch = p->key_pos_stride; a->buckets = p->bias_table ? p->buckets : 0;
    a->splits = a->row_tiles = 1;
    a->stat_floats = TASER_ATTENTION_STATS(p->type, p->head_dim);
    const int size = p->type == TASER_F32 ? 4 : 2, whole = 16 / size;
    bool direct = a->dim % whole == 0 && ((uintptr_t)p->k | (uintptr_t)p->v) % 16 == 0;
    for (int i = 0; i < 3; ++i) direct = direct && p->k_strides[i] % whole == 0 && p->v_strides[i] % whole == 0;
    // a tile of 64 states within the reach of its descriptor, and none of those past its last one
    direct = direct && (p->keys < 2 || (p->k_strides[1] >= a->dim && p->v_strides[1] >= a->dim));
    direct = direct && p->k_strides[1] >= 0 && p->v_strides[1] >= 0 && p->k_strides[1] < kTaserTileBytes / 64 / size && p->v_strides[1] < kTaserTileBytes / 64 / size;
    a->direct = direct;
    return TASER_OK;
}

extern "C" int taser_cross_attention_bytes(const taser_attention* p, uint64_t* work, uint64_t* grad_work) {
    TaserAttentionArgs a;
    if (const int rc = taser_attention_args(p, "cross_attention_bytes", &a)) return rc;
    if (work) *work = work_bytes(a, splits_for(a, p->type));
    if (grad_work) *grad_work = taser_attention_grad_bytes(a, p->type);
    return TASER_OK;
}

extern "C" int taser_cross_attention(const taser_attention* p, void* out, float* stats, void* work, uint64_t work_size, void* hip_stream) {
    TaserAttentionArgs a;
    if (const int rc = taser_attention_args(p, "cross_attention", &a)) return rc;
    if (!a.batch || !a.queries) return TASER_OK;
    if (!out) return taser_fail(TASER_E_ARG, "cross_attention: null output");
    a.splits = splits_for(a, p->type);
    const uint64_t need = work_bytes(a, a.splits);
    if (need > work_size) return taser_fail(TASER_E_RANGE, "cross_attention: %llu bytes of workspace, %llu needed", (unsigned long long)work_size, (unsigned long long)need);
    if (need && (!work || (uintptr_t)work % 16)) return taser_fail(TASER_E_ARG, "cross_attention: null or misaligned workspace");
    hipStream_t stream = (hipStream_t)hip_stream;
    taser_clear_stale_hip_error();
    if (taser_window_fits(a)) return taser_window_attention(a, p->type, out, stats, stream);
    const bool shared = !few_rows(a);
    if (p->type == TASER_F32) return launch_typed<float>(a, shared, out, stats, (float*)work, stream);
    if (p->type == TASER_F16) return launch_typed<_Float16>(a, shared, out, stats, (float*)work, stream);
    return launch_typed<__bf16>(a, shared, out, stats, (float*)work, stream);
}

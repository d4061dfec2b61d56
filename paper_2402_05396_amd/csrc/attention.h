// Shared by the translation units of attention to states of another length: argument blocks, tiles in LDS, matrix
// products and the bias by distance. Not part of the ABI.
//
// All products are D = A B + C on tiles of 32 x 32 with a contraction of 16. Lane l holds 8 values of each operand: row
// (A) or column (B) l % 32, contraction places 8 (l / 32) .. +7. Of the result it holds column l % 32 and the 16 rows
// 8 g + 4 (l / 32) + i (g, i < 4) in register 4 g + i. So what a product leaves in registers 8 s .. 8 s + 7 is at once a
// B operand of the next product, whose contraction then runs over rows 16 s + {8 j + 4 (l / 32) + i: j < 2, i < 4}: only
// the A operand has to be read in that order, and no softmax weight ever leaves its lane.
#pragma once

#include "taser_internal.h"

typedef float taser_f4 __attribute__((ext_vector_type(4)));
typedef float taser_f16 __attribute__((ext_vector_type(16)));
typedef uint32_t taser_u4 __attribute__((ext_vector_type(4)));
typedef short taser_s4 __attribute__((ext_vector_type(4)));

template <typename T> struct TaserFrag { typedef T type __attribute__((ext_vector_type(8))); };
template <typename T> using taser_frag = typename TaserFrag<T>::type;

// What the kernels of one call share.
struct TaserAttentionArgs {
    const void *q, *k, *v;
    int64_t q_batch, q_token, q_head, k_batch, k_token, k_head, v_batch, v_token, v_head;   // strides in elements
    int32_t batch, heads, kv_heads, group, dim, queries, keys, rows;                        // group = heads / kv_heads; rows = queries * group
    float scale;
    const int32_t* lengths;   // or null
    const uint8_t* mask;      // or null
    int64_t mask_batch;
    const void* table;        // [heads, buckets] or null: no bias
    const int64_t *bounds, *query_pos, *key_pos;
    int64_t query_pos_batch, key_pos_batch;
    int32_t buckets;
    int32_t splits, row_tiles;
    int32_t stat_floats;      // of a row: {largest score, sum of exponentials}, then, for 16-bit types, what rounding the output took off
    int32_t direct;           // states are 16-byte aligned and their heads whole 16-byte pieces: tiles are loaded past the registers
};

inline bool taser_single(const TaserAttentionArgs& a) { return a.stat_floats == 2; }   // single precision
// Checks a call's arguments and lays them out for the kernels.
int taser_attention_args(const taser_attention* p, const char* what, TaserAttentionArgs* a);
// In how many parts the long axis of `blocks` blocks is cut, `tiles` tiles of `tile` us each, where `slots` blocks run at a time: the
// parts' sums, `bytes` of them a part, are written in 32 bits and read again, in a launch of its own. The cheapest number of parts by that.
inline int taser_splits(int64_t blocks, int64_t slots, int64_t tiles, double tile, int64_t bytes) {
    if (blocks < 1 || tiles < 2) return 1;
    int best = 1;
    double least = 0.;
    for (int n = 1; n <= 128 && n <= tiles; n += n < 16 ? 1 : 8) {
        const double us = (double)((blocks * n + slots - 1) / slots) * (2. * tile + tile * (double)((tiles + n - 1) / n)) + (n > 1 ? 5. + 2. * (double)(n * bytes) / 4e6 : 0.);
        if (n == 1 || us < 0.95 * least) {
            best = n;
            least = us;
        }
    }
    return best;
}

// Work of taser_cross_attention_grad in bytes.
uint64_t taser_attention_grad_bytes(const TaserAttentionArgs& a, int32_t type);

// Buckets to whole float4: what a row of such parts takes.
__host__ __device__ inline int taser_padded(int buckets) { return (buckets + 3) & ~3; }
// dtable[head][u] = the sum of parts [outer][kv_heads][inner][rows][taser_padded(buckets)] over outer, inner and the rows of that head (row r: head r % group
// of its key head's).
int taser_add_tables(const float* parts, int64_t outer, int64_t inner, int32_t kv_heads, int32_t rows, int32_t group, int32_t buckets, int32_t type, void* dtable, hipStream_t stream);

// Windows of few states and rows: kernels of their own.
bool taser_window_fits(const TaserAttentionArgs& a);
int taser_window_attention(const TaserAttentionArgs& a, int32_t type, void* out, float* stats, hipStream_t stream);
uint64_t taser_window_grad_bytes(const TaserAttentionArgs& a);
int taser_window_attention_grad(const TaserAttentionArgs& a, int32_t type, const float* stats, const void* dout, void* dq, void* dk, void* dv, void* dtable, float* work, hipStream_t stream);

// A batch entry's number of states.
__device__ inline int32_t taser_length(const TaserAttentionArgs& a, int32_t b) {
    if (!a.lengths) return a.keys;
    const int32_t n = a.lengths[b];
    return n < 0 ? 0 : (n > a.keys ? a.keys : n);
}

// What rounding took off an output element goes beside the statistics (single precision: nothing does). With it <dout, out> is as
// good as from a 32-bit output: every gradient is that sum's, and where the terms of dtable cancel its error would be all there is.
template <typename T> __device__ inline T* taser_rest(float* stats, int64_t row, int stat_floats) { return (T*)(stats + row * stat_floats + 2); }

// Up to 8 consecutive elements (n of them; the rest are zeros), at any alignment of the element.
template <typename T, int N> __device__ inline void taser_load(const T* p, int n, T (&x)[N]) {
    if (n >= N) {
        __builtin_memcpy(x, p, N * sizeof(T));
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = i < n ? p[i] : (T)0.f;
    }
}
// Four elements, of which the first n are written.
template <typename T> __device__ inline void taser_store(T* to, int n, const T (&x)[4]) {
    if (n >= 4) {
        __builtin_memcpy(to, x, sizeof(x));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < n) to[i] = x[i];
    }
}
template <typename T> __device__ inline taser_frag<T> taser_load_frag(const T* p, int n) {
    T x[8];
    taser_load<T, 8>(p, n, x);
    taser_frag<T> f;
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = x[i];
    return f;
}

__device__ inline void taser_mma(taser_f16& c, const taser_frag<__bf16>& a, const taser_frag<__bf16>& b) {
    c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ inline void taser_mma(taser_f16& c, const taser_frag<_Float16>& a, const taser_frag<_Float16>& b) {
    c = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
// Single precision: the instruction contracts 2 places, one a half wave; the 8 values a lane holds take 8 of them.
__device__ inline void taser_mma(taser_f16& c, const taser_frag<float>& a, const taser_frag<float>& b) {
#pragma unroll
    for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], b[i], c, 0, 0, 0);
}

// Registers 8 s .. 8 s + 7 of a result, times `by`, as an operand.
template <typename T> __device__ inline taser_frag<T> taser_operand(const taser_f16& c, int s, float by = 1.f) {
    taser_frag<T> f;
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = (T)(c[8 * s + i] * by);
    return f;
}

// Sum and maximum over the two halves of a wave: the halves of two copies change places.
__device__ inline float taser_halves_sum(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    const unsigned a = r[0], b = r[1];   // (a cast of r[1] itself would take element 0)
    return __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
}
__device__ inline float taser_halves_max(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    const unsigned a = r[0], b = r[1];
    return fmaxf(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b));
}

// Half precision ends at 6e-8 and at 65504, and a weight's gradient over thousands of states, of a mean loss or of one scaled up, lies
// beyond. So it is multiplied by a power of two before it is rounded: one for each column of a product's sums, which are held times the same
// and multiplied again where a larger value asks for another. The largest value yet lies in 2^7 .. 2^15 (or below, from the start on).
// (Forward and gradient of 2 x 4096 x 4096, 16 heads on 4 of 128, float16: 1267 us for 1257 without, with a bias 1550 for 1500; of 64
// elements 798 for 772. At a dout of 1e-3 the error of dq is 0.0003 of it, and was 0.003.)
template <typename T> constexpr bool taser_lifted = false;
template <> constexpr inline bool taser_lifted<_Float16> = true;
constexpr float kTaserFirstLift = 0x1p60f, kTaserMostLifted = 0x1p15f;   // (products of half precision numbers, 2^39 at most, stay finite with it)
// The factor that brings a magnitude into 2^7 .. 2^8.
__device__ inline float taser_relift(float most) { return ldexpf(1.f, 134 - (int)(__builtin_bit_cast(uint32_t, most) >> 23)); }
// 1 / a power of two.
__device__ inline float taser_unlift(float lift) { return __builtin_bit_cast(float, 0x7f000000u - __builtin_bit_cast(uint32_t, lift)); }

// ---- tiles ----------------------------------------------------------------------------------------------------------
// A tile holds ROWS rows of DP elements (the head size rounded up, the rest zeros) as 16-byte pieces. Piece c of row r lies
// at place c ^ taser_swizzle(r). 256 bytes of LDS are read at a time: one piece of 16 neighboring rows (or two neighboring pieces of 8),
// or four neighboring pieces of 4 rows, in both cases from every bank once.
// A kernel's products take ND times 32 elements of a row (2: up to 64, 3: up to 96, 4: up to 128); the pieces of a row are a power of
// two. Three instead of four, 96 elements: forward 316 to 287 us, gradient 1149 to 1061 us at 2 x 4096 x 4096, 16 heads, bfloat16; in
// single precision, 80 elements, 3 x 333 x 777, 6 heads, the three kernels with products: 178 to 142 us.
constexpr int taser_row_elements(int nd) { return nd <= 2 ? 64 : 128; }
template <int PIECES> __device__ inline int taser_swizzle(int row) {
    static_assert(PIECES >= 8, "");
    if (PIECES == 8) return ((row >> 1) & 1) << 2 | ((row >> 2) & 1) << 1 | ((row >> 3) & 1);
    return (row & 3) << 2 | ((row >> 2) & 1) << 1 | ((row >> 3) & 1);
}

// Loads tiles of ROWS rows by THREADS threads. Past the registers (`direct`) through a buffer descriptor of the tile: a lane's places
// are the same in every tile, rows and elements that are not there lie outside the descriptor and arrive as zeros; vmcnt says when.
// Else element by element through the registers.
constexpr int kTaserNowhere = 0x7ffffff0, kTaserTileBytes = 0x7ff00000;   // a place outside every descriptor; more than any tile may span
template <typename T, int DP, int ROWS, int THREADS> struct TaserTileLoader {
    static constexpr int PIECES = DP * (int)sizeof(T) / 16, EACH = 16 / (int)sizeof(T), N = ROWS * PIECES / THREADS;
    static_assert(ROWS * PIECES % THREADS == 0 && THREADS % 64 == 0, "");
    int thread, dim, place[N];
    bool direct;
    __device__ int row(int i) const { return (i * THREADS + thread) / PIECES; }
    __device__ int element(int i) const { return ((i * THREADS + thread) % PIECES ^ taser_swizzle<PIECES>(row(i))) * EACH; }

    __device__ TaserTileLoader(int thread_, int dim_, bool direct_) : thread(thread_), dim(dim_), direct(direct_) {}
    // row_at(r): elements from the tile's base to row r.
    template <typename F> __device__ void set(F row_at) {
#pragma unroll
        for (int i = 0; i < N; ++i) place[i] = element(i) < dim ? (int)((row_at(row(i)) + element(i)) * (int)sizeof(T)) : kTaserNowhere;
    }
    // `bytes` from base on belong to rows that are there (direct), of which those without their bit of `keep` are left out (if `some`
    // are); row_at as for set.
    template <typename F> __device__ void load(char* lds, const T* base, int bytes, uint64_t keep, bool some, F row_at) const {
        if (direct) {
            const auto tile = __builtin_amdgcn_make_buffer_rsrc((void*)base, 0, bytes, 0x00027000);
#pragma unroll
            for (int i = 0; i < N; ++i) {
                int at = place[i];
                if (some) at = (keep >> row(i)) & 1 ? at : kTaserNowhere;
                char* to = lds + (((i * THREADS + thread) & ~63) << 4);   // a wave writes 1 KiB from a common address on
                __builtin_amdgcn_raw_ptr_buffer_load_lds(tile, (__attribute__((address_space(3))) void*)to, 16, at, 0, 0, 0);
            }
        } else {
#pragma unroll 1
            for (int i = 0; i < N; ++i) {
                T x[EACH];
                taser_load<T, EACH>(base + row_at(row(i)) + element(i), (keep >> row(i)) & 1 ? dim - element(i) : 0, x);
                taser_u4 u;
                __builtin_memcpy(&u, x, 16);
                *(taser_u4*)(lds + ((i * THREADS + thread) << 4)) = u;
            }
        }
    }
};
// Bytes of n rows that are `stride` bytes apart, of which the last is `row` bytes.
__device__ inline int taser_span(int n, int64_t stride, int row) { return n > 0 ? (int)((n - 1) * stride) + row : 0; }

// Waits for this wave's loads past the registers (and all other loads).
__device__ inline void taser_loads_arrived() {
    __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0)
}

// A barrier for what was written to LDS by instructions: loads past the registers may still be on their way.
__device__ inline void taser_lds_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

// Between the turns of lanes that add to one place of LDS by reading and writing it: the compiler, which looks at a lane by itself, may
// not make one turn of two. (Additions by the LDS itself take it two clocks a lane, from all waves: 16 of a lane's for each of the few
// tiles that have several buckets cost 90 of 551 us of a gradient, reads and writes 20.)
__device__ inline void taser_next_turn() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
    asm volatile("" ::: "memory");
}

// Where a lane's part of a tile lies, once for all tiles: 32 rows further on, everything is 32 rows of bytes further on.
// Operand of the tile's rows (lane l: row l % 32), contraction over elements 16 c ..
template <typename T, int DP> struct TaserRowsAt {
    static constexpr int PIECES = DP * (int)sizeof(T) / 16, BYTES = DP * (int)sizeof(T);
    int at[DP / 16];
    __device__ explicit TaserRowsAt(int lane) {
        const int row = lane & 31, half = lane >> 5, s = taser_swizzle<PIECES>(row);
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) at[c] = row * BYTES + (((sizeof(T) == 2 ? 2 * c + half : 4 * c + 2 * half) ^ s) << 4);
    }
    __device__ taser_frag<T> operand(const char* lds, int row0, int c) const {
        taser_frag<T> f;
        if constexpr (sizeof(T) == 2) {
            const taser_u4 u = *(const taser_u4*)(lds + at[c] + row0 * BYTES);
            __builtin_memcpy(&f, &u, 16);
        } else {
            const taser_f4 x = *(const taser_f4*)(lds + at[c] + row0 * BYTES), y = *(const taser_f4*)(lds + (at[c] ^ 16) + row0 * BYTES);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                f[i] = x[i];
                f[4 + i] = y[i];
            }
        }
        return f;
    }
};

// Operand of the tile's columns (lane l: element 32 d + l % 32), contraction over rows row0 + {8 j + 4 (l / 32) + i}, row0 a multiple
// of 16: the transposed tile in the order in which a product leaves its rows.
template <typename T, int DP> struct TaserColumnsAt {
    static constexpr int PIECES = DP * (int)sizeof(T) / 16, BYTES = DP * (int)sizeof(T), PLACES = sizeof(T) == 2 ? 2 : 8;
    int at[DP / 32][PLACES];
    __device__ explicit TaserColumnsAt(int lane) {
        const int half = lane >> 5;
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int j = 0; j < PLACES; ++j) {
                if constexpr (sizeof(T) == 2) {   // 16 lanes read 4 rows of 16 elements, 8 bytes a lane, and get a column of 4 each
                    const int t = lane & 15, c = 4 * d + 2 * ((lane >> 4) & 1) + ((t & 3) >> 1), row = 8 * j + 4 * half + (t >> 2);
                    at[d][j] = row * BYTES + ((c ^ taser_swizzle<PIECES>(row)) << 4) + ((t & 1) << 3);
                } else {
                    const int e = 32 * d + (lane & 31), row = 8 * (j >> 2) + 4 * half + (j & 3);
                    at[d][j] = row * BYTES + (((e >> 2) ^ taser_swizzle<PIECES>(row)) << 4) + ((e & 3) << 2);
                }
            }
    }
    __device__ taser_frag<T> operand(const char* lds, int row0, int d) const {
        taser_frag<T> f;
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const taser_s4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) taser_s4*)(lds + at[d][j] + row0 * BYTES));
                T y[4];
                __builtin_memcpy(y, &x, 8);
#pragma unroll
                for (int i = 0; i < 4; ++i) f[4 * j + i] = y[i];
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = *(const float*)(lds + at[d][j] + row0 * BYTES);
        }
        return f;
    }
};

// The order of a stretch of products that stands alone between branches: AHEAD reads of LDS first, then READS_EACH under each product
// while there are any: enough on the way for the latency of LDS, without a register for all of them.
template <int AHEAD, int READS_EACH, int PRODUCTS> __device__ inline void taser_order() {
    __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
    for (int i = 0; i < PRODUCTS; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if (AHEAD + i * READS_EACH < PRODUCTS * READS_EACH) __builtin_amdgcn_sched_group_barrier(0x100, READS_EACH, 0);
    }
}

// ---- the bias by distance ----------------------------------------------------------------------------------------------
// Lane l keeps bound l; there are at most 63. A distance common to the wave has as many bounds at most as it as lanes say so.
__device__ inline int64_t taser_lane_bound(const TaserAttentionArgs& a, int lane) {
    return lane < a.buckets - 1 ? a.bounds[lane] : INT64_MAX;
}
__device__ inline int taser_uniform_bucket(int64_t bound, int64_t distance, int buckets) {
    const int n = __popcll(__ballot(bound <= distance));
    return n < buckets ? n : buckets - 1;
}
constexpr float kTaserFoldable = 8192.f;   // the largest bias that may be added to a row's constant rather than to its scores
__device__ inline int64_t taser_apart(int64_t a, int64_t b) { return (int64_t)((uint64_t)a - (uint64_t)b); }
__device__ inline int64_t taser_lane_value(int64_t x, int lane) {
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, lane) |
                     (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)((uint64_t)x >> 32), lane) << 32);
}
// Buckets of single distances. Where all bounds lie within a thousand of one another, as those of token distances do, a table in LDS
// has the bucket of each distance between them, and a distance costs a read. Others are compared with the bounds in question.
constexpr int kTaserNear = 1024;
struct TaserNear {
    int64_t base;   // the table's first entry: just below the first bound
    int last;       // its last; -1: there is no table
    __device__ TaserNear() : base(0), last(-1) {}
    // By all threads of a block, before a barrier; lane l has bound l.
    __device__ TaserNear(int64_t bound, int buckets, uint8_t* near, int room = kTaserNear) : base(0), last(-1) {
        if (buckets < 2) return;
        base = taser_lane_value(bound, 0) - 1;
        const uint64_t span = (uint64_t)taser_lane_value(bound, buckets - 2) - (uint64_t)base;
        if (span >= (uint64_t)room) return;
        last = (int)span;
        for (int e0 = 0; e0 <= last; e0 += blockDim.x) {
            const int e = e0 + threadIdx.x;
            int n = 0;
            for (int u = 0; u < buckets - 1; ++u) n += (int)(taser_lane_value(bound, u) - base) <= e;
            if (e <= last) near[e] = (uint8_t)n;
        }
    }
};
struct TaserBuckets {
    const uint8_t* near;
    int64_t bound;
    int low, high, last;
    uint32_t base;
    bool read;
    // Distances of the tile lie in least .. most, their buckets in low .. high.
    __device__ TaserBuckets(const TaserNear& n, const uint8_t* near_, int64_t bound_, int low_, int high_, int64_t least, int64_t most)
        : near(near_), bound(bound_), low(low_), high(high_), last(n.last), base((uint32_t)(uint64_t)n.base) {
        const int64_t reach = 1 << 30;
        read = last >= 0 && least > n.base - reach && most < n.base + reach;
    }
    // from - to[i], or to[i] - from. (Masked states may lie anywhere: theirs is any bucket of the table.)
    template <bool BACK> __device__ void find(int (&bucket)[4], int64_t from, const int64_t* to) const {
        if (read) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t x = (uint32_t)(uint64_t)from, y = (uint32_t)(uint64_t)to[i];
                int at = (int)((BACK ? y - x : x - y) - base);
                at = at < 0 ? 0 : (at > last ? last : at);
                bucket[i] = near[at];
            }
        } else {
            int64_t apart[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                apart[i] = BACK ? taser_apart(to[i], from) : taser_apart(from, to[i]);
                bucket[i] = low;
            }
            for (int u = low; u < high; ++u) {
                const int64_t x = taser_lane_value(bound, u);
#pragma unroll
                for (int i = 0; i < 4; ++i) bucket[i] += x <= apart[i];
            }
        }
    }
};
// Buckets whose biases of all `group` heads of a table [buckets][group] may be folded, as bits.
__device__ inline uint64_t taser_foldable(const float* table, int buckets, int group, int lane) {
    bool all = lane < buckets;
    if (all)
        for (int g = 0; g < group; ++g) all = all && fabsf(table[lane * group + g]) <= kTaserFoldable;
    return __ballot(all);
}
// The smaller of x and what the lane takes from another one.
__device__ inline int64_t taser_min64(int64_t x, int64_t y) { return y < x ? y : x; }
template <int CONTROL> __device__ inline int64_t taser_min_dpp(int64_t x) {
    const int low = (int)(uint32_t)(uint64_t)x, high = (int)((uint64_t)x >> 32);
    const uint32_t a = (uint32_t)__builtin_amdgcn_update_dpp(0, low, CONTROL, 0xf, 0xf, false), b = (uint32_t)__builtin_amdgcn_update_dpp(0, high, CONTROL, 0xf, 0xf, false);
    return taser_min64(x, (int64_t)((uint64_t)b << 32 | a));
}
// Smallest of each half wave's values, in all its lanes.
__device__ inline int64_t taser_half_min(int64_t x) {
    x = taser_min_dpp<0x121>(x);   // rotations within 16 lanes
    x = taser_min_dpp<0x122>(x);
    x = taser_min_dpp<0x124>(x);
    x = taser_min_dpp<0x128>(x);
    const uint32_t low = (uint32_t)(uint64_t)x, high = (uint32_t)((uint64_t)x >> 32);
    const auto l = __builtin_amdgcn_permlane16_swap(low, low, false, false), h = __builtin_amdgcn_permlane16_swap(high, high, false, false);
    const uint32_t l0 = l[0], l1 = l[1], h0 = h[0], h1 = h[1];
    return taser_min64((int64_t)((uint64_t)h0 << 32 | l0), (int64_t)((uint64_t)h1 << 32 | l1));
}
// {smallest of all lanes' `low`, smallest of all lanes' `high`}, the one in the lower half's lanes and the other in the upper's.
__device__ inline int64_t taser_two_mins(int64_t low, int64_t high) {
    const auto l = __builtin_amdgcn_permlane32_swap((uint32_t)(uint64_t)low, (uint32_t)(uint64_t)high, false, false);
    const auto h = __builtin_amdgcn_permlane32_swap((uint32_t)((uint64_t)low >> 32), (uint32_t)((uint64_t)high >> 32), false, false);
    const uint32_t l0 = l[0], l1 = l[1], h0 = h[0], h1 = h[1];
    return taser_half_min(taser_min64((int64_t)((uint64_t)h0 << 32 | l0), (int64_t)((uint64_t)h1 << 32 | l1)));
}
// Range of the positions of the lanes that have one: ends[0] the smallest, ends[1] the largest (INT64_MAX, -INT64_MAX: none).
__device__ inline void taser_store_range(int64_t pos, bool there, int lane, int64_t* ends) {
    const int64_t x = taser_two_mins(there ? pos : INT64_MAX, there ? -pos : INT64_MAX);
    if (lane == 0) ends[0] = x;
    if (lane == 32) ends[1] = -x;
}
__device__ inline void taser_range(int64_t pos, bool there, int64_t* low, int64_t* high) {
    const int64_t x = taser_two_mins(there ? pos : INT64_MAX, there ? -pos : INT64_MAX);
    *low = taser_lane_value(x, 0);
    *high = -taser_lane_value(x, 32);
}

// Workgroups are handed out to the eight L2 partitions in turn: each partition takes a stretch of consecutive work, so that
// workgroups that read the same states share a cache. -1: nothing to do.
__device__ inline int64_t taser_stretch_of_work(int64_t id, int64_t all) {
    const int64_t each = (all + 7) / 8, at = (id & 7) * each + (id >> 3);
    return (id >> 3) < each && at < all ? at : -1;
}
inline int64_t taser_stretched_grid(int64_t all) { return (all + 7) / 8 * 8; }

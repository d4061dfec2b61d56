// Attention over windows: at most 64 states and 32 rows (queries and heads that share a key head) an item, thousands of items. An
// item's keys and values are read once, all of them on their way before the first is used.
//
// A wavefront has an item. L lanes hold a row of the states, 16 bytes each, so 64 / L states are read at a time, in N turns; state
// s L' + g (L' = 64 / L) is group g's in turn s. A score is a sum over a group; then lane (g, c) takes the score of turn c: each
// state has one lane, whose softmax weight costs one exponential, and where its bucket, its gradient and the sums over all states
// are found. The weights go back to the groups for the sums over the states.
//
// Bound by reading the states: 30000 windows of 25 states, four heads on two of 64, float16, bias: 85 us for 364 MB, 4.4 TB/s; with
// the gradient in bfloat16 97 + 330 us, the latter for 850 MB, far from it: scores pass through scratch memory on their way to their lanes. 12000
// windows of 10 states, two heads of 50, float32: 29 + 48 us for 97 + 200 MB (rows of 200 bytes leave 3 of 16 lanes idle). A score costs as many vector instructions as its row has elements over L, so many rows or states an item are
// left to the tiles.
#include "attention.h"

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kWindowRows = 32;

// x of the lane whose number differs in bit M (for M < 16, among lanes that agree in the bits below: they hold the same value).
template <int M> __device__ inline float other(float x) {
    const int v = __builtin_bit_cast(int, x);
    int y;
    if constexpr (M == 1) y = __builtin_amdgcn_update_dpp(0, v, 0xb1, 0xf, 0xf, false);         // quad_perm 1 0 3 2
    else if constexpr (M == 2) y = __builtin_amdgcn_update_dpp(0, v, 0x4e, 0xf, 0xf, false);    // quad_perm 2 3 0 1
    else if constexpr (M == 4) y = __builtin_amdgcn_update_dpp(0, v, 0x141, 0xf, 0xf, false);   // row_half_mirror
    else if constexpr (M == 8) y = __builtin_amdgcn_update_dpp(0, v, 0x128, 0xf, 0xf, false);   // row_ror 8
    else return __shfl_xor(x, M);
    return __builtin_bit_cast(float, y);
}
struct Pair { float a, b; };
// {a of the lane with bit M clear, b of it} where the bit is clear ... : the two halves of a pair of values change places, so that
// a + b is a's sum over the bit where it is clear, and b's where it is set.
template <int M> __device__ inline Pair swapped(float a, float b, int lane) {
    if constexpr (M == 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b), false, false);
        const unsigned x = r[0], y = r[1];   // (a cast of r[1] itself would take element 0)
        return {__builtin_bit_cast(float, x), __builtin_bit_cast(float, y)};
    } else if constexpr (M == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b), false, false);
        const unsigned x = r[0], y = r[1];   // (a cast of r[1] itself would take element 0)
        return {__builtin_bit_cast(float, x), __builtin_bit_cast(float, y)};
    } else {
        const bool set = lane & M;
        return {set ? b : a, other<M>(set ? a : b)};
    }
}
template <int M> __device__ inline float add_other(float x) {
    if constexpr (M >= 16) {
        const Pair p = swapped<M>(x, x, 0);
        return p.a + p.b;
    } else {
        return x + other<M>(x);
    }
}
template <int M> __device__ inline float max_other(float x) {
    if constexpr (M >= 16) {
        const Pair p = swapped<M>(x, x, 0);
        return fmaxf(p.a, p.b);
    } else {
        return fmaxf(x, other<M>(x));
    }
}
template <int LANES> __device__ inline float group_sum(float x) {   // over LANES neighboring lanes
    x = add_other<1>(x);
    x = add_other<2>(x);
    if constexpr (LANES >= 8) x = add_other<4>(x);
    if constexpr (LANES >= 16) x = add_other<8>(x);
    if constexpr (LANES >= 32) x = add_other<16>(x);
    if constexpr (LANES >= 64) x = add_other<32>(x);
    return x;
}
__device__ inline float wave_max(float x) {
    x = max_other<1>(x);
    x = max_other<2>(x);
    x = max_other<4>(x);
    x = max_other<8>(x);
    x = max_other<16>(x);
    return max_other<32>(x);
}

// Sums of E values over the groups, each lane left with the sums of E / groups of them (at least one), from element first(lane) on.
template <int L, int E> struct Spread {
    static constexpr int kGroups = 64 / L, kLeft = E > kGroups ? E / kGroups : 1;
    template <int M, int N> __device__ static void step(float* x, int lane) {
        if constexpr (M >= L) {
            if constexpr (N > 1) {
#pragma unroll
                for (int i = 0; i < N / 2; ++i) {
                    const Pair p = swapped<M>(x[i], x[i + N / 2], lane);
                    x[i] = p.a + p.b;
                }
                step<M / 2, N / 2>(x, lane);
            } else {
                x[0] = M >= 16 ? add_other<M>(x[0]) : x[0] + other<M>(x[0]);
                step<M / 2, 1>(x, lane);
            }
        }
    }
    __device__ static void sums(float* x, int lane) { step<32, E>(x, lane); }
    __device__ static int first(int lane) {
        int at = 0, n = E;
#pragma unroll
        for (int m = 32; m >= L; m >>= 1)
            if (n > 1) {
                n /= 2;
                at += lane & m ? n : 0;
            }
        return at;
    }
};

template <typename T, int E> struct Chunk { T x[E]; };

// Keeps 16-bit elements as they are across a loop's rounds: widened ahead of it they would take twice the registers, and half the
// waves would fit.
template <typename T, int E> __device__ inline void stay_narrow(Chunk<T, E>& c) {
    if constexpr (sizeof(T) == 2) {
        typedef uint32_t words __attribute__((ext_vector_type(4)));
        words x;
        __builtin_memcpy(&x, c.x, 16);
        asm volatile("" : "+v"(x));
        __builtin_memcpy(c.x, &x, 16);
    }
}

// A lane's 16 bytes of a row: where the row ends inside them they are its last 16 (elements of the lane before it come twice, and
// count once, as zeros of `q`).
template <typename T, int E> __device__ inline Chunk<T, E> load_chunk(const T* row, int at, bool there) {
    Chunk<T, E> c;
    if (there) {
        __builtin_memcpy(c.x, row + at, 16);
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i) c.x[i] = (T)0.f;
    }
    return c;
}
// Values rounded to the type, their 16 bytes by a mask of 4.
template <typename T, int E> __device__ inline Chunk<T, E> masked_chunk(const float (&x)[E], uint32_t mask) {
    typedef uint32_t words __attribute__((ext_vector_type(4)));
    Chunk<T, E> c;
#pragma unroll
    for (int i = 0; i < E; ++i) c.x[i] = (T)x[i];
    words u;
    __builtin_memcpy(&u, c.x, 16);
    u &= mask;
    __builtin_memcpy(c.x, &u, 16);
    return c;
}
template <typename T, int N> __device__ inline void store_values(T* to, const float (&x)[N]) {
    T y[N];
#pragma unroll
    for (int i = 0; i < N; ++i) y[i] = (T)x[i];
    __builtin_memcpy(to, y, sizeof(y));
}

__device__ inline int bucket_of(const int64_t* bounds, int64_t apart) {   // 64 bounds, those past the last INT64_MAX
    int at = 0;
#pragma unroll
    for (int step = 32; step; step >>= 1)
        if (bounds[at + step - 1] <= apart) at += step;
    return at;
}

// What a wave knows of its item.
template <typename T, int L, int N> struct Item {
    static constexpr int E = 16 / (int)sizeof(T), kGroups = 64 / L;
    int lane, group, c, at, b, hk, state;   // at: the lane's first element; state: the lane's own
    bool inside;                            // the lane holds elements
    uint64_t seen;                          // by lane: its state takes part
    const T *k, *v;

    __device__ void open(const TaserAttentionArgs& a, int item, int lane_) {
        lane = lane_;
        group = lane / L;
        c = lane % L;
        b = item / a.kv_heads;
        hk = item - b * a.kv_heads;
        inside = c * E < a.dim;
        at = c * E + E <= a.dim ? c * E : a.dim - E;
        state = c * kGroups + group;
        const int32_t length = taser_length(a, b);
        seen = __ballot(c < N && state < length && (!a.mask || a.mask[b * a.mask_batch + state]));
        k = (const T*)a.k + b * a.k_batch + hk * a.k_head;
        v = (const T*)a.v + b * a.v_batch + hk * a.v_head;
    }
    __device__ int turn_state(int turn) const { return turn * kGroups + group; }
    __device__ bool turn_seen(int turn) const { return inside && (seen >> (group * L + turn)) & 1; }
    __device__ void load_states(const TaserAttentionArgs& a, Chunk<T, E> (&kc)[N], Chunk<T, E> (&vc)[N]) const {
#pragma unroll
        for (int s = 0; s < N; ++s) kc[s] = load_chunk<T, E>(k + turn_state(s) * a.k_token, at, turn_seen(s));
#pragma unroll
        for (int s = 0; s < N; ++s) vc[s] = load_chunk<T, E>(v + turn_state(s) * a.v_token, at, turn_seen(s));
    }
    __device__ const T* query_row(const TaserAttentionArgs& a, int query, int g) const {
        return (const T*)a.q + b * a.q_batch + query * a.q_token + (hk * a.group + g) * a.q_head;
    }
    __device__ Chunk<T, E> load_row(const T* row, bool there) const { return load_chunk<T, E>(row, at, there && inside); }
    // A row's elements, those that the lane before has too as zeros.
    __device__ void widen(const Chunk<T, E>& y, float (&x)[E]) const {
#pragma unroll
        for (int i = 0; i < E; ++i) x[i] = at + i >= c * E ? (float)y.x[i] : 0.f;
    }
    __device__ float dot(const float (&x)[E], const Chunk<T, E>& y) const {
        float d = 0.f;
#pragma unroll
        for (int i = 0; i < E; ++i) d = fmaf(x[i], (float)y.x[i], d);
        return group_sum<L>(d);
    }
    // The value of turn c, which is the lane's own state's. (The compiler makes an indexed array of it, in LDS or, in the gradient where several
    // rows share an item, of 4 or 8 turns, in 32 - 80 bytes a lane of scratch memory.)
    __device__ float own(const float (&x)[N]) const {
        float y = x[0];
#pragma unroll
        for (int s = 1; s < N; ++s) y = c == s ? x[s] : y;
        return y;
    }
    __device__ float of_turn(float x, int turn) const { return __shfl(x, (lane & ~(L - 1)) + turn); }
};

__device__ inline void load_bounds(const TaserAttentionArgs& a, int64_t* bounds) {
    if (threadIdx.x < 64) bounds[threadIdx.x] = (int)threadIdx.x < a.buckets - 1 ? a.bounds[threadIdx.x] : INT64_MAX;
    __syncthreads();
}

template <typename T, int L, int N>
__global__ __launch_bounds__(256) void window_kernel(const TaserAttentionArgs a, T* out, float* stats, int items) {
    using I = Item<T, L, N>;
    constexpr int E = I::E, LEFT = Spread<L, E>::kLeft;
    __shared__ int64_t bounds[64];
    if (a.table) load_bounds(a, bounds);
    const int item = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
    if (item >= items) return;
    I w;
    w.open(a, item, threadIdx.x & 63);
    Chunk<T, E> k[N], v[N];
    w.load_states(a, k, v);
    const bool mine = (w.seen >> w.lane) & 1;
    const int64_t key_pos = a.table && mine ? a.key_pos[w.b * a.key_pos_batch + w.state] : 0;
    Chunk<T, E> next = w.load_row(w.query_row(a, 0, 0), true);
    int64_t apart = 0;
    for (int r = 0, query = 0, g = 0; r < a.rows; ++r) {
        float q[E];
        w.widen(next, q);
        const int head = w.hk * a.group + g;
        if (a.table && g == 0) apart = taser_apart(a.query_pos[w.b * a.query_pos_batch + query], key_pos);
        const int64_t row = ((int64_t)w.b * a.queries + query) * a.heads + head;
        if (++g == a.group) {
            g = 0;
            ++query;
        }
        next = w.load_row(w.query_row(a, query, g), r + 1 < a.rows);
        float s[N];
#pragma unroll
        for (int t = 0; t < N; ++t) stay_narrow(k[t]);
#pragma unroll
        for (int t = 0; t < N; ++t) s[t] = w.dot(q, k[t]);
        float x = w.own(s) * a.scale;
        if (a.table) x += (float)((const T*)a.table)[(int64_t)head * a.buckets + bucket_of(bounds, apart)];
        if (!mine) x = -INFINITY;
        const float top = wave_max(x), p = __builtin_amdgcn_exp2f((x - (top == -INFINITY ? 0.f : top)) * kLog2e), sum = group_sum<64>(p);
        float o[E];
#pragma unroll
        for (int i = 0; i < E; ++i) o[i] = 0.f;
#pragma unroll
        for (int t = 0; t < N; ++t) {
            const float y = w.of_turn(p, t);
            stay_narrow(v[t]);
#pragma unroll
            for (int i = 0; i < E; ++i) o[i] = fmaf(y, (float)v[t].x[i], o[i]);
        }
        Spread<L, E>::sums(o, w.lane);
        const float inverse = sum != 0.f ? 1.f / sum : 0.f;
        float left[LEFT];
#pragma unroll
        for (int i = 0; i < LEFT; ++i) left[i] = o[i] * inverse;
        if (w.inside) store_values<T, LEFT>(out + row * a.dim + w.at + Spread<L, E>::first(w.lane), left);
        if (!stats) continue;
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int i = 0; i < LEFT; ++i) left[i] -= (float)(T)left[i];
            if (w.inside) store_values<T, LEFT>(taser_rest<T>(stats, row, a.stat_floats) + w.at + Spread<L, E>::first(w.lane), left);
        }
        if (w.lane == 0) {
            stats[row * a.stat_floats] = top;
            stats[row * a.stat_floats + 1] = sum;
        }
    }
}

// A wave takes every waves-th item (their number is a multiple of the key heads': a wave's items have one) and keeps the table's
// gradient, lane u bucket u: in a register where its rows are one (ONE), else in LDS.
template <typename T, int L, int N, bool ONE>
__global__ __launch_bounds__(256) void window_grad_kernel(const TaserAttentionArgs a, const T* dout, const float* stats, T* dq, T* dk, T* dv, float* part_table, int items, int waves) {
    using I = Item<T, L, N>;
    constexpr int E = I::E, LEFT = Spread<L, E>::kLeft;
    __shared__ int64_t bounds[64];
    __shared__ float table_sums[ONE ? 1 : 4][ONE ? 1 : kWindowRows][ONE ? 1 : 64];
    // Sums of dk and dv for all states stay in registers where there is room (half of the turns of a 16-bit row and fewer); else weights
    // and dx wait in LDS until all rows have theirs, and the rows are read again for each few turns of states. At 64 states of 128 in
    // 16 bits, two rows, 8000 windows: 385 us (one turn at a time 555, all in registers over 800, spilled); at 50 states of 64 in
    // bfloat16, eight rows, 20000 windows: registers 843 us, waiting 915.
    constexpr bool LATER = !ONE && N >= 16;
    __shared__ float2 waiting[LATER ? 4 : 1][LATER ? kWindowRows : 1][LATER ? 64 : 1];
    if (a.table) load_bounds(a, bounds);
    const int wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)), slot = ONE ? 0 : threadIdx.x >> 6, lane = threadIdx.x & 63;
    if (wave >= waves) return;
    float table_sum = 0.f;
    if (!ONE && a.table)
        for (int r = 0; r < a.rows; ++r) table_sums[slot][r][lane] = 0.f;
    for (int item = wave; item < items; item += waves) {
        I w;
        w.open(a, item, lane);
        Chunk<T, E> k[N], v[N];
        w.load_states(a, k, v);
        const bool mine = (w.seen >> w.lane) & 1;
        const int64_t key_pos = a.table && mine ? a.key_pos[w.b * a.key_pos_batch + w.state] : 0;
        constexpr int HELD = LATER ? 32 / E : N;
        float one[HELD][E], two[HELD][E];   // dk, dv
#pragma unroll
        for (int t = 0; t < HELD; ++t)
#pragma unroll
            for (int i = 0; i < E; ++i) one[t][i] = two[t][i] = 0.f;
        const int64_t row0 = (int64_t)w.b * a.queries * a.heads + w.hk * a.group;
        Chunk<T, E> next_q = w.load_row(w.query_row(a, 0, 0), true), next_y = w.load_row(dout + row0 * a.dim, true);
        int bucket = 0;
        for (int r = 0, query = 0, g = 0; r < (ONE ? 1 : a.rows); ++r) {
            float q[E], y[E];
            w.widen(next_q, q);
            w.widen(next_y, y);
            const int head = w.hk * a.group + g;
            if (a.table && g == 0) bucket = bucket_of(bounds, taser_apart(a.query_pos[w.b * a.query_pos_batch + query], key_pos));
            const int64_t row = row0 + (int64_t)query * a.heads + g;
            const float top = stats[row * a.stat_floats], sum = stats[row * a.stat_floats + 1];
            if (!ONE) {
                if (++g == a.group) {
                    g = 0;
                    ++query;
                }
                next_q = w.load_row(w.query_row(a, query, g), r + 1 < a.rows);
                next_y = w.load_row(dout + (row0 + (int64_t)query * a.heads + g) * a.dim, r + 1 < a.rows);
            }
            float s[N], d[N];
#pragma unroll
            for (int t = 0; t < N; ++t) {
                stay_narrow(k[t]);
                stay_narrow(v[t]);
                s[t] = w.dot(q, k[t]);
                d[t] = w.dot(y, v[t]);
            }
            float x = w.own(s) * a.scale;
            const float dp = w.own(d);
            if (a.table) x += (float)((const T*)a.table)[(int64_t)head * a.buckets + bucket];
            const bool part = mine && sum != 0.f;   // (a row without states gives zeros, whatever comes back to it)
            const float p = part ? __builtin_amdgcn_exp2f((x - top) * kLog2e) / sum : 0.f;
            const float t = group_sum<64>(part ? p * dp : 0.f);
            const float dx = part ? p * (dp - t) : 0.f;
            if (a.table) {   // a lane a bucket: the states' dx pass by in their order
                float add = 0.f;
                for (uint64_t left = w.seen; left; left &= left - 1) {
                    const int l = __builtin_ctzll(left);
                    const float value = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, dx), l));
                    add += __builtin_amdgcn_readlane(bucket, l) == lane ? value : 0.f;
                }
                if (ONE) table_sum += add;
                else table_sums[slot][r][lane] += add;
            }
            float sums[E];
#pragma unroll
            for (int i = 0; i < E; ++i) sums[i] = 0.f;
#pragma unroll
            for (int n = 0; n < N; ++n) {
                const float f = w.of_turn(dx, n) * a.scale;
                stay_narrow(k[n]);
#pragma unroll
                for (int i = 0; i < E; ++i) sums[i] = fmaf(f, (float)k[n].x[i], sums[i]);
                if constexpr (!LATER) {
                    const float h = w.of_turn(p, n);
#pragma unroll
                    for (int i = 0; i < E; ++i) {
                        one[n][i] = fmaf(f, q[i], one[n][i]);
                        two[n][i] = fmaf(h, y[i], two[n][i]);
                    }
                }
            }
            if constexpr (LATER) waiting[slot][r][lane] = float2{dx * a.scale, p};
            Spread<L, E>::sums(sums, w.lane);
            float left[LEFT];
#pragma unroll
            for (int i = 0; i < LEFT; ++i) left[i] = sums[i];
            if (w.inside) store_values<T, LEFT>(dq + row * a.dim + w.at + Spread<L, E>::first(w.lane), left);
        }
        // Which of the group's states take part, by turn (a NaN among the queries is no masked state's). Found here: carried along from the
        // loads of the states it costs 10 to 20 registers.
        uint32_t seen = (uint32_t)(w.seen >> (w.group * L));
        asm volatile("" : "+v"(seen));
        // A lane whose 16 bytes reach back into the lane's before has zeros there: it writes its own elements.
        auto write = [&](int n, const float (&x)[E], const float (&y)[E]) {
            if (!w.inside || w.turn_state(n) >= a.keys) return;
            const int64_t to = (((int64_t)w.b * a.keys + w.turn_state(n)) * a.kv_heads + w.hk) * a.dim;
            const uint32_t keep = 0u - ((seen >> n) & 1);
            const Chunk<T, E> kept_x = masked_chunk<T, E>(x, keep), kept_y = masked_chunk<T, E>(y, keep);
            if (w.at == w.c * E) {
                __builtin_memcpy(dk + to + w.at, kept_x.x, 16);
                __builtin_memcpy(dv + to + w.at, kept_y.x, 16);
            } else {
#pragma unroll
                for (int i = 0; i < E; ++i)
                    if (w.at + i >= w.c * E) {
                        dk[to + w.at + i] = kept_x.x[i];
                        dv[to + w.at + i] = kept_y.x[i];
                    }
            }
        };
        if constexpr (LATER) {
#pragma unroll 1
            for (int n = 0; n * I::kGroups < a.keys; n += HELD) {
#pragma unroll
                for (int t = 0; t < HELD; ++t)
#pragma unroll
                    for (int i = 0; i < E; ++i) one[t][i] = two[t][i] = 0.f;
                Chunk<T, E> next_q = w.load_row(w.query_row(a, 0, 0), true), next_y = w.load_row(dout + row0 * a.dim, true);
                for (int r = 0, query = 0, g = 0; r < a.rows; ++r) {
                    float q[E], y[E];
                    w.widen(next_q, q);
                    w.widen(next_y, y);
                    if (++g == a.group) {
                        g = 0;
                        ++query;
                    }
                    next_q = w.load_row(w.query_row(a, query, g), r + 1 < a.rows);
                    next_y = w.load_row(dout + (row0 + (int64_t)query * a.heads + g) * a.dim, r + 1 < a.rows);
#pragma unroll
                    for (int t = 0; t < HELD; ++t) {
                        const float2 f = waiting[slot][r][(lane & ~(L - 1)) + n + t];
#pragma unroll
                        for (int i = 0; i < E; ++i) {
                            one[t][i] = fmaf(f.x, q[i], one[t][i]);
                            two[t][i] = fmaf(f.y, y[i], two[t][i]);
                        }
                    }
                }
#pragma unroll
                for (int t = 0; t < HELD; ++t) write(n + t, one[t], two[t]);
            }
        } else {
#pragma unroll
            for (int n = 0; n < N; ++n) write(n, one[n], two[n]);
        }
    }
    if (a.table && lane < a.buckets)
        for (int r = 0; r < a.rows; ++r) part_table[((int64_t)wave * a.rows + r) * taser_padded(a.buckets) + lane] = ONE ? table_sum : table_sums[slot][r][lane];
}

struct Call {   // one of the two kernels' arguments
    void* out;
    float* stats;
    const void* dout;
    void *dq, *dk, *dv;
    float* part_table;
    int64_t waves;
    hipStream_t stream;
};

template <typename T, int L, int N> int run(const TaserAttentionArgs& a, const Call& c) {
    const int items = a.batch * a.kv_heads;
    if (c.dout) {
        TaserProfileSpan span(c.stream, "attention_window_grad");
        const dim3 grid((unsigned)((c.waves + 3) / 4));
        if (a.rows == 1) window_grad_kernel<T, L, N, true><<<grid, 256, 0, c.stream>>>(a, (const T*)c.dout, c.stats, (T*)c.dq, (T*)c.dk, (T*)c.dv, c.part_table, items, (int)c.waves);
        else window_grad_kernel<T, L, N, false><<<grid, 256, 0, c.stream>>>(a, (const T*)c.dout, c.stats, (T*)c.dq, (T*)c.dk, (T*)c.dv, c.part_table, items, (int)c.waves);
    } else {
        TaserProfileSpan span(c.stream, "attention_window");
        window_kernel<T, L, N><<<dim3((unsigned)((items + 3) / 4)), 256, 0, c.stream>>>(a, (T*)c.out, c.stats, items);
    }
    TASER_HIP_TRY(hipGetLastError());
    return TASER_OK;
}
// Lanes of a row as few as hold it, turns as few as the states need, out of three.
template <typename T, int L> int run_turns(const TaserAttentionArgs& a, const Call& c) {
    const int turns = (a.keys + 64 / L - 1) / (64 / L);
    if (turns <= L / 4) return run<T, L, L / 4>(a, c);
    if (turns <= L / 2) return run<T, L, L / 2>(a, c);
    return run<T, L, L>(a, c);
}
template <typename T> int run_typed(const TaserAttentionArgs& a, const Call& c) {
    constexpr int E = 16 / (int)sizeof(T);
    if (a.dim <= 8 * E) return run_turns<T, 8>(a, c);
    if constexpr (sizeof(T) == 4)
        if (a.dim > 16 * E) return run_turns<T, 32>(a, c);
    return run_turns<T, 16>(a, c);
}
int run_any(const TaserAttentionArgs& a, int32_t type, const Call& c) {
    if (type == TASER_F32) return run_typed<float>(a, c);
    if (type == TASER_F16) return run_typed<_Float16>(a, c);
    return run_typed<__bf16>(a, c);
}

// Waves of the gradient: enough for the chip, a multiple of the key heads.
int64_t grad_waves(const TaserAttentionArgs& a) {
    const int64_t items = (int64_t)a.batch * a.kv_heads;
    if (!a.table || items <= 4096) return items;
    const int64_t n = 4096 / a.kv_heads * a.kv_heads;
    return n ? n : a.kv_heads;
}

}  // namespace

// Windows cost by rows times states, tiles by their number, one for up to 32 rows and states. 4000 items, heads of 64, here / by tiles, us,
// forward and with the gradient: 16 bits, 16 rows of 10 states 23 / 42, 63 / 148; 8 of 64 40 / 42, 122 / 175; 32 of 64 92 / 37, 353 / 178;
// float32 8 of 64 46 / 105, 167 / 394; 32 of 64 113 / 103, 493 / 400, and 2000 of 128 227 / 87, 659 / 433.
// Calls of a few items go by the same rule: nothing was measured for them. (A row has to have 16 bytes.)
bool taser_window_fits(const TaserAttentionArgs& a) {
    return a.keys >= 1 && a.keys <= 64 && a.rows <= kWindowRows && a.rows * a.keys <= (taser_single(a) ? 1024 : 768) && a.dim >= 8 &&
           (int64_t)a.batch * a.kv_heads < INT32_MAX / 2;
}

int taser_window_attention(const TaserAttentionArgs& a, int32_t type, void* out, float* stats, hipStream_t stream) {
    if (!taser_launch_fits(((int64_t)a.batch * a.kv_heads + 3) / 4, 256)) return taser_fail(TASER_E_RANGE, "cross_attention: too many windows for one launch");
    Call c = {};
    c.out = out;
    c.stats = stats;
    c.stream = stream;
    return run_any(a, type, c);
}

// Never nothing (without a bias no kernel touches it): a caller that brings no workspace learns it from every gradient, not from those alone
// that go over tiles.
uint64_t taser_window_grad_bytes(const TaserAttentionArgs& a) {
    return a.table ? (uint64_t)grad_waves(a) * a.rows * taser_padded(a.buckets) * sizeof(float) : 256;
}

int taser_window_attention_grad(const TaserAttentionArgs& a, int32_t type, const float* stats, const void* dout, void* dq, void* dk, void* dv, void* dtable, float* work, hipStream_t stream) {
    if (!taser_launch_fits((grad_waves(a) + 3) / 4, 256)) return taser_fail(TASER_E_RANGE, "cross_attention_grad: too many windows for one launch");
    Call c = {};
    c.stats = const_cast<float*>(stats);
    c.dout = dout;
    c.dq = dq;
    c.dk = dk;
    c.dv = dv;
    c.part_table = work;
    c.waves = grad_waves(a);
    c.stream = stream;
    if (const int rc = run_any(a, type, c)) return rc;
    return a.table ? taser_add_tables(work, c.waves / a.kv_heads, 1, a.kv_heads, a.rows, a.group, a.buckets, type, dtable, stream) : TASER_OK;
}

// The learned bias by distance as a tensor, and the table's gradient from the tensor's (taser_relative_bias, _grad).
//
// Both are bound by the tensor's bytes. 12 x 1024 x 1024 in bfloat16 written in 8.2 us (3.1 TB/s, a launch included); 4 x 16 x 1000 x 2047 in
// float32 read and summed in 165 us, 3.2 TB/s: bound by what each row of 256 states costs beside its elements, 54 vector and 4 LDS instructions
// in some 800 cycles of a SIMD, among them two searches for the stretch's buckets in 64 bits.
#include "attention.h"

namespace {

struct Distances {
    int32_t heads, buckets, queries, keys;
    int64_t batch;
    const int64_t *bounds, *query_pos, *key_pos;
    int64_t query_pos_batch, key_pos_batch;
};

// A wave's neighboring states, EACH a lane: their positions and the range of those.
template <int EACH> struct States {
    int64_t pos[EACH], least, most;
    int n;
    __device__ States(const int64_t* from, int state, int keys) {
        n = keys - state < EACH ? keys - state : EACH;
        int64_t low = INT64_MAX, high = INT64_MAX;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            pos[i] = i < n ? from[state + i] : 0;
            if (i < n) {
                low = taser_min64(low, pos[i]);
                high = taser_min64(high, -pos[i]);
            }
        }
        const int64_t x = taser_two_mins(low, high);
        least = taser_lane_value(x, 0);
        most = -taser_lane_value(x, 32);
    }
};
constexpr int kNear = 1024;   // distances of the table of buckets
// What all kernels here have in LDS.
struct Near {
    int64_t bound;
    TaserNear map;
};
__device__ inline Near begin(const Distances& d, uint8_t* near, int lane) {
    Near w;
    w.bound = lane < d.buckets - 1 ? d.bounds[lane] : INT64_MAX;
    w.map = TaserNear(w.bound, d.buckets, near, kNear);
    return w;
}
// Buckets of a lane's states.
template <int EACH> __device__ inline void find(const Distances& d, const Near& w, const uint8_t* near, const States<EACH>& s, int64_t from, int low, int high, int (&bucket)[EACH]) {
    const TaserBuckets of(w.map, near, w.bound, low, high, taser_apart(from, s.most), taser_apart(from, s.least));
#pragma unroll
    for (int j = 0; j < EACH / 4; ++j) {
        int four[4];
        of.template find<false>(four, from, s.pos + 4 * j);
#pragma unroll
        for (int i = 0; i < 4; ++i) bucket[4 * j + i] = four[i];
    }
}

// A wave has 64 EACH neighboring states of one query, for all heads of its share: their buckets are found once. Bound by the stores, which
// nothing reads again soon: they go past the caches.
template <typename T, int EACH>
__global__ __launch_bounds__(256) void relative_bias_kernel(const Distances d, const T* table, T* bias, int heads_each) {
    __shared__ uint8_t near[kNear];
    extern __shared__ float values[];   // [heads of this block][buckets]
    const int lane = threadIdx.x & 63, head0 = blockIdx.y * heads_each, heads = d.heads - head0 < heads_each ? d.heads - head0 : heads_each;
    const Near w = begin(d, near, lane);
    for (int i = threadIdx.x; i < heads * d.buckets; i += 256) values[i] = (float)table[(int64_t)head0 * d.buckets + i];
    __syncthreads();
    const int64_t pieces = (d.keys + 64 * EACH - 1) / (64 * EACH), at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (at >= d.batch * d.queries * pieces) return;
    const int64_t row = at / pieces, b = row / d.queries, query = row - b * d.queries;
    const int state = (int)(at - row * pieces) * 64 * EACH + lane * EACH;
    const int64_t from = d.query_pos[b * d.query_pos_batch + query];
    const States<EACH> s(d.key_pos + b * d.key_pos_batch, state, d.keys);
    const int low = taser_uniform_bucket(w.bound, taser_apart(from, s.most), d.buckets), high = taser_uniform_bucket(w.bound, taser_apart(from, s.least), d.buckets);
    int bucket[EACH];
    if (low == high) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) bucket[i] = low;
    } else {
        find<EACH>(d, w, near, s, from, low, high, bucket);
    }
    if (s.n <= 0) return;
    T* to = bias + ((b * d.heads + head0) * d.queries + query) * d.keys + state;
    for (int h = 0; h < heads; ++h, to += (int64_t)d.queries * d.keys) {
        T x[EACH];
        if (low == high) {
            const T one = (T)values[h * d.buckets + low];
#pragma unroll
            for (int i = 0; i < EACH; ++i) x[i] = one;
        } else {
#pragma unroll
            for (int i = 0; i < EACH; ++i) x[i] = (T)values[h * d.buckets + bucket[i]];
        }
        if (s.n == EACH) {
            typedef uint32_t loose __attribute__((ext_vector_type(4), aligned(2)));
            loose u;
            __builtin_memcpy(&u, x, 16);
            __builtin_nontemporal_store(u, (loose*)to);
        } else {
#pragma unroll
            for (int i = 0; i < EACH; ++i)
                if (i < s.n) to[i] = x[i];
        }
    }
}

// A block has one head and a share of the groups of ROWS queries of a batch entry, a wave every fourth of them; it goes over the states 64 EACH
// at a time, the gradients of the next ones of all ROWS queries on their way meanwhile. A stretch of states mostly has one bucket, or at
// least each lane's states do: a lane's sum stays in a register until its bucket changes, then goes to LDS, in a column
// that it shares with one other lane, one after the other: the order of the sums is fixed.
template <typename T> constexpr int kRows = sizeof(T) == 4 ? 8 : 4;   // (bf16: 0.134 ms with 4 rows for what takes 0.190 with 8; float32: 0.165 with 8, 0.176 with 4)
template <typename T, int EACH>
__global__ __launch_bounds__(256) void relative_bias_grad_kernel(const Distances d, const T* dbias, int64_t batch_stride, int64_t head_stride, int64_t query_stride, float* parts) {
    constexpr int ROWS = kRows<T>;
    struct Piece { T x[EACH]; };
    __shared__ uint8_t near[kNear];
    __shared__ int64_t bounds[64];
    extern __shared__ float sums[];   // [4 waves][buckets][32]: lanes l and l + 32 add to column l one after the other
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), head = blockIdx.y;
    float* mine = sums + wave * d.buckets * 32 + (lane & 31);
    auto add = [&](int bucket, float x) {
        if (lane < 32) mine[32 * bucket] += x;
        taser_next_turn();
        if (lane >= 32) mine[32 * bucket] += x;
        taser_next_turn();
    };
    const Near w = begin(d, near, lane);
    if (wave == 0) bounds[lane] = w.bound;
    for (int u = 0; u < d.buckets; ++u) mine[32 * u] = 0.f;
    __syncthreads();
    // The bucket of a distance of the lane's own: from the table if it reaches (the same for all lanes), else by a search.
    auto lane_bucket = [&](int64_t apart, bool read) -> int {
        if (read) {
            int at = (int)((uint32_t)(uint64_t)apart - (uint32_t)(uint64_t)w.map.base);
            at = at < 0 ? 0 : (at > w.map.last ? w.map.last : at);
            return near[at];
        }
        int at = 0;
#pragma unroll
        for (int step = 32; step; step >>= 1)
            if (bounds[at + step - 1] <= apart) at += step;
        return at;
    };
    const int groups = (d.queries + ROWS - 1) / ROWS;
    const int64_t units = d.batch * groups, step = (int64_t)gridDim.x * 4;
    int running = 0;
    float sum = 0.f;
    for (int64_t unit = (int64_t)blockIdx.x * 4 + wave; unit < units; unit += step) {
        const int64_t b = unit / groups;
        const int query0 = (int)(unit - b * groups) * ROWS, rows = d.queries - query0 < ROWS ? d.queries - query0 : ROWS;
        const T* from = dbias + b * batch_stride + head * head_stride + query0 * query_stride;
        const int64_t *key_pos = d.key_pos + b * d.key_pos_batch, *query_pos = d.query_pos + b * d.query_pos_batch + query0;
        auto load = [&](Piece (&x)[ROWS], int state) {
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                if (r < rows && state + EACH <= d.keys) {
                    __builtin_memcpy(x[r].x, from + r * query_stride + state, 16);
                } else {
#pragma unroll
                    for (int i = 0; i < EACH; ++i) x[r].x[i] = r < rows && state + i < d.keys ? from[r * query_stride + state + i] : (T)0.f;
                }
            }
        };
        Piece next[ROWS];
        load(next, lane * EACH);
        for (int state0 = 0; state0 < d.keys; state0 += 64 * EACH) {
            const int state = state0 + lane * EACH;
            Piece x[ROWS];
#pragma unroll
            for (int r = 0; r < ROWS; ++r) x[r] = next[r];
            const States<EACH> s(key_pos, state, d.keys);
            if (state0 + 64 * EACH < d.keys) load(next, state + 64 * EACH);
            int64_t least = s.pos[0], most = s.pos[0];   // of the lane's states
#pragma unroll
            for (int i = 1; i < EACH; ++i)
                if (i < s.n) {
                    least = taser_min64(least, s.pos[i]);
                    most = -taser_min64(-most, -s.pos[i]);
                }
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                if (r >= rows) continue;
                const int64_t at = query_pos[r];
                float all = 0.f;
#pragma unroll
                for (int i = 0; i < EACH; ++i) all += (float)x[r].x[i];   // (past the last state: 0)
                int low = taser_uniform_bucket(w.bound, taser_apart(at, s.most), d.buckets), high = taser_uniform_bucket(w.bound, taser_apart(at, s.least), d.buckets);
                if (low != high) {
                    const int64_t reach = 1 << 30;
                    const bool read = w.map.last >= 0 && taser_apart(at, s.most) > w.map.base - reach && taser_apart(at, s.least) < w.map.base + reach;
                    low = lane_bucket(taser_apart(at, most), read);
                    high = lane_bucket(taser_apart(at, least), read);
                    if (__any(low != high)) {
                        if (low != high) {
#pragma unroll
                            for (int i = 0; i < EACH; ++i)
                                if (i < s.n) add(lane_bucket(taser_apart(at, s.pos[i]), read), (float)x[r].x[i]);
                            all = 0.f;
                            low = running;
                        }
                    }
                }
                if (low != running) {
                    add(running, sum);
                    running = low;
                    sum = 0.f;
                }
                sum += all;
            }
        }
    }
    add(running, sum);
    __syncthreads();
    if ((int)threadIdx.x < d.buckets) {   // a lane a bucket, each starting at a column of its own
        float total = 0.f;
        for (int v = 0; v < 4; ++v) {
            float y = 0.f;
            for (int l = 0; l < 32; ++l) y += sums[(v * d.buckets + threadIdx.x) * 32 + ((l + threadIdx.x) & 31)];
            total += y;
        }
        parts[((int64_t)blockIdx.x * d.heads + head) * taser_padded(d.buckets) + threadIdx.x] = total;
    }
}

int check(const taser_distances* p, const char* what, Distances* d) {
    if (!p) return taser_fail(TASER_E_ARG, "%s: null argument block", what);
    if (p->type < TASER_F32 || p->type > TASER_BF16) return taser_fail(TASER_E_ARG, "%s: unknown element type %d", what, p->type);
    if (p->batch < 0 || p->queries < 0 || p->keys < 0 || p->heads < 1) return taser_fail(TASER_E_ARG, "%s: negative size, or no heads", what);
    if (p->buckets < 1 || p->buckets > TASER_MAX_BUCKETS) return taser_fail(TASER_E_RANGE, "%s: %d buckets (1 to %d)", what, p->buckets, TASER_MAX_BUCKETS);
    const int64_t limit = (int64_t)1 << 31;
    if (p->queries >= limit - 64 || p->keys >= limit - 4096 || p->heads > 65535 || p->batch >= limit ||
        (p->batch && p->queries && p->keys && (double)p->batch * p->queries * p->keys >= 0x1p38))
        return taser_fail(TASER_E_RANGE, "%s: too many queries, states, heads or batch entries", what);
    const bool some = p->batch && p->queries && p->keys;
    if (some && (!p->query_pos || !p->key_pos || (p->buckets > 1 && !p->bounds))) return taser_fail(TASER_E_ARG, "%s: null positions or bounds", what);
    *d = Distances{p->heads, p->buckets, (int32_t)p->queries, (int32_t)p->keys, p->batch, p->bounds, p->query_pos, p->key_pos, p->query_pos_stride, p->key_pos_stride};
    return TASER_OK;
}

// Blocks of a head: some 1024 for all heads, four to a compute unit, as many as its LDS holds with 64 buckets (32 KiB each); none without a
// group of queries for each wave.
int blocks_of_head(const Distances& d, int rows) {
    const int64_t groups = d.batch * ((d.queries + rows - 1) / rows), most = (groups + 3) / 4, wanted = (1024 + d.heads - 1) / d.heads;
    const int64_t n = most < wanted ? most : wanted;
    return n < 1 ? 1 : (int)n;
}
uint64_t work_bytes(const Distances& d, int32_t type) { return (uint64_t)d.heads * blocks_of_head(d, type == TASER_F32 ? kRows<float> : kRows<__bf16>) * taser_padded(d.buckets) * sizeof(float); }

template <typename T> int launch(const Distances& d, const void* table, void* bias, hipStream_t stream) {
    constexpr int EACH = 16 / sizeof(T);
    const int heads_each = d.heads * d.buckets <= 8192 ? d.heads : 8192 / d.buckets;
    const int64_t waves = d.batch * d.queries * ((d.keys + 64 * EACH - 1) / (64 * EACH));
    if (!taser_launch_fits((waves + 3) / 4, 256)) return taser_fail(TASER_E_RANGE, "relative_bias: too many queries and batch entries for one launch");
    TaserProfileSpan span(stream, "relative_bias");
    relative_bias_kernel<T, EACH><<<dim3((unsigned)((waves + 3) / 4), (unsigned)((d.heads + heads_each - 1) / heads_each)), 256, sizeof(float) * heads_each * d.buckets, stream>>>(
        d, (const T*)table, (T*)bias, heads_each);
    TASER_HIP_TRY(hipGetLastError());
    return TASER_OK;
}

template <typename T> int launch_grad(const Distances& d, int32_t type, const void* dbias, const int64_t* strides, void* dtable, float* work, hipStream_t stream) {
    constexpr int EACH = 16 / sizeof(T);
    const int blocks = blocks_of_head(d, kRows<T>);
    const bool some = d.batch && d.queries && d.keys;
    if (some) {
        TaserProfileSpan span(stream, "relative_bias_grad");
        relative_bias_grad_kernel<T, EACH><<<dim3((unsigned)blocks, (unsigned)d.heads), 256, 4 * 32 * sizeof(float) * d.buckets, stream>>>(d, (const T*)dbias, strides[0], strides[1],
                                                                                                                                    strides[2], work);
        TASER_HIP_TRY(hipGetLastError());
    }
    return taser_add_tables(work, some ? blocks : 0, 1, d.heads, 1, 1, d.buckets, type, dtable, stream);
}

}  // namespace

extern "C" int taser_relative_bias_bytes(const taser_distances* p, uint64_t* work) {
    Distances d;
    if (const int rc = check(p, "relative_bias_bytes", &d)) return rc;
    if (work) *work = work_bytes(d, p->type);
    return TASER_OK;
}

extern "C" int taser_relative_bias(const taser_distances* p, const void* table, void* bias, void* hip_stream) {
    Distances d;
    if (const int rc = check(p, "relative_bias", &d)) return rc;
    if (!d.batch || !d.queries || !d.keys) return TASER_OK;
    if (!table || !bias) return taser_fail(TASER_E_ARG, "relative_bias: null table or output");
    hipStream_t stream = (hipStream_t)hip_stream;
    taser_clear_stale_hip_error();
    if (p->type == TASER_F32) return launch<float>(d, table, bias, stream);
    if (p->type == TASER_F16) return launch<_Float16>(d, table, bias, stream);
    return launch<__bf16>(d, table, bias, stream);
}

extern "C" int taser_relative_bias_grad(const taser_distances* p, const void* dbias, const int64_t strides[3], void* dtable, void* work, uint64_t work_size, void* hip_stream) {
    Distances d;
    if (const int rc = check(p, "relative_bias_grad", &d)) return rc;
    if (!dtable) return taser_fail(TASER_E_ARG, "relative_bias_grad: null output");
    if (d.batch && d.queries && d.keys && (!dbias || !strides)) return taser_fail(TASER_E_ARG, "relative_bias_grad: null gradient or strides");
    const uint64_t need = work_bytes(d, p->type);
    if (need > work_size) return taser_fail(TASER_E_RANGE, "relative_bias_grad: %llu bytes of workspace, %llu needed", (unsigned long long)work_size, (unsigned long long)need);
    if (!work || (uintptr_t)work % 16) return taser_fail(TASER_E_ARG, "relative_bias_grad: null or misaligned workspace");
    hipStream_t stream = (hipStream_t)hip_stream;
    taser_clear_stale_hip_error();
    if (p->type == TASER_F32) return launch_grad<float>(d, p->type, dbias, strides, dtable, (float*)work, stream);
    if (p->type == TASER_F16) return launch_grad<_Float16>(d, p->type, dbias, strides, dtable, (float*)work, stream);
    return launch_grad<__bf16>(d, p->type, dbias, strides, dtable, (float*)work, stream);
}

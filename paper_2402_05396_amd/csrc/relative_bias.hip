// The learned bias by distance as a tensor, and the table's gradient from the tensor's (taser_relative_bias, _grad).
#include "attention.h"

namespace {

// How many bounds are at most `apart`: a search over 64 of them (those past the last are INT64_MAX).
__device__ inline int bucket_of(const int64_t* bounds, int64_t apart) {
    int at = 0;
#pragma unroll
    for (int step = 32; step; step >>= 1)
        if (bounds[at + step - 1] <= apart) at += step;
    return at;
}

struct Distances {
    int32_t heads, buckets, queries, keys;
    int64_t batch;
    const int64_t *bounds, *query_pos, *key_pos;
    int64_t query_pos_batch, key_pos_batch;
};

__device__ inline void load_bounds(const Distances& d, int64_t* bounds) {
    if (threadIdx.x < 64) bounds[threadIdx.x] = (int)threadIdx.x < d.buckets - 1 ? d.bounds[threadIdx.x] : INT64_MAX;
}

// A thread has EACH neighboring states of one query: their buckets once, for all heads of its share.
template <typename T, int EACH>
__global__ __launch_bounds__(256) void relative_bias_kernel(const Distances d, const T* table, T* bias, int heads_each) {
    __shared__ int64_t bounds[64];
    extern __shared__ float values[];   // [heads of this block][buckets]
    const int head0 = blockIdx.y * heads_each, heads = d.heads - head0 < heads_each ? d.heads - head0 : heads_each;
    load_bounds(d, bounds);
    for (int i = threadIdx.x; i < heads * d.buckets; i += 256) values[i] = (float)table[(int64_t)head0 * d.buckets + i];
    __syncthreads();
    const int64_t pieces = (d.keys + EACH - 1) / EACH, at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= d.batch * d.queries * pieces) return;
    const int64_t row = at / pieces, b = row / d.queries, query = row - b * d.queries;
    const int state = (int)(at - row * pieces) * EACH, n = d.keys - state < EACH ? d.keys - state : EACH;
    const int64_t from = d.query_pos[b * d.query_pos_batch + query];
    const int64_t* key_pos = d.key_pos + b * d.key_pos_batch + state;
    int bucket[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) bucket[i] = bucket_of(bounds, taser_apart(from, key_pos[i < n ? i : 0]));
    T* to = bias + ((b * d.heads + head0) * d.queries + query) * d.keys + state;
    for (int h = 0; h < heads; ++h, to += (int64_t)d.queries * d.keys) {
        T x[EACH];
#pragma unroll
        for (int i = 0; i < EACH; ++i) x[i] = (T)values[h * d.buckets + bucket[i]];
        if (n == EACH) {
            __builtin_memcpy(to, x, sizeof(x));
        } else {
#pragma unroll
            for (int i = 0; i < EACH; ++i)
                if (i < n) to[i] = x[i];
        }
    }
}

// A block has one head and a share of the (batch entry, query) rows, a wave every fourth of them. A lane adds to a column of sums
// of its own in LDS, so that nothing is added by two lanes and the order of the sums is fixed.
template <typename T, int EACH>
__global__ __launch_bounds__(256) void relative_bias_grad_kernel(const Distances d, const T* dbias, int64_t batch_stride, int64_t head_stride, int64_t query_stride, float* parts) {
    __shared__ int64_t bounds[65];   // bounds[0] is below all
    extern __shared__ float sums[];   // [4 waves][buckets][64 lanes]
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, head = blockIdx.y;
    float* mine = sums + wave * d.buckets * 64 + lane;
    load_bounds(d, bounds + 1);
    if (threadIdx.x == 0) bounds[0] = INT64_MIN;
    for (int u = 0; u < d.buckets; ++u) mine[64 * u] = 0.f;
    __syncthreads();
    const int64_t rows = d.batch * d.queries, step = (int64_t)gridDim.x * 4;
    for (int64_t row = (int64_t)blockIdx.x * 4 + wave; row < rows; row += step) {
        const int64_t b = row / d.queries, query = row - b * d.queries, from = d.query_pos[b * d.query_pos_batch + query];
        const T* x_from = dbias + b * batch_stride + head * head_stride + query * query_stride;
        const int64_t* key_pos = d.key_pos + b * d.key_pos_batch;
        for (int state = lane * EACH; state < d.keys; state += 64 * EACH) {
            const int n = d.keys - state < EACH ? d.keys - state : EACH;
            T x[EACH];
            taser_load<T, EACH>(x_from + state, n, x);
            int64_t apart[EACH];
#pragma unroll
            for (int i = 0; i < EACH; ++i) apart[i] = taser_apart(from, key_pos[state + (i < n ? i : 0)]);
            const int first = bucket_of(bounds + 1, apart[0]);
            const int64_t low = bounds[first], high = bounds[first + 1];
            bool same = true;
            float all = 0.f;
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                same = same && low <= apart[i] && (apart[i] < high);
                all += (float)x[i];
            }
            if (same) {
                mine[64 * first] += all;
            } else {
#pragma unroll
                for (int i = 0; i < EACH; ++i)
                    if (i < n) mine[64 * bucket_of(bounds + 1, apart[i])] += (float)x[i];
            }
        }
    }
    __syncthreads();
    if ((int)threadIdx.x < d.buckets) {   // a lane a bucket, each starting at a column of its own
        float total = 0.f;
        for (int w = 0; w < 4; ++w) {
            float x = 0.f;
            for (int l = 0; l < 64; ++l) x += sums[(w * d.buckets + threadIdx.x) * 64 + ((l + threadIdx.x) & 63)];
            total += x;
        }
        parts[((int64_t)head * gridDim.x + blockIdx.x) * d.buckets + threadIdx.x] = total;
    }
}

template <typename T> __global__ __launch_bounds__(256) void relative_bias_grad_add_kernel(const float* parts, int32_t n, int32_t buckets, T* dtable) {
    __shared__ float sums[4][64];
    const int chain = threadIdx.x >> 6, u = threadIdx.x & 63;
    float x = 0.f;
    if (u < buckets)
        for (int i = chain; i < n; i += 4) x += parts[((int64_t)blockIdx.x * n + i) * buckets + u];
    sums[chain][u] = x;
    __syncthreads();
    if ((int)threadIdx.x < buckets) dtable[(int64_t)blockIdx.x * buckets + u] = (T)((sums[0][u] + sums[1][u]) + (sums[2][u] + sums[3][u]));
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

// Blocks of a head: about 1024 in all, none without a row for each wave.
int blocks_of_head(const Distances& d) {
    const int64_t most = (d.batch * d.queries + 3) / 4, wanted = (1024 + d.heads - 1) / d.heads;
    const int64_t n = most < wanted ? most : wanted;
    return n < 1 ? 1 : (int)n;
}

template <typename T> int launch(const Distances& d, const void* table, void* bias, hipStream_t stream) {
    constexpr int EACH = 16 / sizeof(T);
    const int heads_each = d.heads * d.buckets <= 8192 ? d.heads : 8192 / d.buckets;
    const int64_t threads = d.batch * d.queries * ((d.keys + EACH - 1) / EACH);
    TaserProfileSpan span(stream, "relative_bias");
    relative_bias_kernel<T, EACH><<<dim3((unsigned)((threads + 255) / 256), (unsigned)((d.heads + heads_each - 1) / heads_each)), 256, sizeof(float) * heads_each * d.buckets, stream>>>(
        d, (const T*)table, (T*)bias, heads_each);
    TASER_HIP_TRY(hipGetLastError());
    return TASER_OK;
}

template <typename T> int launch_grad(const Distances& d, const void* dbias, const int64_t* strides, void* dtable, float* work, hipStream_t stream) {
    constexpr int EACH = 16 / sizeof(T);
    const int blocks = blocks_of_head(d);
    const bool some = d.batch && d.queries && d.keys;
    if (some) {
        TaserProfileSpan span(stream, "relative_bias_grad");
        relative_bias_grad_kernel<T, EACH><<<dim3((unsigned)blocks, (unsigned)d.heads), 256, 4 * 64 * sizeof(float) * d.buckets, stream>>>(d, (const T*)dbias, strides[0], strides[1],
                                                                                                                                    strides[2], work);
        TASER_HIP_TRY(hipGetLastError());
    }
    TaserProfileSpan span(stream, "relative_bias_grad_add");
    relative_bias_grad_add_kernel<T><<<dim3((unsigned)d.heads), 256, 0, stream>>>(work, some ? blocks : 0, d.buckets, (T*)dtable);
    TASER_HIP_TRY(hipGetLastError());
    return TASER_OK;
}

}  // namespace

extern "C" int taser_relative_bias_bytes(const taser_distances* p, uint64_t* work) {
    Distances d;
    if (const int rc = check(p, "relative_bias_bytes", &d)) return rc;
    if (work) *work = (uint64_t)d.heads * blocks_of_head(d) * d.buckets * sizeof(float);
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
    const uint64_t need = (uint64_t)d.heads * blocks_of_head(d) * d.buckets * sizeof(float);
    if (need > work_size) return taser_fail(TASER_E_RANGE, "relative_bias_grad: %llu bytes of workspace, %llu needed", (unsigned long long)work_size, (unsigned long long)need);
    if (!work || (uintptr_t)work % 16) return taser_fail(TASER_E_ARG, "relative_bias_grad: null or misaligned workspace");
    hipStream_t stream = (hipStream_t)hip_stream;
    taser_clear_stale_hip_error();
    if (p->type == TASER_F32) return launch_grad<float>(d, dbias, strides, dtable, (float*)work, stream);
    if (p->type == TASER_F16) return launch_grad<_Float16>(d, dbias, strides, dtable, (float*)work, stream);
    return launch_grad<__bf16>(d, dbias, strides, dtable, (float*)work, stream);
}

// Clipped policy loss with a KL term and its gradient (taser_policy_loss): one softmax a row, of which a few places are looked at.
//
// With l = logp of an action: d loss / d l = weight * (-ratio * advantage where that is the smaller term, + kl (1 - exp(ref - l))), and
// d l / d logit[c] = (c is the action) - softmax[c]. So a row's gradient is minus the sum of its actions' slopes times the softmax,
// plus each slope at its action.
//
// Bound by reading the logits once and writing their gradient once: 4096 rows of 64001 in bfloat16 250 us, 1.05 GB at 4.2 TB/s (rows of an odd
// length begin inside cache lines: counters say 0.73 GB read, 0.54 written). 12000 rows of 25 with 10 actions: 6 us, a launch.
#include "attention.h"

namespace {

constexpr float kLog2e = 1.4426950408889634f;

struct Batch {
    int32_t picks, width;
    int64_t rows, stride;
    const int32_t *count, *actions;
    const float *advantage, *old_logp, *ref_logp, *weight;
    float low, high, kl;
};

__device__ inline int32_t taking_part(const Batch& p, int64_t row) {
    if (!p.count) return p.width;
    const int32_t n = p.count[row];
    return n < 0 ? 0 : (n > p.width ? p.width : n);
}

// exp(t) - 1 and exp(t) - 1 - t. The latter is some t^2 / 2 near 0, of which that difference would leave no digits (t = 3e-4: 0 for 4.5e-8):
// up to 1 it is its series, whose next term is below 2^-24 of it there.
__device__ inline void exp_past(float t, float* constant, float* linear) {
    if (fabsf(t) < 1.f) {
        float s = 1.f / 3628800.f;
        s = fmaf(s, t, 1.f / 362880.f);
        s = fmaf(s, t, 1.f / 40320.f);
        s = fmaf(s, t, 1.f / 5040.f);
        s = fmaf(s, t, 1.f / 720.f);
        s = fmaf(s, t, 1.f / 120.f);
        s = fmaf(s, t, 1.f / 24.f);
        s = fmaf(s, t, 1.f / 6.f);
        s = fmaf(s, t, 0.5f);
        *linear = t * t * s;
        *constant = t + *linear;
    } else {
        *constant = expf(t) - 1.f;
        *linear = *constant - t;
    }
}

// Loss of the action at place `at` of the row's, and its slope. An action of weight 0 has neither, whatever else is given for it, and
// does not count: a row without any that does has no gradient, whatever its logits are.
__device__ inline bool action_loss(const Batch& p, int64_t at, float logp, float* loss, float* slope) {
    const float w = p.weight ? p.weight[at] : 1.f, a = p.advantage[at];
    const float ratio = p.old_logp ? expf(logp - p.old_logp[at]) : 1.f;
    const float whole = ratio * a, cut = p.old_logp ? fminf(fmaxf(ratio, 1.f - p.low), 1.f + p.high) * a : whole;
    float x = -(cut < whole ? cut : whole), y = whole <= cut ? -whole : 0.f;
    if (whole != whole) x = y = whole;
    if (p.ref_logp) {
        float slope_of, past;
        exp_past(p.ref_logp[at] - logp, &slope_of, &past);
        x += p.kl * past;
        y -= p.kl * slope_of;
    }
    *loss = w != 0.f ? w * x : 0.f;
    *slope = w != 0.f ? w * y : 0.f;
    return w != 0.f;
}

// Rows of at most 64 candidates and actions: G lanes a row, a candidate and an action a lane.
template <typename T, int G>
__global__ __launch_bounds__(256) void policy_window_kernel(const Batch p, const T* logits, float* loss, float* logp_out, T* grad) {
    const int64_t row = (int64_t)blockIdx.x * (256 / G) + threadIdx.x / G;
    const int lane = threadIdx.x % G;
    if (row >= p.rows) return;   // the lanes of a row leave together
    const int n = taking_part(p, row);
    const float x = lane < n ? (float)logits[row * p.stride + lane] : -INFINITY;
    float top = x;
#pragma unroll
    for (int m = 1; m < G; m <<= 1) top = fmaxf(top, __shfl_xor(top, m, G));
    if (top == -INFINITY) top = 0.f;
    const float e = lane < n ? expf(x - top) : 0.f;
    float sum = e;
#pragma unroll
    for (int m = 1; m < G; m <<= 1) sum += __shfl_xor(sum, m, G);
    const float logsum = logf(sum);
    const int64_t at = row * p.picks + lane;
    const int action = lane < p.picks ? p.actions[at] : -1;
    const bool real = action >= 0 && action < n;
    const float chosen = __shfl(x, real ? action : 0, G);
    float l = 0.f, mine = 0.f, slope = 0.f;
    bool counts = false;
    if (real) {
        l = (chosen - top) - logsum;
        counts = action_loss(p, at, l, &mine, &slope);
    }
    if (lane < p.picks) {
        loss[at] = mine;
        logp_out[at] = l;
    }
    if (!grad) return;
    float all = slope;
#pragma unroll
    for (int m = 1; m < G; m <<= 1) all += __shfl_xor(all, m, G);
    constexpr uint64_t lanes = G == 64 ? ~0ull : (1ull << (G & 63)) - 1;
    const bool some = __ballot(counts) >> (threadIdx.x & 63 & ~(G - 1)) & lanes;
    float g = !some ? 0.f : e / sum * -all;   // (a sum of 0, all are ruled out, or of NaN: NaN, as the softmax is)
    for (int j = 0; j < p.picks; ++j) {
        const int a = __shfl(real ? action : -1, j, G);
        const float y = __shfl(slope, j, G);
        if (a == lane) g += y;
    }
    if (lane < p.width) grad[row * p.width + lane] = (T)(lane < n ? g : 0.f);
}

// The larger of two running (maximum, sum of exponentials).
__device__ inline void join(float& top, float& sum, float other_top, float other_sum) {
    // (Where both are minus infinity the sums are 0, or NaN, of which fmaxf says minus infinity too: they are added all the same.)
    const float best = fmaxf(top, other_top), base = best == -INFINITY ? 0.f : best;
    sum = sum * __builtin_amdgcn_exp2f((top - base) * kLog2e) + other_sum * __builtin_amdgcn_exp2f((other_top - base) * kLog2e);
    top = best;
}

// Any row, a block each. Where a row fits the block's registers (HELD pieces of 16 bytes a thread) it is read once; else what is past them
// is read again for the gradient.
template <typename T, int THREADS, int HELD>
__global__ __launch_bounds__(THREADS, (HELD <= 4 ? 8 : 4)) void policy_row_kernel(const Batch p, const T* logits, float* loss, float* logp_out, T* grad) {
    constexpr int EACH = 16 / sizeof(T);
    struct Piece { T x[EACH]; };
    __shared__ float tops[16], sums[16], slopes[TASER_MAX_PICKS];
    __shared__ int places[TASER_MAX_PICKS];
    __shared__ float whole;
    __shared__ uint32_t some;
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = taking_part(p, row), waves = blockDim.x >> 6;
    const int64_t step = (int64_t)blockDim.x * EACH;
    const T* from = logits + row * p.stride;
    // what the loss needs of the row's actions is on its way too
    const int64_t at = row * p.picks + lane;
    const int action = wave == 0 && lane < p.picks ? p.actions[at] : -1;
    const bool real = action >= 0 && action < n;
    const float chosen = real ? (float)from[action] : 0.f;
    auto load = [&](int64_t c, Piece& x) {   // places past the row's: minus infinity
        if (c + EACH <= n) {
            __builtin_memcpy(x.x, from + c, 16);
        } else {
#pragma unroll
            for (int i = 0; i < EACH; ++i) x.x[i] = c + i < n ? from[c + i] : (T)-INFINITY;
        }
    };
    float top = -INFINITY, sum = 0.f;
    auto take = [&](const Piece& x) {
        float best = (float)x.x[0];
#pragma unroll
        for (int i = 1; i < EACH; ++i) best = fmaxf(best, (float)x.x[i]);
        const float now = fmaxf(top, best), base = now == -INFINITY ? 0.f : now;
        float part = 0.f;
#pragma unroll
        for (int i = 0; i < EACH; ++i) part += __builtin_amdgcn_exp2f(((float)x.x[i] - base) * kLog2e);
        sum = (now == top ? sum : sum * __builtin_amdgcn_exp2f((top - base) * kLog2e)) + part;
        top = now;
    };
    Piece held[HELD];
#pragma unroll
    for (int h = 0; h < HELD; ++h) load(h * step + threadIdx.x * EACH, held[h]);
    {   // all held pieces against their common maximum
        float best = -INFINITY;
#pragma unroll
        for (int h = 0; h < HELD; ++h)
#pragma unroll
            for (int i = 0; i < EACH; ++i) best = fmaxf(best, (float)held[h].x[i]);
        top = best;
        const float base = best == -INFINITY ? 0.f : best;
#pragma unroll
        for (int h = 0; h < HELD; ++h)
#pragma unroll
            for (int i = 0; i < EACH; ++i) sum += __builtin_amdgcn_exp2f(((float)held[h].x[i] - base) * kLog2e);
    }
    for (int64_t c = HELD * step + threadIdx.x * EACH; c < n; c += step) {
        Piece x;
        load(c, x);
        take(x);
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const float t = __shfl_xor(top, m), s = __shfl_xor(sum, m);
        join(top, sum, t, s);
    }
    if (lane == 0) {
        tops[wave] = top;
        sums[wave] = sum;
    }
    __syncthreads();
    top = tops[0];
    sum = sums[0];
    for (int w = 1; w < waves; ++w) join(top, sum, tops[w], sums[w]);
    if (top == -INFINITY) top = 0.f;
    if (wave == 0) {
        float l = 0.f, mine = 0.f, slope = 0.f;
        bool counts = false;
        if (real) {
            l = (chosen - top) - logf(sum);
            counts = action_loss(p, at, l, &mine, &slope);
        }
        if (lane < p.picks) {
            loss[at] = mine;
            logp_out[at] = l;
            places[lane] = real ? action : -1;
            slopes[lane] = slope;
        }
        float all = slope;
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) all += __shfl_xor(all, m);
        const bool any = __any(counts);
        if (lane == 0) {
            whole = all;
            some = any ? ~0u : 0u;
        }
    }
    if (!grad) return;
    __syncthreads();
    const float by = -whole / sum;   // (as in a window)
    const uint32_t keep = __builtin_amdgcn_readfirstlane(some);   // all bits of a gradient, or none
    T* to = grad + row * p.width;
    auto give = [&](int64_t c, const Piece& x) {
        Piece y;
        if (c + EACH <= n) {
#pragma unroll
            for (int i = 0; i < EACH; ++i) y.x[i] = (T)(__builtin_amdgcn_exp2f(((float)x.x[i] - top) * kLog2e) * by);
            typedef uint32_t loose __attribute__((ext_vector_type(4), aligned(2)));
            loose u;
            __builtin_memcpy(&u, y.x, 16);
            u &= keep;
            __builtin_nontemporal_store(u, (loose*)(to + c));
        } else if (c < p.width) {
            for (int i = 0; i < EACH; ++i)
                if (c + i < p.width) to[c + i] = (T)(c + i < n && keep ? __builtin_amdgcn_exp2f(((float)x.x[i] - top) * kLog2e) * by : 0.f);
        }
    };
#pragma unroll
    for (int h = 0; h < HELD; ++h) give(h * step + threadIdx.x * EACH, held[h]);
    for (int64_t c = HELD * step + threadIdx.x * EACH; c < p.width; c += step) {
        Piece x;
        load(c, x);
        give(c, x);
    }
    __syncthreads();   // the row is written: its actions' places are now put right
    if (wave == 0 && real && keep) {
        float g = __builtin_amdgcn_exp2f((chosen - top) * kLog2e) * by;
        for (int j = 0; j < p.picks; ++j) g += places[j] == action ? slopes[j] : 0.f;
        to[action] = (T)g;
    }
}

template <typename T> int launch(const Batch& p, const void* logits, float* loss, float* logp, void* grad, hipStream_t stream) {
    const int most = p.width > p.picks ? p.width : p.picks;
    const int64_t pieces = (p.width + 16 / (int64_t)sizeof(T) - 1) / (16 / (int64_t)sizeof(T));
    const int g = most <= 16 ? 16 : (most <= 32 ? 32 : 64), each = 256 / g;
    const int64_t blocks = most <= 64 ? (p.rows + each - 1) / each : p.rows;
    if (!taser_launch_fits(blocks, most <= 64 || pieces <= 1024 ? 256 : 1024)) return taser_fail(TASER_E_RANGE, "policy_loss: too many rows for one launch");
    const dim3 grid((unsigned)blocks);
    TaserProfileSpan span(stream, "policy_loss");
    if (most <= 64) {
        if (g == 16) policy_window_kernel<T, 16><<<grid, 256, 0, stream>>>(p, (const T*)logits, loss, logp, (T*)grad);
        else if (g == 32) policy_window_kernel<T, 32><<<grid, 256, 0, stream>>>(p, (const T*)logits, loss, logp, (T*)grad);
        else policy_window_kernel<T, 64><<<grid, 256, 0, stream>>>(p, (const T*)logits, loss, logp, (T*)grad);
    } else {
        // Short rows are held by as few threads as it takes. Of longer ones as much as leaves registers for two blocks a compute unit, one writing
        // while the other reads: 64 001 bf16 logits 251 us for 4 096 rows, 274 with the whole row held by one block.
        if (pieces <= 256) policy_row_kernel<T, 256, 1><<<grid, 256, 0, stream>>>(p, (const T*)logits, loss, logp, (T*)grad);
        else if (pieces <= 1024) policy_row_kernel<T, 256, 4><<<grid, 256, 0, stream>>>(p, (const T*)logits, loss, logp, (T*)grad);
        else policy_row_kernel<T, 1024, (sizeof(T) == 2 ? 4 : 8)><<<grid, 1024, 0, stream>>>(p, (const T*)logits, loss, logp, (T*)grad);
    }
    TASER_HIP_TRY(hipGetLastError());
    return TASER_OK;
}

}  // namespace

extern "C" int taser_policy_loss(const taser_policy_batch* b, float* loss, float* logp, void* grad, void* hip_stream) {
    if (!b) return taser_fail(TASER_E_ARG, "policy_loss: null argument block");
    if (b->type < TASER_F32 || b->type > TASER_BF16) return taser_fail(TASER_E_ARG, "policy_loss: unknown element type %d", b->type);
    if (b->rows < 0 || b->width < 1 || b->picks < 1) return taser_fail(TASER_E_ARG, "policy_loss: negative number of rows, or no candidates or actions");
    if (b->picks > TASER_MAX_PICKS || b->width >= (int64_t)1 << 31 || b->rows >= (int64_t)1 << 31)
        return taser_fail(TASER_E_RANGE, "policy_loss: more than %d actions a row, or too many rows or candidates", TASER_MAX_PICKS);
    if (!(b->clip_low >= 0.f) || !(b->clip_high >= 0.f) || !(b->kl >= 0.f)) return taser_fail(TASER_E_ARG, "policy_loss: clip_low, clip_high and kl must not be negative");
    if (!b->rows) return TASER_OK;
    if (!b->logits || !b->actions || !b->advantage || !loss || !logp) return taser_fail(TASER_E_ARG, "policy_loss: null logits, actions, advantages or outputs");
    if (b->logits_stride < b->width && b->rows > 1) return taser_fail(TASER_E_ARG, "policy_loss: rows of logits overlap");
    const Batch p{b->picks, (int32_t)b->width, b->rows, b->logits_stride, b->count, b->actions, b->advantage, b->old_logp, b->ref_logp, b->weight, b->clip_low, b->clip_high, b->kl};
    hipStream_t stream = (hipStream_t)hip_stream;
    taser_clear_stale_hip_error();
    if (b->type == TASER_F32) return launch<float>(p, b->logits, loss, logp, grad, stream);
    if (b->type == TASER_F16) return launch<_Float16>(p, b->logits, loss, logp, grad, stream);
    return launch<__bf16>(p, b->logits, loss, logp, grad, stream);
}

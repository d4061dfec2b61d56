// Draws from a policy's logits with temperature, top-k, top-p and min-p, by given random numbers (taser_policy_draw).
//
// A candidate's weight w = exp((x - top) / temperature) is held as a whole number of 2^-43, so that sums have one value whatever their order, and
// thresholds and draws do not depend on how a row is cut. Nothing is sorted: top-k and top-p keep the candidates above a value, and the first few
// by index of those at it. The value is found by a histogram of counts (top-k) or weights (top-p) over 1024 bins of the distance to the largest
// logit, and within a bin over the logits' bits, until a bin has one value: mostly at once. A draw finds its piece of the row in the
// pieces' running sums, then its candidate in the piece.
//
// Rows of up to 64 candidates and draws: a part of a wave, a lane a candidate, whose rank comes from a look at every other one.
// Longer rows: a block, which holds the row in registers (up to 65536 logits in 16 bits, 32768 in 32; what is past them is read again for each pass).
#include "pieces.h"

namespace {

constexpr int kBits = 43;   // of a weight of 1
constexpr int kBins = 1024;
constexpr double kLog2e = 1.4426950408889634;

struct Draws {
    int32_t picks, width;
    int64_t rows, stride;
    const int32_t* count;
    const float* uniform;
    float temperature, top_p, min_p;
    int32_t top_k;
    const float *row_temperature, *row_top_p, *row_min_p;
    const int32_t* row_top_k;
};

// A row's settings.
struct Rule {
    bool greedy;
    double beta;      // w = 2^(-beta (top - x))
    int32_t top_k;    // 0: none
    uint64_t top_p;   // times 2^64; 0: none, 1 stands for the largest alone
    uint64_t least;   // the smallest weight that min_p keeps
};

__device__ inline int32_t taking_part(const Draws& p, int64_t row) {
    if (!p.count) return p.width;
    const int32_t n = p.count[row];
    return n < 0 ? 0 : (n > p.width ? p.width : n);
}
__device__ inline Rule rule_of(const Draws& p, int64_t row) {
    const float t = p.row_temperature ? p.row_temperature[row] : p.temperature, top_p = p.row_top_p ? p.row_top_p[row] : p.top_p, least = p.row_min_p ? p.row_min_p[row] : p.min_p;
    const int32_t k = p.row_top_k ? p.row_top_k[row] : p.top_k;
    Rule r;
    r.greedy = !(t > 0.f) || k == 1;
    r.beta = r.greedy ? 0. : kLog2e / (double)t;
    r.top_k = k > 0 ? k : 0;
    r.top_p = top_p >= 1.f ? 0 : top_p > 0.f ? (uint64_t)ldexp((double)top_p, 64) : 1;
    if (top_p < 1.f && !r.top_p) r.top_p = 1;
    if (top_p != top_p) r.top_p = 1;
    r.least = least > 0.f ? (uint64_t)ceil(ldexp((double)fminf(least, 1.f), kBits)) : 0;
    return r;
}

__device__ inline uint64_t weight_of(const Rule& r, float top, float x) {
    if (x == -INFINITY) return 0;
    return (uint64_t)rint(ldexp(exp2(-((double)top - (double)x) * r.beta), kBits));
}

// A share of a sum, rounded up; and the place of a number in [0, 1) in it, rounded down.
__device__ inline uint64_t share_of(uint64_t share, uint64_t sum) { return __umul64hi(share, sum) + (share * sum ? 1 : 0); }
__device__ inline uint64_t place_of(float u, uint64_t sum) {
    const uint64_t bits = u < 1.f ? (u > 0.f ? (uint64_t)ldexp((double)u, 64) : 0) : ~0ull;   // (NaN: as 1)
    return __umul64hi(bits, sum);
}

__device__ inline uint64_t shuffle(uint64_t x, int lane, int width = 64) {
    return (uint64_t)__shfl((uint32_t)(x >> 32), lane, width) << 32 | __shfl((uint32_t)x, lane, width);
}
__device__ inline uint64_t shuffle_up(uint64_t x, int by, int width = 64) {
    return (uint64_t)__shfl_up((uint32_t)(x >> 32), by, width) << 32 | __shfl_up((uint32_t)x, by, width);
}
__device__ inline uint64_t shuffle_xor(uint64_t x, int mask) { return (uint64_t)__shfl_xor((uint32_t)(x >> 32), mask) << 32 | __shfl_xor((uint32_t)x, mask); }
template <int G> __device__ inline uint64_t sum_of(uint64_t x) {
#pragma unroll
    for (int m = 1; m < G; m <<= 1) x += shuffle_xor(x, m);
    return x;
}
template <int G> __device__ inline uint64_t running(uint64_t x) {   // inclusive
    const int lane = threadIdx.x % G;
#pragma unroll
    for (int by = 1; by < G; by <<= 1) {
        const uint64_t y = shuffle_up(x, by, G);
        if (lane >= by) x += y;
    }
    return x;
}

// Rows of at most 64 candidates and draws: G lanes a row.
template <typename T, int G> __global__ __launch_bounds__(256) void draw_window_kernel(const Draws p, const T* logits, int32_t* actions, float* logp) {
    const int64_t row = (int64_t)blockIdx.x * (256 / G) + threadIdx.x / G;
    const int lane = threadIdx.x % G, first = threadIdx.x & 63 & ~(G - 1);
    if (row >= p.rows) return;   // the lanes of a row leave together
    constexpr uint64_t lanes = G == 64 ? ~0ull : (1ull << (G & 63)) - 1;
    auto ballot = [&](bool yes) { return __ballot(yes) >> first & lanes; };
    const int n = taking_part(p, row);
    const Rule rule = rule_of(p, row);
    const float x = lane < n ? (float)logits[row * p.stride + lane] : -INFINITY;
    const bool bad = ballot(x != x || x == INFINITY);
    float top = x;
#pragma unroll
    for (int m = 1; m < G; m <<= 1) top = fmaxf(top, __shfl_xor(top, m, G));
    const bool none = bad || top == -INFINITY;
    float total = x > -INFINITY ? expf(x - top) : 0.f;
#pragma unroll
    for (int m = 1; m < G; m <<= 1) total += __shfl_xor(total, m, G);
    uint64_t w;
    if (rule.greedy) {
        w = lane == __ffsll((long long)ballot(x == top)) - 1 ? 1 : 0;
    } else {
        w = weight_of(rule, top, x);
        bool keep = w >= rule.least;
        if (rule.top_k || rule.top_p) {
            int rank = 0;
            uint64_t before = 0;
            for (int j = 0; j < n; ++j) {
                const float other = __shfl(x, j, G);
                const uint64_t weight = shuffle(w, j, G);
                const bool ahead = other > x || (other == x && j < lane);
                rank += ahead;
                before += ahead ? weight : 0;
            }
            const bool in = !rule.top_k || rank < rule.top_k;
            const uint64_t share = share_of(rule.top_p, sum_of<G>(in ? w : 0));
            keep = keep && in && (!rule.top_p || rank == 0 || before < share);
        }
        w = keep ? w : 0;
    }
    const uint64_t upto = running<G>(w), whole = shuffle(upto, G - 1, G);
    const int64_t at = row * p.picks + lane;
    const uint64_t place = lane < p.picks ? place_of(p.uniform[at], whole) : 0;
    int action = -1;
    for (int j = 0; j < p.picks; ++j) {
        const uint64_t hit = ballot(upto > shuffle(place, j, G));
        if (lane == j) action = __ffsll((long long)hit) - 1;
    }
    const float chosen = __shfl(x, action < 0 ? 0 : action, G);
    if (lane >= p.picks) return;
    actions[at] = none ? -1 : action;
    logp[at] = bad ? __builtin_nanf("") : none ? 0.f : (chosen - top) - logf(total);
}

// Numbers in the order of the floats (no NaN).
__device__ inline uint32_t order_of(float x) {
    const uint32_t b = __float_as_uint(x);
    return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ inline float float_of(uint32_t order) { return __uint_as_float(order ^ ((order >> 31) ? 0x80000000u : 0xffffffffu)); }

template <typename T, int THREADS, int HELD> __global__ __launch_bounds__(THREADS) void draw_row_kernel(const Draws p, const T* logits, int32_t* actions, float* logp) {
    constexpr int EACH = kTaserEach<T>, WAVES = THREADS / 64, STEP = THREADS * EACH;
    extern __shared__ uint64_t running_sums[];   // of each wave's pieces, in the order of their candidates
    __shared__ uint64_t bins[kBins];
    __shared__ double powers[256];               // 2^(kBits - i / 256)
    __shared__ uint64_t found_before, found_sum;
    __shared__ float tops[WAVES], totals[WAVES];
    __shared__ uint32_t counts[WAVES], bads[WAVES], lowest, highest, found_bin, cut_at;
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = taking_part(p, row);
    const Rule rule = rule_of(p, row);
    const T* from = logits + row * p.stride;
    const int chunks = (n + STEP - 1) / STEP, pieces = chunks * WAVES;

    // -0 is taken as 0: they are equal.
    auto load = [&](int64_t c, TaserPiece<T>& x) { taser_load_piece<T>(from, c, n, (T)-INFINITY, x); };
    TaserPiece<T> held[HELD];
#pragma unroll
    for (int h = 0; h < HELD; ++h) load((int64_t)h * STEP + threadIdx.x * EACH, held[h]);
    // take(chunk, first candidate, logits) for the row's pieces; whole waves come together.
    auto each = [&](auto&& take) {
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
            if (h >= chunks) break;
            // (What one pass makes of a piece is not kept for the next: it would not fit.)
            uint32_t words[4];
            __builtin_memcpy(words, held[h].x, 16);
            asm volatile("" : "+v"(words[0]), "+v"(words[1]), "+v"(words[2]), "+v"(words[3]));
            TaserPiece<T> x;
            __builtin_memcpy(x.x, words, 16);
            float v[EACH];
#pragma unroll
            for (int i = 0; i < EACH; ++i) v[i] = (float)x.x[i] + 0.f;
            take(h, h * STEP + (int)threadIdx.x * EACH, v);
            __builtin_amdgcn_sched_barrier(0);   // pieces one by one: side by side they would need more registers than there are
        }
        for (int h = HELD; h < chunks; ++h) {
            TaserPiece<T> x;
            load((int64_t)h * STEP + threadIdx.x * EACH, x);
            float v[EACH];
#pragma unroll
            for (int i = 0; i < EACH; ++i) v[i] = (float)x.x[i] + 0.f;
            take(h, h * STEP + (int)threadIdx.x * EACH, v);
        }
    };

    float top = -INFINITY;
    uint32_t finite = 0, bad = 0;
    each([&](int, int, const float (&v)[EACH]) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            top = fmaxf(top, v[i]);
            finite += v[i] > -INFINITY;
            bad |= !(v[i] < INFINITY);
        }
    });
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        top = fmaxf(top, __shfl_xor(top, m));
        finite += __shfl_xor(finite, m);
        bad |= __shfl_xor(bad, m);
    }
    if (lane == 0) {
        tops[wave] = top;
        counts[wave] = finite;
        bads[wave] = bad;
    }
    if (threadIdx.x < 256) powers[threadIdx.x] = exp2(kBits - threadIdx.x / 256.);
    if (threadIdx.x == 0) cut_at = 0xffffffffu;
    __syncthreads();
    finite = bad = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        top = fmaxf(top, tops[w]);
        finite += counts[w];
        bad |= bads[w];
    }
    if (bad || !finite) {   // the whole block
        for (int j = threadIdx.x; j < p.picks; j += THREADS) {
            actions[row * p.picks + j] = -1;
            logp[row * p.picks + j] = bad ? __builtin_nanf("") : 0.f;
        }
        return;
    }
    float total = 0.f;
    each([&](int, int, const float (&v)[EACH]) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) total += __builtin_amdgcn_exp2f((v[i] - top) * (float)kLog2e);
    });
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) total += __shfl_xor(total, m);
    if (lane == 0) totals[wave] = total;
    // (read behind a later barrier)

    // 2^-y by a table of 256 powers and a series for the rest, |rest| <= 2^-9: 2^-42 off.
    const double beta = rule.beta * 256.;
    auto weight = [&](float x) -> uint64_t {
        const double y = fmin(((double)top - (double)x) * beta, 60. * 256.), z = rint(y), r = (y - z) * (-0.6931471805599453 / 256.);
        const int j = (int)z;
        const double e = powers[j & 255] * (1. + r * (1. + r * (0.5 + r * (1. / 6.))));
        return (uint64_t)__double_as_longlong(ldexp(e, -(j >> 8)) + 4503599627370496.) - 0x4330000000000000ull;   // 2^52 more: rounded to a whole number
    };

    float limit = -INFINITY;   // kept are those above it, and those at it up to the candidate cut
    uint32_t cut = 0xffffffffu;
    uint64_t at_limit = 0;     // how many of those at it, in the order of their candidates
    if (rule.greedy) {
        uint32_t mine = 0xffffffffu;
        each([&](int, int c, const float (&v)[EACH]) {
#pragma unroll
            for (int i = EACH - 1; i >= 0; --i) mine = v[i] == top && (uint32_t)(c + i) < mine ? (uint32_t)(c + i) : mine;
        });
        atomicMin(&cut_at, mine);
        __syncthreads();
        const int action = (int)cut_at;
        total = 0.f;
        for (int w = 0; w < WAVES; ++w) total += totals[w];
        for (int j = threadIdx.x; j < p.picks; j += THREADS) {
            actions[row * p.picks + j] = action;
            logp[row * p.picks + j] = -logf(total);
        }
        return;
    }

    // The value at which the numbers of candidates (or, `weigh`, their weights) above `limit` come to the target, from the largest down, and
    // what comes before it. target(sum of all): 0 if it is not among them.
    const float scale = (float)(rule.beta * (kBins / 40.));
    auto bin_of = [&](float x) { return (int)fminf((top - x) * scale, (float)(kBins - 1)); };
    auto clear = [&]() {
        for (int i = threadIdx.x; i < kBins; i += THREADS) bins[i] = 0;
        if (threadIdx.x == 0) {
            lowest = 0xffffffffu;
            highest = 0;
        }
        __syncthreads();
    };
    auto find = [&](auto&& target) {   // wave 0: the bin
        __syncthreads();
        if (wave == 0) {
            uint64_t mine[kBins / 64], sum = 0;
#pragma unroll
            for (int i = 0; i < kBins / 64; ++i) sum += mine[i] = bins[lane * (kBins / 64) + i];
            const uint64_t upto = running<64>(sum), all = shuffle(upto, 63), wanted = target(all);
            const uint64_t hit = __ballot(upto >= wanted);
            if (lane == 0) found_sum = wanted;
            if (wanted && lane == __ffsll((long long)hit) - 1) {
                uint64_t before = upto - sum;
                int b = 0;
#pragma unroll
                for (int i = 0; i < kBins / 64 - 1; ++i) {
                    const bool past = b == i && before + mine[i] < wanted;
                    before += past ? mine[i] : 0;
                    b += past;
                }
                found_bin = lane * (kBins / 64) + b;
                found_before = before;
            }
        }
        __syncthreads();
    };
    auto narrow = [&](uint32_t& low, uint32_t& high, auto&& inside) {   // to the smallest and largest there are
        uint32_t a = 0xffffffffu, b = 0;
        each([&](int, int, const float (&v)[EACH]) {
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                const uint32_t o = order_of(v[i]);
                if (inside(v[i], o)) {
                    a = o < a ? o : a;
                    b = o > b ? o : b;
                }
            }
        });
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            const uint32_t x = __shfl_xor(a, m), y = __shfl_xor(b, m);
            a = x < a ? x : a;
            b = y > b ? y : b;
        }
        if (lane == 0 && b) {
            atomicMin(&lowest, a);
            atomicMax(&highest, b);
        }
        __syncthreads();
        low = lowest;
        high = highest;
        __syncthreads();
    };
    auto select = [&](auto&& amount, auto&& target, float& value, uint64_t& before, uint64_t& wanted) {
        clear();
        const float above = limit;
        each([&](int, int, const float (&v)[EACH]) {
#pragma unroll
            for (int i = 0; i < EACH; ++i)
                if (v[i] > above) atomicAdd((unsigned long long*)&bins[bin_of(v[i])], (unsigned long long)amount(v[i]));
        });
        find(target);
        wanted = found_sum;
        if (!wanted) return;
        before = found_before;
        const int bin = (int)found_bin;
        uint32_t low, high;
        narrow(low, high, [&](float x, uint32_t) { return x > above && bin_of(x) == bin; });
        while (low != high) {
            const int shift = 32 - __clz(high - low) > 10 ? 32 - __clz(high - low) - 10 : 0;
            clear();
            each([&](int, int, const float (&v)[EACH]) {
#pragma unroll
                for (int i = 0; i < EACH; ++i) {
                    const uint32_t o = order_of(v[i]);
                    if (o >= low && o <= high) atomicAdd((unsigned long long*)&bins[(high - o) >> shift], (unsigned long long)amount(v[i]));
                }
            });
            const uint64_t rest = wanted - before;
            find([&](uint64_t) { return rest; });
            before += found_before;
            high -= found_bin << shift;
            const uint32_t down = high - ((1u << shift) - 1);
            low = down > low && down <= high ? down : low;
            if (shift) narrow(low, high, [&](float, uint32_t o) { return o >= low && o <= high; });
        }
        value = float_of(high);
    };

    if (rule.top_k && (uint32_t)rule.top_k < finite) {
        uint64_t before, wanted;
        float value;
        select([](float) { return (uint64_t)1; }, [&](uint64_t) { return (uint64_t)rule.top_k; }, value, before, wanted);
        limit = value;
        at_limit = wanted - before;
    }
    if (rule.top_p) {
        const uint64_t one = at_limit ? weight(limit) : 0, rest = at_limit * one;
        uint64_t sum_above = 0, before, wanted;
        float value;
        // The share of all that are left; where it is past those above the limit, as many at it as it takes.
        uint64_t beyond = 0;
        auto target = [&](uint64_t sum) {
            const uint64_t all = share_of(rule.top_p, sum + rest), least = all ? all : 1;
            beyond = least > sum ? least - sum : 0;
            return beyond ? 0 : least;
        };
        select(weight, target, value, before, wanted);
        if (wanted) {
            const uint64_t w = weight(value);
            limit = value;
            at_limit = (wanted - before + w - 1) / w;
        } else {
            if (threadIdx.x == 0) found_before = beyond;   // wave 0 has it
            __syncthreads();
            at_limit = (found_before + one - 1) / one;
        }
        (void)sum_above;
    }
    if (at_limit) {   // where fewer than there are at the limit are kept: up to which candidate
        each([&](int h, int, const float (&v)[EACH]) {
            int here = 0;
#pragma unroll
            for (int i = 0; i < EACH; ++i) here += __popcll(__ballot(v[i] == limit));
            if (lane == 0) running_sums[h * WAVES + wave] = here;
        });
        __syncthreads();
        if (wave == 0) {
            uint64_t before = 0;
            for (int s = 0; s < pieces; s += 64) {
                const uint64_t mine = s + lane < pieces ? running_sums[s + lane] : 0, upto = before + running<64>(mine);
                const uint64_t hit = __ballot(upto >= at_limit);
                if (hit) {
                    const int at = __ffsll((long long)hit) - 1;
                    uint64_t left = at_limit - shuffle(upto - mine, at);   // the left-th one of piece s + at
                    const int c = (s + at) / WAVES * STEP + ((s + at) % WAVES * 64 + lane) * EACH;
                    TaserPiece<T> x;
                    load(c, x);
                    uint32_t here = 0;
#pragma unroll
                    for (int i = 0; i < EACH; ++i) here += (float)x.x[i] + 0.f == limit;
                    uint64_t past = running<64>(here) - here;
#pragma unroll
                    for (int i = 0; i < EACH; ++i) {
                        past += (float)x.x[i] + 0.f == limit;
                        if ((float)x.x[i] + 0.f == limit && past == left) cut_at = c + i;
                    }
                    break;
                }
                before = shuffle(upto, 63);
            }
        }
        __syncthreads();
        cut = cut_at;
    }
    auto kept_weight = [&](float x, int c) -> uint64_t {
        if (!(x > limit || (x == limit && at_limit && (uint32_t)c <= cut))) return 0;
        const uint64_t w = weight(x);
        return w >= rule.least ? w : 0;
    };
    each([&](int h, int c, const float (&v)[EACH]) {
        uint64_t sum = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) sum += kept_weight(v[i], c + i);
        if (__ballot(sum != 0)) sum = sum_of<64>(sum);
        if (lane == 0) running_sums[h * WAVES + wave] = sum;
    });
    __syncthreads();
    if (wave == 0) {
        uint64_t before = 0;
        for (int s = 0; s < pieces; s += 64) {
            const uint64_t upto = before + running<64>(s + lane < pieces ? running_sums[s + lane] : 0);
            if (s + lane < pieces) running_sums[s + lane] = upto;
            before = shuffle(upto, 63);
        }
    }
    __syncthreads();
    total = 0.f;
    for (int w = 0; w < WAVES; ++w) total += totals[w];
    const uint64_t whole = running_sums[pieces - 1];
    for (int j = wave; j < p.picks; j += WAVES) {
        const uint64_t place = place_of(p.uniform[row * p.picks + j], whole);
        int at = 0;
        for (int s = 0; s < pieces; s += 64) {
            const uint64_t hit = __ballot(s + lane < pieces && running_sums[s + lane] > place);
            if (hit) {
                at = s + __ffsll((long long)hit) - 1;
                break;
            }
        }
        const int c = at / WAVES * STEP + (at % WAVES * 64 + lane) * EACH;
        TaserPiece<T> x;
        load(c, x);
        uint64_t w[EACH], sum = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) sum += w[i] = kept_weight((float)x.x[i] + 0.f, c + i);
        uint64_t upto = (at ? running_sums[at - 1] : 0) + running<64>(sum);
        const uint64_t hit = __ballot(upto > place);
        if (lane != __ffsll((long long)hit) - 1) continue;
        upto -= sum;
        bool done = false;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            upto += w[i];
            if (!done && upto > place) {
                done = true;
                actions[row * p.picks + j] = c + i;
                logp[row * p.picks + j] = ((float)x.x[i] - top) - logf(total);
            }
        }
    }
}

template <typename T> int launch(const Draws& p, const void* logits, int32_t* actions, float* logp, hipStream_t stream) {
    const int most = p.width > p.picks ? p.width : p.picks;
    const int64_t pieces = (p.width + kTaserEach<T> - 1) / kTaserEach<T>;
    const int g = most <= 16 ? 16 : (most <= 32 ? 32 : 64), each = 256 / g, threads = most <= 64 || pieces <= 1024 ? 256 : 1024;
    const int64_t blocks = most <= 64 ? (p.rows + each - 1) / each : p.rows;
    if (!taser_launch_fits(blocks, threads)) return taser_fail(TASER_E_RANGE, "policy_draw: too many rows for one launch");
    const unsigned grid = (unsigned)blocks, sums = (unsigned)((pieces + threads - 1) / threads * (threads / 64) * sizeof(uint64_t));
    TaserProfileSpan span(stream, "policy_draw");
    if (most <= 64) {
        if (g == 16) draw_window_kernel<T, 16><<<grid, 256, 0, stream>>>(p, (const T*)logits, actions, logp);
        else if (g == 32) draw_window_kernel<T, 32><<<grid, 256, 0, stream>>>(p, (const T*)logits, actions, logp);
        else draw_window_kernel<T, 64><<<grid, 256, 0, stream>>>(p, (const T*)logits, actions, logp);
    } else if (threads == 256) {
        draw_row_kernel<T, 256, 4><<<grid, 256, sums, stream>>>(p, (const T*)logits, actions, logp);
    } else {
        draw_row_kernel<T, 1024, 8><<<grid, 1024, sums, stream>>>(p, (const T*)logits, actions, logp);
    }
    TASER_HIP_TRY(hipGetLastError());
    return TASER_OK;
}

int check(const taser_policy_draws* b) {
    if (!b) return taser_fail(TASER_E_ARG, "policy_draw: null argument block");
    if (b->type < TASER_F32 || b->type > TASER_BF16) return taser_fail(TASER_E_ARG, "policy_draw: unknown element type %d", b->type);
    if (b->rows < 0 || b->width < 1 || b->picks < 1) return taser_fail(TASER_E_ARG, "policy_draw: negative number of rows, or no candidates or draws");
    if (b->picks > TASER_MAX_PICKS || b->width > TASER_MAX_DRAW_WIDTH || b->rows >= (int64_t)1 << 31)
        return taser_fail(TASER_E_RANGE, "policy_draw: more than %d draws a row, or too many rows or candidates", TASER_MAX_PICKS);
    if ((!b->row_temperature && !(b->temperature >= 0.f)) || (!b->row_top_k && b->top_k < 0) || (!b->row_top_p && !(b->top_p >= 0.f && b->top_p <= 1.f)) ||
        (!b->row_min_p && !(b->min_p >= 0.f && b->min_p <= 1.f)))
        return taser_fail(TASER_E_ARG, "policy_draw: temperature and top_k must not be negative, top_p and min_p lie in [0, 1]");
    if (b->rows > 1 && b->logits_stride < b->width) return taser_fail(TASER_E_ARG, "policy_draw: rows of logits overlap");
    return TASER_OK;
}

}  // namespace

extern "C" int taser_policy_draw_bytes(const taser_policy_draws* b, uint64_t* work_bytes) {
    if (const int rc = check(b)) return rc;
    if (!work_bytes) return taser_fail(TASER_E_ARG, "policy_draw_bytes: null output");
    *work_bytes = 0;
    return TASER_OK;
}

extern "C" int taser_policy_draw(const taser_policy_draws* b, int32_t* actions, float* logp, void* work, uint64_t work_bytes, void* hip_stream) {
    if (const int rc = check(b)) return rc;
    if (!b->rows) return TASER_OK;
    if (!b->logits || !b->uniform || !actions || !logp) return taser_fail(TASER_E_ARG, "policy_draw: null logits, random numbers or outputs");
    const Draws p{b->picks, (int32_t)b->width, b->rows, b->logits_stride, b->count, b->uniform, b->temperature, b->top_p, b->min_p, b->top_k,
                  b->row_temperature, b->row_top_p, b->row_min_p, b->row_top_k};
    hipStream_t stream = (hipStream_t)hip_stream;
    taser_clear_stale_hip_error();
    if (b->type == TASER_F32) return launch<float>(p, b->logits, actions, logp, stream);
    if (b->type == TASER_F16) return launch<_Float16>(p, b->logits, actions, logp, stream);
    return launch<__bf16>(p, b->logits, actions, logp, stream);
}

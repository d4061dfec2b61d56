// Draws from a policy's logits with temperature, top-k, top-p and min-p, by given random numbers (taser_policy_draw).
//
// A candidate's weight w = exp((x - top) / temperature) is held as a whole number of 2^-43, so that sums have one value whatever their order, and
// thresholds and draws do not depend on how a row is cut. Nothing is sorted: top-k and top-p keep the candidates above a value, and the first few
// by index of those at it. The value is found by a histogram of counts (top-k) or weights (top-p) over 1024 bins of the distance to the largest
// logit, and within a bin over the logits' bits, until a bin has one value: mostly at once. A draw finds its piece of the row in the
// pieces' running sums, then its candidate in the piece. Short lists around the threshold are ranked by comparing all pairs.
//
// Rows of up to 64 candidates and draws: a part of a wave, a lane a candidate, whose rank comes from a look at every other one.
// Longer rows: a block of 512 threads, three of them a compute unit; few of them: slices, four launches. Bound by the vector units: weights take some 20
// instructions a candidate, twice where top-p looks for its threshold. 4096 x 64 001 bf16: top-p 0.95 555 us, top-k 50 with top-p 318, neither 281, the largest
// 183 (the logits alone 102); 1 x 64 001 with both 20, 64 x 130 000 f32 with top-p 53. (All on a card at its clock: the first 25 ms after a rest take up to a quarter more.)
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
// x of the lane that a DPP control names, 0 where there is none.
template <int CONTROL, int ROWS> __device__ inline uint64_t moved(uint64_t x) {
    const uint32_t low = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, CONTROL, ROWS, 0xf, true), high = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(x >> 32), CONTROL, ROWS, 0xf, true);
    return (uint64_t)high << 32 | low;
}
// Sums up to each lane of a group of G.
template <int G> __device__ inline uint64_t running(uint64_t x) {
    x += moved<0x111, 0xf>(x);   // within rows of 16: from 1, 2, 4 and 8 lanes below
    x += moved<0x112, 0xf>(x);
    x += moved<0x114, 0xf>(x);
    x += moved<0x118, 0xf>(x);
    if (G >= 32) x += moved<0x142, 0xa>(x);   // the row below's last
    if (G == 64) x += moved<0x143, 0xc>(x);   // the lower half's last
    return x;
}
// The largest of a wave's, in the last lane.
__device__ inline uint32_t largest(uint32_t x) {
    auto with = [&](uint32_t y) { x = y > x ? y : x; };
    with(__builtin_amdgcn_update_dpp(0, (int)x, 0x111, 0xf, 0xf, true));
    with(__builtin_amdgcn_update_dpp(0, (int)x, 0x112, 0xf, 0xf, true));
    with(__builtin_amdgcn_update_dpp(0, (int)x, 0x114, 0xf, 0xf, true));
    with(__builtin_amdgcn_update_dpp(0, (int)x, 0x118, 0xf, 0xf, true));
    with(__builtin_amdgcn_update_dpp(0, (int)x, 0x142, 0xa, 0xf, true));
    with(__builtin_amdgcn_update_dpp(0, (int)x, 0x143, 0xc, 0xf, true));
    return x;
}
template <int G> __device__ inline uint64_t sum_of(uint64_t x) { return shuffle(running<G>(x), G - 1, G); }

// Rows of at most 64 candidates and draws: G lanes a row.
template <typename T, int G> __global__ __launch_bounds__(256) void draw_window_kernel(const Draws p, const T* logits, int32_t* actions, float* logp) {
    struct __attribute__((aligned(16))) Candidate {
        float x;
        uint64_t w;
    };
    __shared__ Candidate seen[256];   // each lane's, for the others of its row: one LDS read a look, where lanes asked for by number are three
    __shared__ uint64_t sums[256];
    const int64_t row = (int64_t)blockIdx.x * (256 / G) + threadIdx.x / G;
    const int lane = threadIdx.x % G, first = threadIdx.x & 63 & ~(G - 1), row_at = threadIdx.x - lane;
    if (row >= p.rows) return;   // the lanes of a row leave together
    // What this wave wrote to LDS is there for it to read.
    auto written = [] {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
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
            seen[threadIdx.x] = Candidate{x, w};
            written();
#pragma unroll 4
            for (int j = 0; j < n; ++j) {
                const Candidate other = seen[row_at + j];
                const bool ahead = other.x > x || (other.x == x && j < lane);
                rank += ahead;
                before += ahead ? other.w : 0;
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
    sums[threadIdx.x] = upto;
    written();
    int action = 0;   // the first sum past the place: they ascend
#pragma unroll
    for (int step = G / 2; step; step >>= 1) action += sums[row_at + action + step - 1] <= place ? step : 0;
    const float chosen = __shfl(x, action, G);
    if (lane >= p.picks) return;
    actions[at] = none ? -1 : action;
    logp[at] = bad ? __builtin_nanf("") : none ? 0.f : (chosen - top) - logf(total);
}

// Numbers in the order of the floats (no NaN).
__device__ inline uint32_t order_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);   // -0 is 0: they are equal
    return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ inline float float_of(uint32_t order) { return __uint_as_float(order ^ ((order >> 31) ? 0x80000000u : 0xffffffffu)); }

// ---- longer rows -----------------------------------------------------------------------------------

constexpr int kGapped = kBins + kBins / 16;   // bins in LDS: every 16, which a lane adds up, are followed by a gap, so that lanes read from different banks
__device__ inline int bin_at(int bin) { return bin + (bin >> 4); }

__device__ inline bool wants_number(const Rule& rule, int n) { return !rule.greedy && rule.top_k && rule.top_k < n; }
// The softmax's sum is the weights' at a temperature of 1, where all are added up.
__device__ inline bool by_weights(const Rule& rule, int n) { return !rule.greedy && rule.beta == kLog2e && !wants_number(rule, n) && (rule.top_p || !rule.least); }

// A row's logits as distances to the largest and as weights.
template <typename T> struct Row {
    static constexpr int EACH = kTaserEach<T>;
    const T* from;
    int n;
    float top, scale;       // scale: bins of a distance of 1, 32 for candidates by number, 32 to a power of two of weight for weights
    double beta;            // 256 times the rule's
    const double* powers;   // in LDS: 2^(kBits + i / 256)

    __device__ Row(const Draws& p, const T* logits, int64_t row, const Rule& rule, const double* powers)
        : from(logits + row * p.stride), n(taking_part(p, row)), top(0.f), scale(wants_number(rule, n) ? 32.f : by_weight(rule)), beta(rule.beta * 256.), powers(powers) {}
    __device__ static float by_weight(const Rule& rule) { return (float)fmin(rule.beta * 32., 1e30); }   // finite: the largest logit's distance is 0 at any temperature
    __device__ static void fill(double* powers) {
        for (int i = threadIdx.x; i < 256; i += blockDim.x) powers[i] = exp2(kBits + i / 256.);
    }
    __device__ void load(int64_t c, float (&v)[EACH]) const {
        TaserPiece<T> x;
        taser_load_piece<T>(from, c, n, (T)-INFINITY, x);
#pragma unroll
        for (int i = 0; i < EACH; ++i) v[i] = (float)x.x[i];
    }
    // In bins; past the floats, or NaN (minus infinity at a temperature of infinity): the last. It falls as logits rise, roundings included.
    __device__ float distance(float x) const { return fminf((top - x) * scale, (float)(kBins - 1)); }
    // 2^y, y <= 0, by a table of 256 powers and a series for the rest, |rest| <= 2^-9: 2^-42 off. (The whole part of 256 y is read off a sum with 1.5 2^52.)
    __device__ uint64_t weight(float x) const {
        const double y = fmax(((double)x - (double)top) * beta, -60. * 256.), up = y + 6755399441055744., r = y - (up - 6755399441055744.);
        constexpr double c = 0.6931471805599453 / 256.;
        const int j = (int)__double2loint(up);
        const double e = powers[j & 255] * fma(fma(fma(r, c * c * c / 6., c * c / 2.), r, c), r, 1.);
        const double w = __hiloint2double(__double2hiint(e) + ((j >> 8) << 20), __double2loint(e));   // by 2^-60 at least: no exponent runs out
        const double whole = w + 4503599627370496.;   // 2^52 more: rounded to a whole number
        return (uint64_t)(uint32_t)(__double2hiint(whole) - 0x43300000) << 32 | (uint32_t)__double2loint(whole);
    }
    // The smallest logit closer than so many bins.
    __device__ float closer(float bins_away) const {
        if (!(bins_away > 0.f)) return INFINITY;
        if (bins_away >= (float)kBins) return -3.402823466e38f;
        const int lane = threadIdx.x & 63;
        uint32_t low = order_of(-3.402823466e38f), high = order_of(top);   // the top is
        while (low < high) {   // 64 places at a time, the last at `high`
            const uint32_t step = (high - low) / 64 + 1, place = high - low < step * (63 - lane) ? low : high - step * (63 - lane);
            const int hit = __ffsll((long long)__ballot(distance(float_of(place)) < bins_away)) - 1;
            low = hit ? __builtin_amdgcn_readlane(place, hit - 1) + 1 : low;
            high = __builtin_amdgcn_readlane(place, hit);
        }
        return float_of(high);
    }
    __device__ static float soft(float top, const float (&v)[EACH]) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < EACH; ++i) sum += __builtin_amdgcn_exp2f((v[i] - top) * (float)kLog2e);
        return sum;
    }
    // Candidates, or their weights, by distance.
    template <typename F> __device__ void count_in(uint64_t* bins, const float (&v)[EACH], F&& amount) const {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            if (EACH == 8 && i == 4) __builtin_amdgcn_sched_barrier(0);   // four weights at a time: eight need more registers than there are
            atomicAdd((unsigned long long*)&bins[bin_at((int)distance(v[i]))], (unsigned long long)amount(v[i]));
        }
    }
    // A piece's weights of the logits that are kept for sure, those that min_p leaves; in the last lane.
    template <typename F> __device__ uint64_t sure(const float (&v)[EACH], uint64_t least, F&& kept) const {
        bool some = false;
#pragma unroll
        for (int i = 0; i < EACH; ++i) some |= kept(v[i]);
        uint64_t sum = 0;
        if (!__ballot(some)) return 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            if (EACH == 8 && i == 4) __builtin_amdgcn_sched_barrier(0);
            const uint64_t w = weight(v[i]);
            sum += kept(v[i]) && w >= least ? w : 0;
        }
        return running<64>(sum);
    }
};

// Logits that are to be looked at go to the list, as many as it takes; `listed` counts all.
template <int EACH, typename F> __device__ inline void enlist(int64_t c, const float (&v)[EACH], uint64_t* list, uint32_t most, uint32_t* listed, F&& between) {
    uint64_t those[EACH];
    uint32_t count = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        those[i] = __ballot(between(v[i]));
        count += (uint32_t)__popcll(those[i]);
    }
    if (!count) return;
    uint32_t at = 0;
    if ((threadIdx.x & 63) == 0) at = atomicAdd(listed, count);
    at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        if (!those[i]) continue;
        const uint32_t to = at + __builtin_amdgcn_mbcnt_hi((uint32_t)(those[i] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)those[i], 0));
        if (between(v[i]) && to < most) list[to] = (uint64_t)__float_as_uint(v[i]) << 32 | (uint32_t)(c + i);
        at += (uint32_t)__popcll(those[i]);
    }
}

struct Found {
    uint64_t before, wanted, all;
    uint32_t bin, upto;
};
// The first bin at which the bins' sum comes to target(sum of all), what comes before it and, in 32 bits, what with it (a target of 0, or past the sum: none). By
// wave 0, which leaves the bins empty.
template <typename F> __device__ inline void find_bin(uint64_t* bins, Found* found, F&& target) {
    __syncthreads();
    if (threadIdx.x < 64) {
        const int lane = threadIdx.x;
        uint64_t mine[kBins / 64], sum = 0;
#pragma unroll
        for (int i = 0; i < kBins / 64; ++i) {
            sum += mine[i] = bins[bin_at(lane * (kBins / 64) + i)];
            bins[bin_at(lane * (kBins / 64) + i)] = 0;
        }
        const uint64_t upto = running<64>(sum), all = shuffle(upto, 63), asked = target(all), wanted = asked <= all ? asked : 0;
        const uint64_t hit = __ballot(upto >= wanted);
        if (lane == 0) {
            found->wanted = wanted;
            found->all = all;
        }
        if (wanted && lane == __ffsll((long long)hit) - 1) {
            uint64_t before = upto - sum, here = mine[0];
            int b = 0;
#pragma unroll
            for (int i = 0; i < kBins / 64 - 1; ++i) {
                const bool past = b == i && before + here < wanted;
                before += past ? here : 0;
                here = past ? mine[i + 1] : here;
                b += past;
            }
            found->bin = lane * (kBins / 64) + b;
            found->before = before;
            found->upto = (uint32_t)(before + here < 0xffffffffu ? before + here : 0xffffffffu);
        }
    }
    __syncthreads();
}

// What a first look at a row, a histogram of its candidates (top-k) or of their weights (top-p), leaves open: candidates of a distance below `near` are
// kept, those from `far` on are not, those between are looked at one by one.
struct Open {
    float near, far;
    uint64_t more;    // by number (top-k), or by weight (top-p alone), the best of those between are kept
    uint32_t number;  // whether there is a top-k of fewer than there are
    uint32_t all;     // whether those between are all that may be kept
};
constexpr uint32_t kListed = 2048;   // looked at one by one, in LDS and in the workspace
__device__ inline Open open_by(const Rule& rule, bool number, const Found& found) {
    // Both: the row's best by number are looked at one by one, then the share of those.
    const bool all = number && (rule.top_p || found.upto <= kListed);
    return Open{all ? -1.f : (float)found.bin, (float)(found.bin + 1), all ? found.wanted : found.wanted - found.before, number, all};
}

// A row cut into slices, each a block's, for calls of few rows: the largest logit; the histogram; what is kept for sure and what is looked at. Each
// is a launch: a block sees the others' results only in the next.
struct Slices {
    int32_t slices, span, pieces;   // of a row; span: chunks of a slice, 256 threads' pieces each
    uint64_t stride;                // of a row's part of the workspace, in numbers of 64 bits: [kBins] bins, [kListed] candidates, [pieces] sums, then
                                    // {listed, lowest}, Open, the weights' sum, [slices] {largest (NaN: one is not a number, or plus infinity), softmax's sum}
    uint64_t* work;
};
constexpr int kSliceThreads = 256;
struct RowWork {
    uint64_t *bins, *list, *sums;
    uint32_t *listed, *lowest;
    Open* open;
    uint64_t* whole;
    float2* seen;
    __device__ RowWork(const Slices& s, int64_t row) {
        bins = s.work + row * s.stride;
        list = bins + kBins;
        sums = list + kListed;
        listed = (uint32_t*)(sums + s.pieces);
        lowest = listed + 1;
        open = (Open*)(sums + s.pieces + 1);
        whole = (uint64_t*)(open + 1);
        seen = (float2*)(whole + 1);
    }
    // The row's largest logit; NaN where something is not a number.
    __device__ float top(int slices) const {
        float top = -INFINITY;
        bool bad = false;
        for (int i = threadIdx.x & 63; i < slices; i += 64) {
            const float x = seen[i].x;
            top = fmaxf(top, x);
            bad |= x != x;
        }
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) top = fmaxf(top, __shfl_xor(top, m));
        return __ballot(bad) ? __builtin_nanf("") : top;
    }
};

template <typename T> __global__ __launch_bounds__(kSliceThreads) void draw_tops_kernel(const Draws p, const Slices s, const T* logits) {
    constexpr int EACH = kTaserEach<T>;
    __shared__ float tops[kSliceThreads / 64];
    const int64_t row = blockIdx.y;
    const int slice = blockIdx.x;
    RowWork w(s, row);
    for (int i = slice * kSliceThreads + threadIdx.x; i < kBins; i += s.slices * kSliceThreads) w.bins[i] = 0;
    for (int i = slice * kSliceThreads + threadIdx.x; i < s.pieces; i += s.slices * kSliceThreads) w.sums[i] = 0;
    if (slice == 0 && threadIdx.x == 0) {
        *w.listed = 0;
        *w.lowest = 0xffffffffu;
    }
    const Row<T> r(p, logits, row, Rule{}, nullptr);
    float top = -INFINITY;
    bool bad = false;
    for (int h = 0; h < s.span; ++h) {
        float v[EACH];
        r.load((((int64_t)slice * s.span + h) * kSliceThreads + threadIdx.x) * EACH, v);
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            top = fmaxf(top, v[i]);
            bad |= v[i] != v[i];
        }
    }
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) top = fmaxf(top, __shfl_xor(top, m));
    bad = __ballot(bad || top == INFINITY) != 0;
    if ((threadIdx.x & 63) == 0) tops[threadIdx.x >> 6] = bad ? __builtin_nanf("") : top;
    __syncthreads();
    if (threadIdx.x) return;
    for (int i = 1; i < kSliceThreads / 64; ++i) top = top != top || tops[i] != tops[i] ? __builtin_nanf("") : fmaxf(top, tops[i]);
    w.seen[slice].x = bad ? __builtin_nanf("") : top;
}

template <typename T> __global__ __launch_bounds__(kSliceThreads) void draw_histogram_kernel(const Draws p, const Slices s, const T* logits) {
    constexpr int EACH = kTaserEach<T>;
    __shared__ uint64_t bins[kGapped];
    __shared__ double powers[256];
    __shared__ float totals[kSliceThreads / 64];
    const int64_t row = blockIdx.y;
    RowWork w(s, row);
    const Rule rule = rule_of(p, row);
    Row<T> r(p, logits, row, rule, powers);
    r.top = w.top(s.slices);
    if (!(r.top > -INFINITY)) return;
    const bool number = wants_number(rule, r.n), look = number || (!rule.greedy && rule.top_p), softly = !by_weights(rule, r.n);
    if (look) {
        for (int i = threadIdx.x; i < kGapped; i += kSliceThreads) bins[i] = 0;
        if (!number) r.fill(powers);
        __syncthreads();
    }
    float total = 0.f;
    uint32_t first = 0xffffffffu;
    for (int h = 0; h < s.span; ++h) {
        float v[EACH];
        const int64_t c = (((int64_t)blockIdx.x * s.span + h) * kSliceThreads + threadIdx.x) * EACH;
        r.load(c, v);
        if (number) r.count_in(bins, v, [](float x) { return (uint64_t)(x > -INFINITY); });
        else if (look) r.count_in(bins, v, [&](float x) { return r.weight(x); });
        if (rule.greedy) {
#pragma unroll
            for (int i = EACH - 1; i >= 0; --i) first = v[i] == r.top && (uint32_t)(c + i) < first ? (uint32_t)(c + i) : first;
        }
        if (softly) total += r.soft(r.top, v);
    }
    if (first != 0xffffffffu) atomicMin(w.lowest, first);
    if (softly) {
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) total += __shfl_xor(total, m);
        if ((threadIdx.x & 63) == 0) totals[threadIdx.x >> 6] = total;
    }
    __syncthreads();
    if (threadIdx.x == 0 && softly) {
        total = totals[0];
        for (int i = 1; i < kSliceThreads / 64; ++i) total += totals[i];
        w.seen[blockIdx.x].y = total;
    }
    if (look)
        for (int i = threadIdx.x; i < kBins; i += kSliceThreads) {
            const uint64_t x = bins[bin_at(i)];
            if (x) atomicAdd((unsigned long long*)&w.bins[i], (unsigned long long)x);
        }
}

template <typename T> __global__ __launch_bounds__(kSliceThreads) void draw_pieces_kernel(const Draws p, const Slices s, const T* logits) {
    constexpr int EACH = kTaserEach<T>;
    __shared__ uint64_t bins[kGapped];
    __shared__ double powers[256];
    __shared__ uint64_t list[kListed];
    __shared__ Found found;
    __shared__ uint32_t listed, base;
    const int64_t row = blockIdx.y;
    RowWork w(s, row);
    const Rule rule = rule_of(p, row);
    Row<T> r(p, logits, row, rule, powers);
    auto first_of = [&](int h) { return (((int64_t)blockIdx.x * s.span + h) * kSliceThreads + threadIdx.x) * EACH; };
    float v[EACH];
    r.load(first_of(0), v);   // on its way while the threshold is found
    r.top = w.top(s.slices);
    if (!(r.top > -INFINITY) || rule.greedy) return;
    r.fill(powers);
    if (threadIdx.x == 0) listed = 0;
    const bool number = wants_number(rule, r.n);
    Open o{INFINITY, INFINITY, 0, 0, 0};
    if (number || rule.top_p) {
        for (int i = threadIdx.x; i < kBins; i += kSliceThreads) bins[bin_at(i)] = w.bins[i];
        find_bin(bins, &found, [&](uint64_t all) -> uint64_t {
            if (number) return (uint64_t)rule.top_k < all ? (uint64_t)rule.top_k : 0;
            const uint64_t share = share_of(rule.top_p, all);
            return share ? share : 1;
        });
        if (found.wanted) o = open_by(rule, number, found);
        else if (rule.top_p) o.far = -1.f;   // no more candidates than top-k asks for, and no look at their weights yet: the last kernel's
    } else {
        __syncthreads();
    }
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        *w.open = o;
        *w.whole = found.all;
    }
    if (o.far < 0.f) return;
    for (int h = 0; h < s.span; ++h) {
        const int64_t c = first_of(h);
        if (h) r.load(c, v);
        const uint64_t sum = r.sure(v, rule.least, [&](float x) { return r.distance(x) < o.near && x > -INFINITY; });
        if ((threadIdx.x & 63) == 63 && sum) w.sums[c / (64 * EACH)] = sum;
        if (o.near < o.far) enlist(c, v, list, kListed, &listed, [&](float x) {
            const float d = r.distance(x);
            return d >= o.near && d < o.far && x > -INFINITY;
        });
    }
    if (!(o.near < o.far)) return;
    __syncthreads();
    if (threadIdx.x == 0) base = listed ? atomicAdd(w.listed, listed) : 0;   // more than fit here: more than fit there
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < listed && i < kListed; i += kSliceThreads)
        if (base + i < kListed) w.list[base + i] = list[i];
}

// Lists in which every candidate is compared with every other one, 16 pairs a thread: up to 64, 90 or 128 in blocks of 256, 512 or 1024. Longer ones are settled
// sooner by histograms (4096 x 4000 bf16, lists of 180: 88 us so, 159 by pairs; 2000 x 20 000, of 150: 84 and 101).
constexpr int kFew = 128;

// A row's draws. CUT: slices have gone before. Rows are read again for each pass: held in registers they would leave room for one block a compute
// unit, whose waits nothing hides (4096 x 64 001 bf16 with top-p, with the rest as it was then: 898 us so held, 606 with three blocks, which are 555 now). Three blocks
// leave 80 registers: 112 bytes a lane of a 16-bit row are spilled, 60 of a float32 one; the other sizes of block spill 48 in 16 bits, where the last loop's load is a call.
template <typename T, int THREADS, bool CUT> __global__ __launch_bounds__(THREADS, THREADS == 512 ? 6 : 4) void draw_row_kernel(const Draws p, const Slices s, const T* logits, int32_t* actions, float* logp) {
    constexpr int EACH = kTaserEach<T>, WAVES = THREADS / 64, STEP = THREADS * EACH;
    extern __shared__ uint64_t running_sums[];   // of the row's pieces, 64 lanes' each
    __shared__ uint64_t bins[kGapped], list[kListed];   // list: candidates around a threshold, {logit, number}
    __shared__ double powers[256];
    __shared__ Found found;
    __shared__ float tops[WAVES], totals[WAVES];
    __shared__ uint32_t bads[WAVES], lowest[3], highest[3], first_at, listed, few_rank[kFew];
    __shared__ uint64_t few_weight[kFew], few_sum[kFew], few_all;
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const Rule rule = rule_of(p, row);
    Row<T> r(p, logits, row, rule, powers);
    const int n = r.n, chunks = (n + STEP - 1) / STEP, pieces = chunks * WAVES;
    // take(piece, its first candidate, logits) for the row's pieces; whole waves come together.
    auto each = [&](auto&& take) {
#pragma clang loop unroll(disable)
        for (int h = 0; h < chunks; ++h) {
            float v[EACH];
            const int c = h * STEP + (int)threadIdx.x * EACH;
            r.load(c, v);
            take(h * WAVES + wave, c, v);
        }
    };
    float total = 0.f;
    auto join_total = [&]() {   // read behind the next barrier
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) total += __shfl_xor(total, m);
        if (lane == 0) totals[wave] = total;
    };
    r.fill(powers);
    for (int i = threadIdx.x; i < kGapped; i += THREADS) bins[i] = 0;
    for (int i = threadIdx.x; i < pieces; i += THREADS) running_sums[i] = 0;
    if (threadIdx.x == 0) {
        listed = 0;
        lowest[0] = first_at = 0xffffffffu;
        highest[0] = 0;
    }
    int slot = 0;
    if (CUT) {
        r.top = RowWork(s, row).top(s.slices);
        __syncthreads();
    } else {
        float top = -INFINITY;
        bool bad = false;
        each([&](int, int, const float (&v)[EACH]) {
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                top = fmaxf(top, v[i]);
                bad |= v[i] != v[i];
            }
        });
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) top = fmaxf(top, __shfl_xor(top, m));
        bad = __ballot(bad || top == INFINITY) != 0;
        if (lane == 0) {
            tops[wave] = top;
            bads[wave] = bad;
        }
        __syncthreads();
        bad = false;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            top = fmaxf(top, tops[w]);
            bad |= bads[w] != 0;
        }
        r.top = bad ? __builtin_nanf("") : top;
    }
    if (!(r.top > -INFINITY)) {   // the whole block
        for (int j = threadIdx.x; j < p.picks; j += THREADS) {
            actions[row * p.picks + j] = -1;
            logp[row * p.picks + j] = r.top != r.top ? __builtin_nanf("") : 0.f;
        }
        return;
    }
    if (rule.greedy) {
        uint32_t first = 0xffffffffu;
        if (CUT) {
            const RowWork w(s, row);
            first = *w.lowest;
            for (int i = lane; i < s.slices; i += 64) total += w.seen[i].y;
#pragma unroll
            for (int m = 1; m < 64; m <<= 1) total += __shfl_xor(total, m);
        } else {
            each([&](int, int c, const float (&v)[EACH]) {
#pragma unroll
                for (int i = EACH - 1; i >= 0; --i) first = v[i] == r.top && (uint32_t)(c + i) < first ? (uint32_t)(c + i) : first;
                total += r.soft(r.top, v);
            });
            if (first != 0xffffffffu) atomicMin(&first_at, first);
            join_total();
            __syncthreads();
            first = first_at;
            total = 0.f;
            for (int w = 0; w < WAVES; ++w) total += totals[w];
        }
        for (int j = threadIdx.x; j < p.picks; j += THREADS) {
            actions[row * p.picks + j] = (int)first;
            logp[row * p.picks + j] = -logf(total);
        }
        return;
    }

    // Among the candidates that `visit` shows (x, c) with a key: the key at which their amounts, from the largest key down, come to the target, and what
    // comes before it. Keys' bits, ten at a time, until there is one key left. known: the target does not go by the sum.
    auto select = [&](bool known, auto&& visit, auto&& key, auto&& amount, auto&& target, uint32_t& at, uint64_t& before, uint64_t& wanted) {
        uint32_t low = 0, high = 0xffffffffu;
        // To the smallest and largest there are. Of three slots one is in use, one may still be read and one is made ready: one barrier is enough.
        auto narrow = [&]() {
            const int now = slot, next = slot == 2 ? 0 : slot + 1;
            if (threadIdx.x == 0) {
                lowest[next] = 0xffffffffu;
                highest[next] = 0;
            }
            uint32_t a = 0xffffffffu, b = 0;
            visit([&](float x, uint32_t c) {
                const uint32_t k = key(x, c);
                if (k && k >= low && k <= high) {
                    a = k < a ? k : a;
                    b = k > b ? k : b;
                }
            });
            if (__ballot(b != 0)) {
                a = ~largest(~a);
                b = largest(b);
                if (lane == 63) {
                    atomicMin(&lowest[now], a);
                    atomicMax(&highest[now], b);
                }
            }
            __syncthreads();
            low = lowest[now];
            high = highest[now];
            slot = next;
        };
        narrow();
        before = wanted = at = 0;
        if (known && low == high) {
            at = high;
            wanted = target((uint64_t)0);
            return;
        }
        for (bool first = true;; first = false) {
            const uint32_t range = high - low;
            const int shift = range >= kBins ? 22 - __clz(range) : 0;
            if (!first && !range) break;
            visit([&](float x, uint32_t c) {
                const uint32_t k = key(x, c);
                if (k && k >= low && k <= high) atomicAdd((unsigned long long*)&bins[bin_at((int)((high - k) >> shift))], (unsigned long long)amount(x));
            });
            const uint64_t rest = wanted - before;
            if (first) find_bin(bins, &found, target);
            else find_bin(bins, &found, [&](uint64_t) { return rest; });
            if (first) wanted = found.wanted;
            if (!wanted) return;
            before += found.before;
            high -= found.bin << shift;
            const uint32_t down = (1u << shift) - 1;
            low = high - low > down ? high - down : low;
            if (shift) narrow();
            else low = high;
        }
        at = high;
    };
    auto weight = [&](float x) { return r.weight(x); };

    const bool by_number = wants_number(rule, n);
    bool softly = false, again = false;   // softly: the softmax's sum is still to come
    Open o{INFINITY, INFINITY, 0, 0, 0};
    uint64_t all_weights = 0;
    if (CUT) {
        const RowWork w(s, row);
        o = *w.open;
        all_weights = *w.whole;
        again = o.far < 0.f;
        const uint32_t there = *w.listed;
        if (!by_weights(rule, n)) {
            for (int i = lane; i < s.slices; i += 64) total += w.seen[i].y;
#pragma unroll
            for (int m = 1; m < 64; m <<= 1) total += __shfl_xor(total, m);
        }
        if (!again) {
            if (!o.all)
                for (int i = threadIdx.x; i < pieces; i += THREADS) running_sums[i] = i < s.pieces ? w.sums[i] : 0;
            for (int i = threadIdx.x; i < (int)(there < kListed ? there : kListed); i += THREADS) list[i] = w.list[i];
            if (threadIdx.x == 0) listed = there;
        }
        __syncthreads();
    } else {
        softly = !by_weights(rule, n);
        if (by_number) {
            each([&](int, int, const float (&v)[EACH]) {
                r.count_in(bins, v, [](float x) { return (uint64_t)(x > -INFINITY); });
                total += r.soft(r.top, v);
            });
            softly = false;
            join_total();
            find_bin(bins, &found, [&](uint64_t all) { return (uint64_t)rule.top_k < all ? (uint64_t)rule.top_k : 0; });
            total = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) total += totals[w];
            if (found.wanted) o = open_by(rule, true, found);
            else again = rule.top_p;   // no more candidates than are asked for
        }
    }
    if (again || (!CUT && !by_number && rule.top_p)) {
        if (again) r.scale = r.by_weight(rule);
        each([&](int, int, const float (&v)[EACH]) {
            r.count_in(bins, v, weight);
            if (softly) total += r.soft(r.top, v);
        });
        if (softly) join_total();
        find_bin(bins, &found, [&](uint64_t all) {
            const uint64_t share = share_of(rule.top_p, all);
            return share ? share : 1;
        });
        if (softly) {
            total = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) total += totals[w];
            softly = false;
        }
        o = open_by(rule, false, found);
        all_weights = found.all;
    }
    const bool number = o.number, open = number || rule.top_p;
    if (rule.top_p && by_weights(rule, n)) total = (float)all_weights * 0x1p-43f;
    float surely = 0.f, maybe = 0.f;
    auto bounds = [&]() {
        surely = r.closer(o.near);
        maybe = r.closer(o.far);
    };
    if (!CUT || again) {
        bounds();
        __syncthreads();
        each([&](int piece, int c, const float (&v)[EACH]) {
            if (!o.all) {
                const uint64_t sum = r.sure(v, rule.least, [&](float x) { return x >= surely; });
                if (lane == 63 && sum) running_sums[piece] = sum;
            }
            if (open) enlist(c, v, list, kListed, &listed, [&](float x) { return x >= maybe && x < surely; });
            if (softly) total += r.soft(r.top, v);
        });
        if (softly) join_total();
        __syncthreads();
        if (softly) {
            total = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) total += totals[w];
        }
    }

    float limit = -INFINITY;   // kept are those above it, and those at it up to the candidate cut
    uint32_t cut = 0xffffffffu;
    uint64_t at_limit = 0;     // how many of those at it, in the order of their candidates
    auto kept_weight = [&](float x, uint32_t c) -> uint64_t {
        if (!(x > limit || (x == limit && at_limit && c <= cut))) return 0;
        const uint64_t w = r.weight(x);
        return w >= rule.least ? w : 0;
    };
    // Top-k, then top-p, of the candidates that `visit` shows, those that were left open.
    auto settle = [&](auto&& visit) {
        uint64_t before, wanted;
        uint32_t at;
        if (number) {
            select(true, visit, [](float x, uint32_t) { return order_of(x); }, [](float) { return (uint64_t)1; }, [&](uint64_t) { return o.more; }, at, before, wanted);
            limit = float_of(at);
            at_limit = wanted - before;
        }
        if (rule.top_p) {
            const float over = limit;
            const uint64_t one = at_limit ? r.weight(over) : 0, rest = at_limit * one;
            // The share of all that are left; where it is past those over the limit, as many at it as it takes.
            uint64_t past = 0;
            auto target = [&](uint64_t here) -> uint64_t {
                if (!number) return o.more;
                const uint64_t share = share_of(rule.top_p, here + rest), least = share ? share : 1;
                past = least > here ? least - here : 0;
                return past ? 0 : least;
            };
            select(!number, visit, [&](float x, uint32_t) { return x > over ? order_of(x) : 0u; }, weight, target, at, before, wanted);
            if (wanted) {
                limit = float_of(at);
                const uint64_t w = r.weight(limit);
                at_limit = (wanted - before + w - 1) / w;
            } else {
                if (threadIdx.x == 0) found.before = past;   // wave 0 has it
                __syncthreads();
                at_limit = (found.before + one - 1) / one;
            }
        }
        // The first ones by number of those at the limit: the largest of ~c down.
        select(true, visit, [&](float x, uint32_t c) { return x == limit ? ~c : 0u; }, [](float) { return (uint64_t)1; }, [&](uint64_t) { return at_limit; }, cut, before, wanted);
        cut = ~cut;
    };
    if (open && listed && listed <= (uint32_t)kFew && listed * listed <= 16u * THREADS) {
        // How many lie before each of a short list, and what they weigh: all pairs, a part of them a thread.
        const int count = (int)listed, wide = (count + 63) & ~63, parts = THREADS / wide, mine = threadIdx.x % wide, part = threadIdx.x / wide, each_part = (count + parts - 1) / parts;
        const bool real = (int)threadIdx.x < count;
        auto logit = [&](uint64_t one) { return __uint_as_float((uint32_t)(one >> 32)); };
        if ((int)threadIdx.x < wide) {
            few_weight[threadIdx.x] = real ? r.weight(logit(list[threadIdx.x])) : 0;
            few_sum[threadIdx.x] = 0;
            few_rank[threadIdx.x] = 0;
        }
        if (threadIdx.x == 0) few_all = 0;
        __syncthreads();
        const uint64_t own = mine < count ? list[mine] : 0;
        const int from = part * each_part, to = from + each_part < count ? from + each_part : count;
        if (part < parts && mine < count) {
            uint32_t rank = 0;
            uint64_t before = 0;
#pragma unroll 4
            for (int j = from; j < to; ++j) {
                const uint64_t other = list[j], weighs = few_weight[j];
                const bool ahead = logit(other) > logit(own) || (logit(other) == logit(own) && (uint32_t)other < (uint32_t)own);
                rank += ahead;
                before += ahead ? weighs : 0;
            }
            if (rank) {
                atomicAdd(&few_rank[mine], rank);
                atomicAdd((unsigned long long*)&few_sum[mine], (unsigned long long)before);
            }
        }
        __syncthreads();
        const uint32_t rank = real ? few_rank[threadIdx.x] : 0;
        const uint64_t before = real ? few_sum[threadIdx.x] : 0, w = real ? few_weight[threadIdx.x] : 0;
        bool keep = real && (number ? rank < o.more : before < o.more);
        if (number && rule.top_p) {
            const uint64_t sum = running<64>(keep ? w : 0);
            if (lane == 63 && sum) atomicAdd((unsigned long long*)&few_all, (unsigned long long)sum);
            __syncthreads();
            keep = keep && (!rank || before < share_of(rule.top_p, few_all));
        }
        const uint64_t kept = keep && w >= rule.least ? w : 0;
        __syncthreads();   // all have read
        if (real) few_weight[threadIdx.x] = kept;
        if (threadIdx.x == 0) first_at = 0;
        if (o.all) {   // and draws from these: each one's sum of those up to it
            if (real) few_sum[threadIdx.x] = 0;
            __syncthreads();
            if (part < parts && mine < count) {
                uint64_t upto = 0;
#pragma unroll 4
                for (int j = from; j < to; ++j) upto += (uint32_t)list[j] <= (uint32_t)own ? few_weight[j] : 0;
                if (upto) atomicAdd((unsigned long long*)&few_sum[mine], (unsigned long long)upto);
            }
            __syncthreads();
            uint64_t whole = 0;
            for (int i = lane; i < count; i += 64) whole += few_weight[i];
            whole = sum_of<64>(whole);
            for (int j = wave; j < p.picks; j += WAVES) {
                const uint64_t place = place_of(p.uniform[row * p.picks + j], whole);
                for (int i = lane; i < count; i += 64) {
                    const uint64_t weighs = few_weight[i], upto = few_sum[i];
                    if (weighs && upto > place && upto - weighs <= place) {
                        actions[row * p.picks + j] = (int)(uint32_t)list[i];
                        logp[row * p.picks + j] = (logit(list[i]) - r.top) - logf(total);
                    }
                }
            }
            return;
        }
        __syncthreads();
        if (keep) atomicMax(&first_at, rank + 1);   // the last one kept is the limit
        if (kept) atomicAdd((unsigned long long*)&running_sums[(uint32_t)list[threadIdx.x] / (64 * EACH)], (unsigned long long)kept);
        __syncthreads();
        if (keep && rank + 1 == first_at) found.before = list[threadIdx.x];
        __syncthreads();
        limit = logit(found.before);
        cut = (uint32_t)found.before;
        at_limit = 1;
    } else if (open) {
        auto add_kept = [&](float x, uint32_t c) {
            const uint64_t w = kept_weight(x, c);
            if (w) atomicAdd((unsigned long long*)&running_sums[c / (64 * EACH)], (unsigned long long)w);
        };
        if (listed <= kListed) {
            auto in_list = [&](auto&& see) {
                for (int i = threadIdx.x; i < (int)listed; i += THREADS) see(__uint_as_float((uint32_t)(list[i] >> 32)), (uint32_t)list[i]);
            };
            settle(in_list);
            in_list(add_kept);
        } else {   // more than the list takes: the row again for each look
            bounds();
            auto in_row = [&](auto&& see) {
                each([&](int, int c, const float (&v)[EACH]) {
#pragma unroll
                    for (int i = 0; i < EACH; ++i)
                        if (v[i] >= maybe && v[i] < surely) see(v[i], (uint32_t)(c + i));
                });
            };
            settle(in_row);
            in_row(add_kept);
        }
    }
    __syncthreads();
    if (wave == 0) {
        uint64_t before = 0;
        for (int i = 0; i < pieces; i += 64) {
            const uint64_t upto = before + running<64>(i + lane < pieces ? running_sums[i + lane] : 0);
            if (i + lane < pieces) running_sums[i + lane] = upto;
            before = shuffle(upto, 63);
        }
    }
    __syncthreads();
    const uint64_t whole = running_sums[pieces - 1];
    if (!rule.top_p && by_weights(rule, n)) total = (float)whole * 0x1p-43f;
    for (int j = wave; j < p.picks; j += WAVES) {
        const uint64_t place = place_of(p.uniform[row * p.picks + j], whole);
        int at = 0;
        for (int i = 0; i < pieces; i += 64) {
            const uint64_t hit = __ballot(i + lane < pieces && running_sums[i + lane] > place);
            if (hit) {
                at = i + __ffsll((long long)hit) - 1;
                break;
            }
        }
        const int c = (at * 64 + lane) * EACH;
        float v[EACH];
        r.load(c, v);
        uint64_t w[EACH], sum = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) sum += w[i] = kept_weight(v[i], (uint32_t)(c + i));
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
                logp[row * p.picks + j] = (v[i] - r.top) - logf(total);
            }
        }
    }
}

// Rows of one block each leave compute units idle where there are few of them: such rows are cut (1 x 64 001 bf16, top-k and top-p: 41 us by one block, 64 x
// 130 000 f32, top-p: 138).
constexpr int64_t kFewRows = 256;
bool is_cut(const Draws& p, int32_t type) { return p.rows <= kFewRows && p.width > kSliceThreads * 4 * (type == TASER_F32 ? 4 : 8); }
Slices slices_of(const Draws& p, int32_t type) {
    const int each = type == TASER_F32 ? 4 : 8;
    const int64_t chunks = (p.width + kSliceThreads * each - 1) / (kSliceThreads * each), most = (1024 + p.rows - 1) / p.rows;
    Slices s = {};
    s.span = (int32_t)((chunks + most - 1) / most);
    s.slices = (int32_t)((chunks + s.span - 1) / s.span);
    s.pieces = s.slices * s.span * (kSliceThreads / 64);
    s.stride = kBins + kListed + (uint64_t)s.pieces + 1 + sizeof(Open) / 8 + 1 + (uint64_t)s.slices;
    return s;
}

template <typename T> int launch(const Draws& p, int32_t type, const void* logits, int32_t* actions, float* logp, uint64_t* work, hipStream_t stream) {
    const int most = p.width > p.picks ? p.width : p.picks;
    const int64_t pieces = (p.width + kTaserEach<T> - 1) / kTaserEach<T>;
    const int g = most <= 16 ? 16 : (most <= 32 ? 32 : 64), each = 256 / g;
    const bool cut = is_cut(p, type);
    const int threads = most <= 64 || pieces <= 1024 ? 256 : cut ? 1024 : 512;
    const int64_t blocks = most <= 64 ? (p.rows + each - 1) / each : p.rows;
    if (!taser_launch_fits(blocks, threads)) return taser_fail(TASER_E_RANGE, "policy_draw: too many rows for one launch");
    const unsigned grid = (unsigned)blocks, sums = (unsigned)((pieces + threads - 1) / threads * (threads / 64) * sizeof(uint64_t));
    TaserProfileSpan span(stream, "policy_draw");
    if (most <= 64) {
        if (g == 16) draw_window_kernel<T, 16><<<grid, 256, 0, stream>>>(p, (const T*)logits, actions, logp);
        else if (g == 32) draw_window_kernel<T, 32><<<grid, 256, 0, stream>>>(p, (const T*)logits, actions, logp);
        else draw_window_kernel<T, 64><<<grid, 256, 0, stream>>>(p, (const T*)logits, actions, logp);
    } else if (cut) {
        Slices s = slices_of(p, type);
        s.work = work;
        const dim3 across((unsigned)s.slices, grid);
        draw_tops_kernel<T><<<across, kSliceThreads, 0, stream>>>(p, s, (const T*)logits);
        draw_histogram_kernel<T><<<across, kSliceThreads, 0, stream>>>(p, s, (const T*)logits);
        draw_pieces_kernel<T><<<across, kSliceThreads, 0, stream>>>(p, s, (const T*)logits);
        draw_row_kernel<T, 1024, true><<<grid, 1024, sums, stream>>>(p, s, (const T*)logits, actions, logp);
    } else if (threads == 256) {
        draw_row_kernel<T, 256, false><<<grid, 256, sums, stream>>>(p, Slices{}, (const T*)logits, actions, logp);
    } else {
        draw_row_kernel<T, 512, false><<<grid, 512, sums, stream>>>(p, Slices{}, (const T*)logits, actions, logp);
    }
    TASER_HIP_TRY(hipGetLastError());
    return TASER_OK;
}

Draws draws_of(const taser_policy_draws* b) {
    return Draws{b->picks, (int32_t)b->width, b->rows, b->logits_stride, b->count, b->uniform, b->temperature, b->top_p, b->min_p, b->top_k,
                 b->row_temperature, b->row_top_p, b->row_min_p, b->row_top_k};
}
uint64_t draw_bytes(const Draws& p, int32_t type) { return p.rows && is_cut(p, type) ? (uint64_t)p.rows * slices_of(p, type).stride * sizeof(uint64_t) : 0; }

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
    *work_bytes = draw_bytes(draws_of(b), b->type);
    return TASER_OK;
}

extern "C" int taser_policy_draw(const taser_policy_draws* b, int32_t* actions, float* logp, void* work, uint64_t work_bytes, void* hip_stream) {
    if (const int rc = check(b)) return rc;
    if (!b->rows) return TASER_OK;
    if (!b->logits || !b->uniform || !actions || !logp) return taser_fail(TASER_E_ARG, "policy_draw: null logits, random numbers or outputs");
    const Draws p = draws_of(b);
    const uint64_t bytes = draw_bytes(p, b->type);
    if (bytes && (!work || work_bytes < bytes || (uintptr_t)work % 16)) return taser_fail(TASER_E_ARG, "policy_draw: less workspace than taser_policy_draw_bytes says, or not aligned to 16 bytes");
    hipStream_t stream = (hipStream_t)hip_stream;
    taser_clear_stale_hip_error();
    if (b->type == TASER_F32) return launch<float>(p, b->type, b->logits, actions, logp, (uint64_t*)work, stream);
    if (b->type == TASER_F16) return launch<_Float16>(p, b->type, b->logits, actions, logp, (uint64_t*)work, stream);
    return launch<__bf16>(p, b->type, b->logits, actions, logp, (uint64_t*)work, stream);
}

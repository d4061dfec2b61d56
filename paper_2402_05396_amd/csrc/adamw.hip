// The AdamW step over a list of tensors (taser_adamw_step) and 8-bit moments as numbers (taser_adamw_moments).
//
//   m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2,  p = p (1 - lr decay) - (lr / c1) m / (sqrt(v) / sqrt(c2) + eps)
// with c = 1 - beta^step, everything in 32 bits.
//
// Moments in 32 bits: bound by memory, 16 bytes of them of the 22 to 28 that an element moves (100 M elements in bfloat16: 433 us, 5.1 TB/s). In 8
// bits: 4.1 of 10 to 16, and some hundred vector instructions, which take nearly as long (118 M elements, parameters in single precision, gradients in
// bfloat16: 1.66 GB in 325 us, 5.1 TB/s; both in bfloat16: 1.19 GB in 287 us, 4.1 TB/s).
//
// A launch takes up to kTensors tensors, their addresses among its arguments (nothing is copied to the device, so a captured call replays
// as it is); a block finds its tensor by one comparison a lane. 48 tensors of 0.48 M elements in all: 6 us, and 8 for the host's call.
//
// Moments in 8 bits share a unit among 256 neighbors of a tensor: m = sign c^2 unit (7 bits of c), sqrt(v) = c^2 unit. Steps
// between codes are 2 / c (m) and 4 / c (v) of a value, 1.6 % for the block's largest, over a range of 4.2 (m) and 9.6 (v) decades. Rounded to the
// nearer code, a second moment would not move at all where beta2 = 0.999 changes it by a tenth of a percent a step; so it goes up with
// the chance that makes its expectation exact. A v that is not 0 keeps a code of 1 at least: the update divides by its root.
#include "pieces.h"
#include "sampling_device.h"

#include <algorithm>
#include <cmath>
#include <utility>
#include <vector>

namespace {

constexpr int kTensors = 56;      // of a launch
constexpr int kChunk = 2048;      // elements of a block (100 M elements: 433 us; 457 with twice, 462 with four times as many, whose loads wait for stores)
constexpr int kShared = TASER_ADAMW_BLOCK;
constexpr uint32_t kTag = 0x4144414Du;

struct Tensor {
    void* p;
    const void* g;
    void *m, *v;
    float *m_unit, *v_unit;
    int64_t n;
    uint32_t first;    // its first block of the launch
    uint16_t types;    // of p, and 4 times that of g
    uint16_t unused;
};
struct Step {
    double lr, log_beta1, log_beta2, decay;
    float b1, b1_rest, b2, b2_rest, eps;
    int32_t tensors;
    int64_t step;
    const int64_t* step_at;
    const float *lr_at, *grad_scale;
    uint32_t seed_lo, seed_hi;
};
struct Launch {
    Step s;
    uint32_t numbers[kTensors];   // of the tensors in the caller's list
    Tensor t[kTensors];
};
static_assert(sizeof(Launch) <= 4096, "arguments of a launch");

// What a step multiplies by: 1 - lr decay, lr / c1, 1 / sqrt(c2), the gradients' factor.
struct Factors { float keep, rate, root, scale; };
__host__ __device__ inline Factors factors_of(const Step& s, double lr, int64_t step) {
    const double c1 = 1. - exp((double)step * s.log_beta1), c2 = 1. - exp((double)step * s.log_beta2);
    return {(float)(1. - lr * s.decay), (float)(lr / c1), (float)(1. / sqrt(c2)), 1.f};
}

// One element. Without contraction: moments are the same bits as from separate products and sums. EXACT: the root is rounded correctly; else it is off by
// one in its last place, and 0 for a v below 2^-126 (ten vector instructions an element less, which is what 8-bit moments wait for; needs_exact_root
// says where that would show).
template <bool EXACT> __device__ inline void update(const Step& s, const Factors& f, float& p, float g, float& m, float& v, float& root) {
#pragma clang fp contract(off)
    g = g * f.scale;
    m = m * s.b1 + g * s.b1_rest;
    v = v * s.b2 + (g * g) * s.b2_rest;
    root = EXACT ? sqrtf(v) : __builtin_amdgcn_sqrtf(v);
    p = p * f.keep - (m * f.rate) * __builtin_amdgcn_rcpf(root * f.root + s.eps);
}

// The tensor that a block belongs to, and the factors; false: nothing is to be done. With the step's number or the rate on the device each thread works the factors out,
// in 64 bits and before its loads: 8-bit moments 372 to 374 us for 325, both in bfloat16 334 to 343 for 287; 32-bit ones 434 for 432.
__device__ inline bool find(const Launch& a, const Factors& given, int& tensor, Factors& f, int64_t& step) {
    const int lane = threadIdx.x & 63;
    const uint32_t first = lane < a.s.tensors ? a.t[lane].first : ~0u;
    tensor = __builtin_amdgcn_readfirstlane(__popcll(__ballot(first <= blockIdx.x)) - 1);
    f = given;
    step = a.s.step_at ? *a.s.step_at : a.s.step;
    if (a.s.step_at || a.s.lr_at) f = factors_of(a.s, a.s.lr_at ? (double)*a.s.lr_at : a.s.lr, step);
    if (a.s.grad_scale) f.scale = *a.s.grad_scale;
    return f.scale == f.scale && step >= 1;
}

__global__ __launch_bounds__(256) void adamw_kernel(const Launch a, const Factors given) {
    int i;
    Factors f;
    int64_t step;
    if (!find(a, given, i, f, step)) return;
    const Tensor& t = a.t[i];
    const int64_t n = t.n, base = (int64_t)(blockIdx.x - t.first) * kChunk;
    const int p_type = t.types & 3, g_type = t.types >> 2;
    constexpr int AT_ONCE = 2;
    static_assert(AT_ONCE * 1024 == kChunk, "256 threads of 4 elements");
    float p[AT_ONCE][4], g[AT_ONCE][4], m[AT_ONCE][4], v[AT_ONCE][4];
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
        const int64_t at = base + j * 1024 + threadIdx.x * 4;
        taser_load_floats<4>(t.p, p_type, at, n, p[j]);
        taser_load_floats<4>(t.g, g_type, at, n, g[j]);
        taser_load_as<float, 4>(t.m, at, n, m[j]);
        taser_load_as<float, 4>(t.v, at, n, v[j]);
    }
#pragma unroll
    for (int j = 0; j < AT_ONCE; ++j) {
        const int64_t at = base + j * 1024 + threadIdx.x * 4;
        float root;
#pragma unroll
        for (int k = 0; k < 4; ++k) update<true>(a.s, f, p[j][k], g[j][k], m[j][k], v[j][k], root);
        taser_store_floats<4>(t.p, p_type, at, n, p[j]);
        taser_store_as<float, 4>(t.m, at, n, m[j]);
        taser_store_as<float, 4>(t.v, at, n, v[j]);
    }
}

// ---- moments in 8 bits ---------------------------------------------------------------------------

__device__ inline float number_of(uint32_t code, float unit) {
    float c = (float)code;
    asm("" : "+v"(c));   // squared as a float (exactly): the compiler would go back to packed products of 16-bit integers
    return (c * c) * unit;
}

// The unit of values up to `most` (as bits, so that NaN is the largest): NaN where one is not finite.
__device__ inline float unit_of(uint32_t most, float share) {
    return most >= 0x7f800000u ? __builtin_nanf("") : __uint_as_float(most) * share;
}

// c with unit c^2 near `value`, below MOST + 1: between two by chance, so that the expectation of unit c^2 (QUAD: of its square) is right.
template <int MOST, bool QUAD> __device__ inline uint32_t code_of(float value, float inverse, float chance) {
#pragma clang fp contract(off)
    float y = value * inverse;
    const float c = fminf(floorf(__builtin_amdgcn_sqrtf(y)), (float)(MOST - 1));
    float low = c * c, apart = c + c + 1.f;   // to (c + 1)^2
    if (QUAD) {
        y = y * y;
        apart = apart * (low + low + (c + c) + 1.f);
        low = low * low;
    }
    return (uint32_t)c + (y - low > chance * apart ? 1u : 0u);
}

__device__ inline void load_codes(const uint8_t* from, int64_t at, int64_t n, uint8_t (&to)[8]) {
    if (at + 8 <= n) {
        __builtin_memcpy(to, from + at, 8);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) to[i] = at + i < n ? from[at + i] : 0;
    }
}
__device__ inline void store_codes(uint8_t* to, int64_t at, int64_t n, const uint8_t (&from)[8]) {
    if (at + 8 <= n) {
        __builtin_memcpy(to + at, from, 8);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (at + i < n) to[at + i] = from[i];
    }
}
__device__ inline float m_of(uint8_t code, float unit) {
    const float x = number_of(code & 127u, unit);
    return code & 128u ? -x : x;
}
__device__ inline float v_of(uint8_t code, float unit) {
    const float root = number_of(code, unit);
    return root * root;
}

// 32 lanes share a unit's 256 elements, eight each: as many 16-bit chances as one draw of four words holds.
template <bool EXACT> __global__ __launch_bounds__(256) void adamw_bytes_kernel(const Launch a, const Factors given) {
    static_assert(kShared == 256, "32 lanes of 8 elements");
    int i;
    Factors f;
    int64_t step;
    if (!find(a, given, i, f, step)) return;
    const Tensor& t = a.t[i];
    const int64_t n = t.n, base = (int64_t)(blockIdx.x - t.first) * kChunk;
    const int p_type = t.types & 3, g_type = t.types >> 2, lane = threadIdx.x & 31;
    const uint32_t number = a.numbers[i];
    const int64_t at = base + threadIdx.x * 8, block = at / kShared;
    if (block * kShared >= n) return;   // a block's lanes leave together
    float p[8], g[8];
    uint8_t mc[8], vc[8];
    taser_load_floats<8>(t.p, p_type, at, n, p);
    taser_load_floats<8>(t.g, g_type, at, n, g);
    load_codes((const uint8_t*)t.m, at, n, mc);
    load_codes((const uint8_t*)t.v, at, n, vc);
    const float m_unit = t.m_unit[block], v_unit = t.v_unit[block];
    uint32_t c[4] = {(uint32_t)(at >> 3), number, (uint32_t)step, kTag}, k0 = a.s.seed_lo, k1 = a.s.seed_hi;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        philox_round<true>(c, k0, k1);
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    float m[8], root[8];
    uint32_t m_most = 0, v_most = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        m[j] = m_of(mc[j], m_unit);
        float v = v_of(vc[j], v_unit);
        update<EXACT>(a.s, f, p[j], g[j], m[j], v, root[j]);   // (places past the tensor's end hold zeros)
        const uint32_t size = __float_as_uint(m[j]) & 0x7fffffffu, other = __float_as_uint(root[j]);   // NaN is the largest, of either sign
        m_most = size > m_most ? size : m_most;
        v_most = other > v_most ? other : v_most;
    }
    taser_store_floats<8>(t.p, p_type, at, n, p);
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) {
        const uint32_t x = __shfl_xor(m_most, s), y = __shfl_xor(v_most, s);
        m_most = x > m_most ? x : m_most;
        v_most = y > v_most ? y : v_most;
    }
    const float m_next = unit_of(m_most, 1.f / (127.f * 127.f)), v_next = unit_of(v_most, 1.f / (255.f * 255.f));
    // (A unit below 2^-126 has an inverse that may be infinite: moments that small count as 0.)
    const float m_inverse = m_next >= 1.17549435e-38f ? 1.f / m_next : 0.f, v_inverse = v_next >= 1.17549435e-38f ? 1.f / v_next : 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float chance = ((float)(c[j >> 1] >> (16 * (j & 1)) & 0xffffu) + 0.5f) * (1.f / 65536.f);
        const uint32_t code = code_of<127, false>(fabsf(m[j]), m_inverse, chance);
        mc[j] = (uint8_t)(code | (m[j] < 0.f && code ? 128u : 0u));
        const uint32_t other = code_of<255, true>(root[j], v_inverse, chance);
        vc[j] = (uint8_t)(root[j] > 0.f && !other ? 1u : other);
    }
    store_codes((uint8_t*)t.m, at, n, mc);
    store_codes((uint8_t*)t.v, at, n, vc);
    if (lane == 0) {
        t.m_unit[block] = m_next;
        t.v_unit[block] = v_next;
    }
}

__global__ __launch_bounds__(256) void adamw_moments_kernel(const uint8_t* m, const uint8_t* v, const float* m_unit, const float* v_unit, int64_t n, int32_t type, void* m_out, void* v_out) {
    const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (at >= n) return;
    uint8_t mc[8], vc[8];
    load_codes(m, at, n, mc);
    load_codes(v, at, n, vc);
    const float mu = m_unit[at / kShared], vu = v_unit[at / kShared];
    float x[8], y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        x[j] = m_of(mc[j], mu);
        y[j] = v_of(vc[j], vu);
    }
    taser_store_floats<8>(m_out, type, at, n, x);
    taser_store_floats<8>(v_out, type, at, n, y);
}

// ---- on the host ---------------------------------------------------------------------------------

struct Span {
    uintptr_t from, to;
    bool written;
};

// Whether memory that the step writes is named twice, as another tensor's or as a gradient. Lists that ascend and lie behind each other, as
// views of a few buffers do, need no sorting.
bool overlap(std::vector<Span>* lists, int n_lists) {
    bool in_order = true;
    for (int i = 0; i < n_lists && in_order; ++i)
        for (size_t j = 1; j < lists[i].size() && in_order; ++j) in_order = lists[i][j - 1].to <= lists[i][j].from;
    for (int i = 0; i < n_lists && in_order; ++i)
        for (int j = 0; j < i && in_order; ++j)
            in_order = lists[i].empty() || lists[j].empty() || lists[i].back().to <= lists[j].front().from || lists[j].back().to <= lists[i].front().from;
    if (in_order) return false;
    std::vector<Span> all;
    for (int i = 0; i < n_lists; ++i) all.insert(all.end(), lists[i].begin(), lists[i].end());
    std::sort(all.begin(), all.end(), [](const Span& x, const Span& y) { return x.from < y.from; });
    uintptr_t end = 0, written = 0;   // of any so far, and of any that is written
    for (const Span& s : all) {
        if (s.from < written || (s.written && s.from < end)) return true;
        end = std::max(end, s.to);
        if (s.written) written = std::max(written, s.to);
    }
    return false;
}

int check(const taser_adamw* a, const taser_adamw_tensor* tensors, int64_t n) {
    if (!a) return taser_fail(TASER_E_ARG, "adamw_step: null argument block");
    if (a->bits != 8 && a->bits != 32) return taser_fail(TASER_E_ARG, "adamw_step: moments have 8 or 32 bits, not %d", a->bits);
    if (n < 0 || (n && !tensors)) return taser_fail(TASER_E_ARG, "adamw_step: negative number of tensors, or none given");
    if (n >= (int64_t)1 << 31) return taser_fail(TASER_E_RANGE, "adamw_step: too many tensors");
    if (!(a->beta1 >= 0.) || !(a->beta1 < 1.) || !(a->beta2 >= 0.) || !(a->beta2 < 1.)) return taser_fail(TASER_E_ARG, "adamw_step: beta1 and beta2 lie in [0, 1)");
    if (!(a->eps >= 0.) || !std::isfinite(a->eps) || !(a->weight_decay >= 0.) || !std::isfinite(a->weight_decay))
        return taser_fail(TASER_E_ARG, "adamw_step: eps and weight_decay must not be negative, and finite");
    if (!a->lr_at && !(std::isfinite(a->lr) && a->lr >= 0.)) return taser_fail(TASER_E_ARG, "adamw_step: the rate must not be negative, and finite");
    if (!a->step_at && a->step < 1) return taser_fail(TASER_E_ARG, "adamw_step: steps count from 1");
    std::vector<Span> lists[6];
    for (auto& l : lists) l.reserve((size_t)n);
    for (int64_t i = 0; i < n; ++i) {
        const taser_adamw_tensor& t = tensors[i];
        if (t.elements < 0) return taser_fail(TASER_E_ARG, "adamw_step: tensor %lld has a negative size", (long long)i);
        if (!t.elements || !t.grad) continue;
        if (t.type < TASER_F32 || t.type > TASER_BF16 || t.grad_type < TASER_F32 || t.grad_type > TASER_BF16) return taser_fail(TASER_E_ARG, "adamw_step: unknown element type of tensor %lld", (long long)i);
        if (t.elements > (int64_t)1 << 34) return taser_fail(TASER_E_RANGE, "adamw_step: tensor %lld has more than 2^34 elements", (long long)i);
        if (!t.param || !t.m || !t.v || (a->bits == 8 && (!t.m_unit || !t.v_unit))) return taser_fail(TASER_E_ARG, "adamw_step: null memory of tensor %lld", (long long)i);
        const uint64_t size = t.type == TASER_F32 ? 4 : 2, g_size = t.grad_type == TASER_F32 ? 4 : 2, moment = a->bits == 8 ? 1 : 4, e = (uint64_t)t.elements;
        const uint64_t units = (e + kShared - 1) / kShared * sizeof(float);
        auto add = [&](int list, const void* p, uint64_t bytes, bool written) { lists[list].push_back({(uintptr_t)p, (uintptr_t)p + bytes, written}); };
        add(0, t.param, e * size, true);
        add(1, t.grad, e * g_size, false);
        add(2, t.m, e * moment, true);
        add(3, t.v, e * moment, true);
        if (a->bits == 8) {
            add(4, t.m_unit, units, true);
            add(5, t.v_unit, units, true);
        }
    }
    // Blocks read these while others write.
    const Span read[3] = {{(uintptr_t)a->step_at, (uintptr_t)a->step_at + 8, false}, {(uintptr_t)a->lr_at, (uintptr_t)a->lr_at + 4, false}, {(uintptr_t)a->grad_scale, (uintptr_t)a->grad_scale + 4, false}};
    for (const Span& r : read)
        if (r.from)
            for (const auto& list : lists)
                for (const Span& s : list)
                    if (s.written && s.from < r.to && r.from < s.to) return taser_fail(TASER_E_ARG, "adamw_step: the step's number, the rate or the gradients' factor lies in memory that is written");
    if (overlap(lists, 6)) return taser_fail(TASER_E_ARG, "adamw_step: tensors overlap in memory");
    return TASER_OK;
}

// A root that is 0 instead of up to 2^-63 is at most 2^-63 / sqrt(1 - beta2) less in the denominator, at any step: nothing beside an eps 2^24 times that (5.7e-11
// where beta2 is 0.999). Below it the root decides, and an eps of 0 would leave 1 / 0. (118 M elements, parameters in single precision, gradients in bfloat16: 325 us, with
// the exact root 337.)
bool needs_exact_root(const taser_adamw* a) { return !(a->eps >= 0x1p-39 / std::sqrt(1. - a->beta2)); }

}  // namespace

extern "C" int taser_adamw_step(const taser_adamw* a, const taser_adamw_tensor* tensors, int64_t n, void* hip_stream) try {
    if (const int rc = check(a, tensors, n)) return rc;
    hipStream_t stream = (hipStream_t)hip_stream;
    taser_clear_stale_hip_error();
    Launch l = {};
    l.s.lr = a->lr;
    l.s.log_beta1 = std::log(a->beta1);
    l.s.log_beta2 = std::log(a->beta2);
    l.s.decay = a->weight_decay;
    l.s.b1 = (float)a->beta1;
    l.s.b1_rest = (float)(1. - a->beta1);
    l.s.b2 = (float)a->beta2;
    l.s.b2_rest = (float)(1. - a->beta2);
    // v_rcp_f32 of a number below 2^-126 may be infinite, and a moment of 0 times that NaN. No root but 0 is below 2^-75: beside the others a raised eps is nothing.
    l.s.eps = a->eps > 0. ? std::max((float)a->eps, 0x1p-126f) : 0.f;
    l.s.step = a->step;
    l.s.step_at = a->step_at;
    l.s.lr_at = a->lr_at;
    l.s.grad_scale = a->grad_scale;
    l.s.seed_lo = (uint32_t)a->seed;
    l.s.seed_hi = (uint32_t)(a->seed >> 32);
    const Factors given = factors_of(l.s, a->lr, a->step_at ? 1 : a->step);
    int64_t blocks = 0;
    auto flush = [&]() -> int {
        if (!blocks) return TASER_OK;
        TaserProfileSpan span(stream, "adamw_step");
        if (a->bits == 8 && needs_exact_root(a)) adamw_bytes_kernel<true><<<(unsigned)blocks, 256, 0, stream>>>(l, given);
        else if (a->bits == 8) adamw_bytes_kernel<false><<<(unsigned)blocks, 256, 0, stream>>>(l, given);
        else adamw_kernel<<<(unsigned)blocks, 256, 0, stream>>>(l, given);
        TASER_HIP_TRY(hipGetLastError());
        blocks = 0;
        l.s.tensors = 0;
        return TASER_OK;
    };
    for (int64_t i = 0; i < n; ++i) {
        const taser_adamw_tensor& t = tensors[i];
        if (!t.elements || !t.grad) continue;
        const int64_t own = (t.elements + kChunk - 1) / kChunk;
        if (l.s.tensors == kTensors || !taser_launch_fits(blocks + own, 256))
            if (const int rc = flush()) return rc;
        const int at = l.s.tensors++;
        l.numbers[at] = (uint32_t)i;
        l.t[at] = Tensor{t.param, t.grad, t.m, t.v, t.m_unit, t.v_unit, t.elements, (uint32_t)blocks, (uint16_t)(t.type + 4 * t.grad_type), 0};
        blocks += own;
    }
    return flush();
} catch (const std::exception& e) {
    return taser_fail(TASER_E_OOM, "adamw_step: %s", e.what());
}

extern "C" int taser_adamw_moments(const uint8_t* m, const uint8_t* v, const float* m_unit, const float* v_unit, int64_t elements, int32_t type, void* m_out, void* v_out, void* hip_stream) {
    if (elements < 0) return taser_fail(TASER_E_ARG, "adamw_moments: negative number of elements");
    if (type < TASER_F32 || type > TASER_BF16) return taser_fail(TASER_E_ARG, "adamw_moments: unknown element type %d", type);
    if (!elements) return TASER_OK;
    if (!m || !v || !m_unit || !v_unit || !m_out || !v_out) return taser_fail(TASER_E_ARG, "adamw_moments: null argument");
    const int64_t blocks = (elements + 2047) / 2048;
    if (elements > (int64_t)1 << 35 || !taser_launch_fits(blocks, 256)) return taser_fail(TASER_E_RANGE, "adamw_moments: too many elements for one launch");
    hipStream_t stream = (hipStream_t)hip_stream;
    taser_clear_stale_hip_error();
    TaserProfileSpan span(stream, "adamw_moments");
    adamw_moments_kernel<<<(unsigned)blocks, 256, 0, stream>>>(m, v, m_unit, v_unit, elements, type, m_out, v_out);
    TASER_HIP_TRY(hipGetLastError());
    return TASER_OK;
}

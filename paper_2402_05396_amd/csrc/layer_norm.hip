// Layer norm and its gradient (taser_layer_norm, taser_layer_norm_grad).
//
//   out = xhat weight + bias,  xhat = (x - mean) rstd;  with g = dout weight:
//   dx = rstd (g - mean(g) - xhat mean(g xhat)),  dweight = sum over rows of dout xhat,  dbias = sum over rows of dout
//
// Both are bound by reading and writing rows once. A row belongs to a group of threads, each with up to 16 of its columns (in the gradient 8) in registers:
// mean first, then the squares of what is away from it (no difference of large sums). A group goes from row to row, its columns' weights and,
// in the gradient, its columns' sums of dweight and dbias staying in registers, the next row on its way; a block adds its groups' sums
// through LDS, a second launch the blocks', in an order that the sizes fix. Rows of more than 8192 are a block's each, held in registers up to 32768
// and read again for each pass past that, and their dweight and dbias come from a kernel of their own, by columns.
//
// 8192 x 5120 bf16, the answer: 33 us (168 MB at 5.1 TB/s; 5120 is five waves' 1024 columns each: with groups of powers of two 50). 16 384 x 4096 bf16: 48 and,
// for the gradient, 100 + 5 us (4.1 TB/s; two blocks of eight waves a compute unit are what its registers leave, and 17 MB of parts are written and read).
// 12 000 x 100 f32: 5.5 and 7 + 3.5 us: three launches. One row of 4096: 4 us.
#include "pieces.h"

namespace {

constexpr int64_t kHeld = 8192;       // rows up to it stay in registers, with what belongs to their columns

struct Norm {
    int64_t rows, width, x_stride, dout_stride;
    const void *weight, *bias;
    int32_t weight_type;
    float eps;
};

// Sums of two numbers over a group of threads: G lanes of a wave, or (G = 0) `waves` waves, by way of LDS, `turn` alternating between its two halves.
template <int G> __device__ inline void group_sums(float& a, float& b, float2 (*shared)[16], int turn, int waves) {
    constexpr int LANES = G ? G : 64;
#pragma unroll
    for (int m = 1; m < LANES; m <<= 1) {
        a += __shfl_xor(a, m);
        b += __shfl_xor(b, m);
    }
    if (G || waves == 1) return;
    const int wave = threadIdx.x >> 6, first = wave / waves * waves;
    if ((threadIdx.x & 63) == 0) shared[turn & 1][wave] = make_float2(a, b);
    __syncthreads();
    a = b = 0.f;
    for (int w = 0; w < waves; ++w) {
        const float2 x = shared[turn & 1][first + w];
        a += x.x;
        b += x.y;
    }
}

// A thread's columns: piece h at (h threads + lane) EACH.
template <typename T, int HELD> __device__ inline void load_row(const T* row, int threads, int lane, int64_t width, TaserPiece<T> (&p)[HELD]) {
#pragma unroll
    for (int h = 0; h < HELD; ++h) taser_load_piece<T>(row, (int64_t)(h * threads + lane) * kTaserEach<T>, width, (T)0.f, p[h]);
}
template <typename T, int HELD> __device__ inline void load_weights(const void* from, int32_t type, int threads, int lane, int64_t width, float none, float (&w)[HELD][kTaserEach<T>]) {
#pragma unroll
    for (int h = 0; h < HELD; ++h) {
        if (from) {
            taser_load_floats<kTaserEach<T>>(from, type, (int64_t)(h * threads + lane) * kTaserEach<T>, width, w[h]);
        } else {
#pragma unroll
            for (int i = 0; i < kTaserEach<T>; ++i) w[h][i] = none;
        }
    }
}

// G: lanes of a group, or 0: groups of `waves` waves.
template <typename T, int G, int HELD, int THREADS> __global__ __launch_bounds__(THREADS) void norm_kernel(const Norm p, int waves, const T* x, T* out, float* stats) {
    constexpr int EACH = kTaserEach<T>;
    __shared__ float2 shared[2][16];
    const int threads = G ? G : waves * 64, lane = threadIdx.x % threads, here = blockDim.x / threads;
    const int64_t groups = (int64_t)gridDim.x * here, turns = (p.rows + groups - 1) / groups;
    float weight[HELD][EACH], bias[HELD][EACH];
    load_weights<T, HELD>(p.weight, p.weight_type, threads, lane, p.width, 1.f, weight);
    load_weights<T, HELD>(p.bias, p.weight_type, threads, lane, p.width, 0.f, bias);
    TaserPiece<T> next[HELD];
    // A group without a row of its own left takes the last one once more: it writes nothing.
    int64_t row = (int64_t)blockIdx.x * here + threadIdx.x / threads;
    load_row<T, HELD>(x + (row < p.rows ? row : p.rows - 1) * p.x_stride, threads, lane, p.width, next);
    const float by = 1.f / (float)p.width;
    for (int64_t turn = 0; turn < turns; ++turn, row += groups) {
        float v[HELD][EACH];
        float sum = 0.f, none = 0.f;
#pragma unroll
        for (int h = 0; h < HELD; ++h)
#pragma unroll
            for (int i = 0; i < EACH; ++i) sum += v[h][i] = (float)next[h].x[i];
        if (turn + 1 < turns) load_row<T, HELD>(x + (row + groups < p.rows ? row + groups : p.rows - 1) * p.x_stride, threads, lane, p.width, next);
        group_sums<G>(sum, none, shared, 0, waves);
        const float mean = sum * by;
        float squares = 0.f;
#pragma unroll
        for (int h = 0; h < HELD; ++h)
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                v[h][i] = (int64_t)(h * threads + lane) * EACH + i < p.width ? v[h][i] - mean : 0.f;
                squares = fmaf(v[h][i], v[h][i], squares);
            }
        group_sums<G>(squares, none, shared, 1, waves);
        const float rstd = 1.f / sqrtf(squares * by + p.eps);
        if (row >= p.rows) continue;   // its last turn
        if (stats && lane == 0) {
            stats[2 * row] = mean;
            stats[2 * row + 1] = rstd;
        }
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
            TaserPiece<T> y;
#pragma unroll
            for (int i = 0; i < EACH; ++i) y.x[i] = (T)fmaf(v[h][i] * rstd, weight[h][i], bias[h][i]);
            taser_store_piece<T>(out + row * p.width, (int64_t)(h * threads + lane) * EACH, p.width, y);
        }
    }
}

template <typename T> __device__ inline void put_out(const Norm& p, int64_t c, float mean, float rstd, const TaserPiece<T>& v, T* to) {
    constexpr int EACH = kTaserEach<T>;
    float weight[EACH], bias[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) weight[i] = 1.f, bias[i] = 0.f;
    if (p.weight) taser_load_floats<EACH>(p.weight, p.weight_type, c, p.width, weight);
    if (p.bias) taser_load_floats<EACH>(p.bias, p.weight_type, c, p.width, bias);
    TaserPiece<T> y;
#pragma unroll
    for (int i = 0; i < EACH; ++i) y.x[i] = (T)fmaf(((float)v.x[i] - mean) * rstd, weight[i], bias[i]);
    taser_store_piece<T>(to, c, p.width, y);
}

// Longer rows: a block each. HELD pieces stay in registers; what is past them is read three times.
template <typename T, int HELD> __global__ __launch_bounds__(1024) void norm_long_kernel(const Norm p, const T* x, T* out, float* stats) {
    constexpr int EACH = kTaserEach<T>;
    __shared__ float2 shared[2][16];
    const T* from = x + (int64_t)blockIdx.x * p.x_stride;
    T* to = out + (int64_t)blockIdx.x * p.width;
    const int waves = blockDim.x >> 6;
    const int64_t step = blockDim.x * EACH, past = HELD * step + threadIdx.x * EACH;
    TaserPiece<T> held[HELD], v;
    load_row<T, HELD>(from, blockDim.x, threadIdx.x, p.width, held);
    float sum = 0.f, none = 0.f, squares = 0.f;
    auto add = [&](const TaserPiece<T>& piece) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) sum += (float)piece.x[i];
    };
#pragma unroll
    for (int h = 0; h < HELD; ++h) add(held[h]);
    for (int64_t c = past; c < p.width; c += step) {
        taser_load_piece<T>(from, c, p.width, (T)0.f, v);
        add(v);
    }
    group_sums<0>(sum, none, shared, 0, waves);
    const float mean = sum / (float)p.width;
    auto add_square = [&](const TaserPiece<T>& piece, int64_t c) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const float away = c + i < p.width ? (float)piece.x[i] - mean : 0.f;
            squares = fmaf(away, away, squares);
        }
    };
#pragma unroll
    for (int h = 0; h < HELD; ++h) add_square(held[h], h * step + threadIdx.x * EACH);
    for (int64_t c = past; c < p.width; c += step) {
        taser_load_piece<T>(from, c, p.width, (T)0.f, v);
        add_square(v, c);
    }
    group_sums<0>(squares, none, shared, 1, waves);
    const float rstd = 1.f / sqrtf(squares / (float)p.width + p.eps);
    if (stats && threadIdx.x == 0) {
        stats[2 * (int64_t)blockIdx.x] = mean;
        stats[2 * (int64_t)blockIdx.x + 1] = rstd;
    }
#pragma unroll
    for (int h = 0; h < HELD; ++h) put_out<T>(p, h * step + threadIdx.x * EACH, mean, rstd, held[h], to);
    for (int64_t c = past; c < p.width; c += step) {
        taser_load_piece<T>(from, c, p.width, (T)0.f, v);
        put_out<T>(p, c, mean, rstd, v, to);
    }
}

template <int S> struct Slot { static constexpr int value = S; };

// dx, and of each block [2][width] sums of dout xhat and dout, if `parts` is given.
template <typename T, int G, int HELD, int THREADS>
__global__ __launch_bounds__(THREADS) void norm_grad_kernel(const Norm p, int waves, const T* x, const T* dout, const float* stats, T* dx, float* parts) {
    constexpr int EACH = kTaserEach<T>, COLUMNS = HELD * EACH;
    __shared__ float2 shared[2][16];
    __shared__ float sums[THREADS <= 512 ? THREADS / 64 * 2 * COLUMNS * (G ? G : 64) : 1];   // (a block of more is one group)
    const int threads = G ? G : waves * 64, lane = threadIdx.x % threads, mine = threadIdx.x / threads, here = blockDim.x / threads;
    const int64_t groups = (int64_t)gridDim.x * here, turns = (p.rows + groups - 1) / groups;
    float weight[HELD][EACH], dweight[HELD][EACH] = {}, dbias[HELD][EACH] = {};
    load_weights<T, HELD>(p.weight, p.weight_type, threads, lane, p.width, 1.f, weight);
    // Two rows ahead of the one at hand are on their way. (One does as well: 16 384 x 4096 bf16 100 to 101 us with either, 12 000 x 100 f32 and its join 10.0.)
    TaserPiece<T> next_x[2][HELD], next_y[2][HELD];
    float2 next_stats[2];
    int64_t row = (int64_t)blockIdx.x * here + mine;
    auto load = [&](int slot, int64_t r) {
        r = r < p.rows ? r : p.rows - 1;
        load_row<T, HELD>(x + r * p.x_stride, threads, lane, p.width, next_x[slot]);
        load_row<T, HELD>(dout + r * p.dout_stride, threads, lane, p.width, next_y[slot]);
        next_stats[slot] = make_float2(stats[2 * r], stats[2 * r + 1]);
    };
    load(0, row);
    if (turns > 1) load(1, row + groups);
    const float by = 1.f / (float)p.width;
    auto take = [&](auto at, int64_t turn) {   // the row in a slot
        constexpr int slot = decltype(at)::value;
        const float mean = next_stats[slot].x, rstd = next_stats[slot].y;
        float xhat[HELD][EACH], y[HELD][EACH];
        float a = 0.f, b = 0.f;
#pragma unroll
        for (int h = 0; h < HELD; ++h)
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                xhat[h][i] = (int64_t)(h * threads + lane) * EACH + i < p.width ? ((float)next_x[slot][h].x[i] - mean) * rstd : 0.f;
                y[h][i] = (float)next_y[slot][h].x[i];
                const float g = y[h][i] * weight[h][i];   // 0 past the row's end, where dout was taken as 0
                a += g;
                b = fmaf(g, xhat[h][i], b);
            }
        if (turn + 2 < turns) load(slot, row + 2 * groups);
        group_sums<G>(a, b, shared, slot, waves);
        if (row < p.rows) {   // else its last turn
            a *= by;
            b *= by;
#pragma unroll
            for (int h = 0; h < HELD; ++h) {
                TaserPiece<T> d;
#pragma unroll
                for (int i = 0; i < EACH; ++i) {
                    d.x[i] = (T)(rstd * (fmaf(y[h][i], weight[h][i], -a) - xhat[h][i] * b));
                    dweight[h][i] = fmaf(y[h][i], xhat[h][i], dweight[h][i]);
                    dbias[h][i] += y[h][i];
                }
                taser_store_piece<T>(dx + row * p.width, (int64_t)(h * threads + lane) * EACH, p.width, d);
            }
        }
        row += groups;
    };
    for (int64_t turn = 0; turn < turns; turn += 2) {
        take(Slot<0>(), turn);
        if (turn + 1 < turns) take(Slot<1>(), turn + 1);
    }
    if (!parts) return;
    float* to = parts + (int64_t)blockIdx.x * 2 * p.width;
    // Groups of a part of a wave add up across it, then what is left of them in LDS, in their order.
    if (G)
#pragma unroll
        for (int m = G; m < 64; m <<= 1)
#pragma unroll
            for (int h = 0; h < HELD; ++h)
#pragma unroll
                for (int i = 0; i < EACH; ++i) {
                    dweight[h][i] += __shfl_xor(dweight[h][i], m);
                    dbias[h][i] += __shfl_xor(dbias[h][i], m);
                }
    const int units = G ? THREADS / 64 : here, unit = G ? threadIdx.x >> 6 : mine;
    if (units == 1) {
#pragma unroll
        for (int h = 0; h < HELD; ++h) {
            taser_store_as<float, EACH>(to, (int64_t)(h * threads + lane) * EACH, p.width, dweight[h]);
            taser_store_as<float, EACH>(to + p.width, (int64_t)(h * threads + lane) * EACH, p.width, dbias[h]);
        }
        return;
    }
    if (!G || (threadIdx.x & 63) < G) {
#pragma unroll
        for (int h = 0; h < HELD; ++h)
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                sums[(unit * 2 * COLUMNS + h * EACH + i) * threads + lane] = dweight[h][i];
                sums[(unit * 2 * COLUMNS + COLUMNS + h * EACH + i) * threads + lane] = dbias[h][i];
            }
    }
    __syncthreads();
    for (int at = threadIdx.x; at < 2 * COLUMNS * threads; at += blockDim.x) {
        float sum = 0.f;
        for (int u = 0; u < units; ++u) sum += sums[u * 2 * COLUMNS * threads + at];
        const int k = at / threads, which = k / COLUMNS, of = k % COLUMNS;
        const int64_t column = (int64_t)(of / EACH * threads + at % threads) * EACH + of % EACH;
        if (column < p.width) to[which * p.width + column] = sum;
    }
}

// dx of longer rows: a block each. HELD pieces of either input stay in registers; what is past them is read twice.
template <typename T, int HELD> __global__ __launch_bounds__(1024) void norm_grad_long_kernel(const Norm p, const T* x, const T* dout, const float* stats, T* dx) {
    constexpr int EACH = kTaserEach<T>;
    __shared__ float2 shared[2][16];
    const int64_t row = blockIdx.x, step = blockDim.x * EACH, past = HELD * step + threadIdx.x * EACH;
    const T *from = x + row * p.x_stride, *grads = dout + row * p.dout_stride;
    TaserPiece<T> held_x[HELD], held_y[HELD], v, y;
    load_row<T, HELD>(from, blockDim.x, threadIdx.x, p.width, held_x);
    load_row<T, HELD>(grads, blockDim.x, threadIdx.x, p.width, held_y);
    const float mean = stats[2 * row], rstd = stats[2 * row + 1];
    float a = 0.f, b = 0.f;
    auto times_weight = [&](int64_t c, const TaserPiece<T>& of, float (&g)[EACH]) {   // 0 past the row's end
#pragma unroll
        for (int i = 0; i < EACH; ++i) g[i] = 1.f;
        if (p.weight) taser_load_floats<EACH>(p.weight, p.weight_type, c, p.width, g);
#pragma unroll
        for (int i = 0; i < EACH; ++i) g[i] *= (float)of.x[i];
    };
    auto add = [&](int64_t c, const TaserPiece<T>& of_x, const TaserPiece<T>& of_y) {
        float g[EACH];
        times_weight(c, of_y, g);
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            a += g[i];
            if (c + i < p.width) b = fmaf(g[i], ((float)of_x.x[i] - mean) * rstd, b);
        }
    };
#pragma unroll
    for (int h = 0; h < HELD; ++h) add(h * step + threadIdx.x * EACH, held_x[h], held_y[h]);
    for (int64_t c = past; c < p.width; c += step) {
        taser_load_piece<T>(from, c, p.width, (T)0.f, v);
        taser_load_piece<T>(grads, c, p.width, (T)0.f, y);
        add(c, v, y);
    }
    group_sums<0>(a, b, shared, 0, blockDim.x >> 6);
    a /= (float)p.width;
    b /= (float)p.width;
    auto put = [&](int64_t c, const TaserPiece<T>& of_x, const TaserPiece<T>& of_y) {
        float g[EACH];
        TaserPiece<T> d;
        times_weight(c, of_y, g);
#pragma unroll
        for (int i = 0; i < EACH; ++i) d.x[i] = (T)(rstd * (g[i] - a - ((float)of_x.x[i] - mean) * rstd * b));
        taser_store_piece<T>(dx + row * p.width, c, p.width, d);
    };
#pragma unroll
    for (int h = 0; h < HELD; ++h) put(h * step + threadIdx.x * EACH, held_x[h], held_y[h]);
    for (int64_t c = past; c < p.width; c += step) {
        taser_load_piece<T>(from, c, p.width, (T)0.f, v);
        taser_load_piece<T>(grads, c, p.width, (T)0.f, y);
        put(c, v, y);
    }
}

// Sums of dout xhat and dout over a slice of the rows: a block has 64 pieces of columns, each of its waves rows of its own.
template <typename T> __global__ __launch_bounds__(256) void norm_columns_kernel(const Norm p, const T* x, const T* dout, const float* stats, float* parts) {
    constexpr int EACH = kTaserEach<T>;
    __shared__ float sums[3][2][EACH][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = ((int64_t)blockIdx.x * 64 + lane) * EACH;
    float dweight[EACH] = {}, dbias[EACH] = {};
    for (int64_t row = (int64_t)blockIdx.y * 4 + wave; row < p.rows; row += (int64_t)gridDim.y * 4) {
        const float mean = stats[2 * row], rstd = stats[2 * row + 1];
        TaserPiece<T> v, y;
        taser_load_piece<T>(x + row * p.x_stride, c, p.width, (T)0.f, v);
        taser_load_piece<T>(dout + row * p.dout_stride, c, p.width, (T)0.f, y);
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            dweight[i] = fmaf((float)y.x[i], ((float)v.x[i] - mean) * rstd, dweight[i]);
            dbias[i] += (float)y.x[i];
        }
    }
    if (wave) {
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            sums[wave - 1][0][i][lane] = dweight[i];
            sums[wave - 1][1][i][lane] = dbias[i];
        }
    }
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int w = 0; w < 3; ++w)
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            dweight[i] += sums[w][0][i][lane];
            dbias[i] += sums[w][1][i][lane];
        }
    float* to = parts + (int64_t)blockIdx.y * 2 * p.width;
    taser_store_as<float, EACH>(to, c, p.width, dweight);
    taser_store_as<float, EACH>(to + p.width, c, p.width, dbias);
}

// The parts' sums: 32 columns a block, 32 threads a column.
__global__ __launch_bounds__(1024) void norm_join_kernel(const float* parts, int64_t n_parts, int64_t width, int32_t type, void* dweight, void* dbias) {
    __shared__ float sums[32][33];
    const int column = threadIdx.x & 31, slice = threadIdx.x >> 5;
    const int64_t c = (int64_t)blockIdx.x * 32 + column;
    float sum = 0.f;
    if (c < 2 * width)
#pragma unroll 8
        for (int64_t i = slice; i < n_parts; i += 32) sum += parts[i * 2 * width + c];
    sums[slice][column] = sum;
    __syncthreads();
    sum = sums[column][slice];   // of a column, one slice a lane
#pragma unroll
    for (int m = 1; m < 32; m <<= 1) sum += __shfl_xor(sum, m);
    const int64_t at = (int64_t)blockIdx.x * 32 + slice;
    if (column || at >= 2 * width) return;
    void* to = at < width ? dweight : dbias;
    const float one[1] = {sum};
    if (to) taser_store_floats<1>(to, type, at < width ? at : at - width, width, one);
}

// ---- on the host ---------------------------------------------------------------------------------

// How rows are cut: lanes of a group (0: whole waves), waves of a group, pieces of a thread, threads of a block.
struct Shape { int lanes, waves, held, threads; };
// Groups of a part of a wave with one piece a lane, or of as many waves as it takes with `columns` columns a thread; blocks of 256 threads or so for the
// answer, 512 for the gradient, whose blocks' sums are fewer so.
Shape shape_of(int64_t width, int32_t type, int columns, int threads) {
    const int each = type == TASER_F32 ? 4 : 8, held = columns / each;
    const int64_t pieces = (width + each - 1) / each;
    for (int lanes = 8; lanes <= 64; lanes *= 2)
        if (pieces <= lanes) return {lanes, 1, 1, threads};
    const int waves = (int)((pieces + 64 * held - 1) / (64 * held));
    int groups = 1;
    while (2 * groups * waves * 64 <= threads) groups *= 2;
    return {0, waves, held, groups * waves * 64};
}
Shape forward_shape(int64_t width, int32_t type) { return shape_of(width, type, 16, 256); }
Shape grad_shape(int64_t width, int32_t type) { return shape_of(width, type, 8, 512); }
int64_t groups_of(const Shape& s) { return s.threads / (s.lanes ? s.lanes : s.waves * 64); }
int64_t blocks_of(int64_t rows, const Shape& s, int64_t most) {
    const int64_t blocks = (rows + groups_of(s) - 1) / groups_of(s);
    return blocks < most ? blocks : most;
}
// The gradient's: two of 512 threads a compute unit. More would read a little faster and leave more sums to join.
int64_t grad_blocks(const Norm& p, int32_t type) {
    const Shape s = grad_shape(p.width, type);
    return blocks_of(p.rows, s, 256 * (s.threads > 512 ? 1 : 2));
}
// Longer rows' slices for the sums by column.
int64_t column_slices(const Norm& p) {
    const int64_t n = (p.rows + 15) / 16;
    return n < 64 ? n : 64;
}
unsigned long_threads(int64_t width, int32_t type) {
    const int64_t pieces = (width + 31) / 32, threads = (pieces + 63) / 64 * 64;   // 32 columns a thread
    return (unsigned)(threads < 1024 ? threads : 1024);
}

template <typename T> int forward(const Norm& p, int32_t type, const void* x, void* out, float* stats, hipStream_t stream) {
    constexpr int MANY = 16 / kTaserEach<T>;
    TaserProfileSpan span(stream, "layer_norm");
    if (p.width > kHeld) {
        norm_long_kernel<T, 2 * MANY><<<(unsigned)p.rows, long_threads(p.width, type), 0, stream>>>(p, (const T*)x, (T*)out, stats);
    } else {
        const Shape s = forward_shape(p.width, type);
        const unsigned blocks = (unsigned)blocks_of(p.rows, s, 256 * (1024 / s.threads));
        auto run = [&](auto kernel) { kernel<<<blocks, s.threads, 0, stream>>>(p, s.waves, (const T*)x, (T*)out, stats); };
        if (s.lanes == 8) run(norm_kernel<T, 8, 1, 256>);
        else if (s.lanes == 16) run(norm_kernel<T, 16, 1, 256>);
        else if (s.lanes == 32) run(norm_kernel<T, 32, 1, 256>);
        else if (s.lanes == 64) run(norm_kernel<T, 64, 1, 256>);
        else run(norm_kernel<T, 0, MANY, 512>);
    }
    TASER_HIP_TRY(hipGetLastError());
    return TASER_OK;
}

template <typename T>
int backward(const Norm& p, int32_t type, const void* x, const void* dout, const float* stats, void* dx, void* dweight, void* dbias, float* parts, hipStream_t stream) {
    constexpr int EACH = kTaserEach<T>;
    int64_t n_parts;
    {
        TaserProfileSpan span(stream, "layer_norm_grad");
        if (p.width > kHeld) {
            n_parts = column_slices(p);
            norm_grad_long_kernel<T, 32 / EACH><<<(unsigned)p.rows, long_threads(p.width, type), 0, stream>>>(p, (const T*)x, (const T*)dout, stats, (T*)dx);
            const int64_t across = (p.width + 64 * EACH - 1) / (64 * EACH);
            if (parts) norm_columns_kernel<T><<<dim3((unsigned)across, (unsigned)n_parts), 256, 0, stream>>>(p, (const T*)x, (const T*)dout, stats, parts);
        } else {
            const Shape s = grad_shape(p.width, type);
            n_parts = grad_blocks(p, type);
            auto run = [&](auto kernel) { kernel<<<(unsigned)n_parts, s.threads, 0, stream>>>(p, s.waves, (const T*)x, (const T*)dout, stats, (T*)dx, parts); };
            if (s.lanes == 8) run(norm_grad_kernel<T, 8, 1, 512>);
            else if (s.lanes == 16) run(norm_grad_kernel<T, 16, 1, 512>);
            else if (s.lanes == 32) run(norm_grad_kernel<T, 32, 1, 512>);
            else if (s.lanes == 64) run(norm_grad_kernel<T, 64, 1, 512>);
            else if (s.threads <= 512) run(norm_grad_kernel<T, 0, 8 / EACH, 512>);
            else run(norm_grad_kernel<T, 0, 8 / EACH, 1024>);
        }
        TASER_HIP_TRY(hipGetLastError());
    }
    if (parts) {
        TaserProfileSpan span(stream, "layer_norm_grad_join");
        norm_join_kernel<<<(unsigned)((2 * p.width + 31) / 32), 1024, 0, stream>>>(parts, n_parts, p.width, p.weight_type, dweight, dbias);
        TASER_HIP_TRY(hipGetLastError());
    }
    return TASER_OK;
}

int norm_args(const taser_norm* n, const char* what, Norm* p) {
    if (!n) return taser_fail(TASER_E_ARG, "%s: null argument block", what);
    if (n->type < TASER_F32 || n->type > TASER_BF16) return taser_fail(TASER_E_ARG, "%s: unknown element type %d", what, n->type);
    if (n->weight_type != n->type && n->weight_type != TASER_F32) return taser_fail(TASER_E_ARG, "%s: weights are of the elements' type or float32", what);
    if (n->rows < 0 || n->width < 1) return taser_fail(TASER_E_ARG, "%s: negative number of rows, or empty rows", what);
    if (!taser_launch_fits((n->width + 15) / 16, 1024) || !taser_launch_fits(n->rows, n->width > kHeld ? 1024 : 1))
        return taser_fail(TASER_E_RANGE, "%s: too many rows or elements for one launch", what);
    if (!(n->eps >= 0.f) || n->eps > 3e38f) return taser_fail(TASER_E_ARG, "%s: eps must not be negative, and finite", what);
    if (n->rows && !n->x) return taser_fail(TASER_E_ARG, "%s: null rows", what);
    if (n->rows > 1 && n->x_stride < n->width) return taser_fail(TASER_E_ARG, "%s: rows overlap", what);
    *p = Norm{n->rows, n->width, n->x_stride, n->width, n->weight, n->bias, n->weight_type, n->eps};
    return TASER_OK;
}
uint64_t grad_bytes(const Norm& p, int32_t type) {
    if (!p.rows) return 0;
    return (uint64_t)(p.width > kHeld ? column_slices(p) : grad_blocks(p, type)) * 2 * (uint64_t)p.width * sizeof(float);
}

}  // namespace

extern "C" int taser_layer_norm(const taser_norm* n, void* out, float* stats, void* hip_stream) {
    Norm p;
    if (const int rc = norm_args(n, "layer_norm", &p)) return rc;
    if (!p.rows) return TASER_OK;
    if (!out) return taser_fail(TASER_E_ARG, "layer_norm: null output");
    hipStream_t stream = (hipStream_t)hip_stream;
    taser_clear_stale_hip_error();
    if (n->type == TASER_F32) return forward<float>(p, n->type, n->x, out, stats, stream);
    if (n->type == TASER_F16) return forward<_Float16>(p, n->type, n->x, out, stats, stream);
    return forward<__bf16>(p, n->type, n->x, out, stats, stream);
}

extern "C" int taser_layer_norm_grad_bytes(const taser_norm* n, uint64_t* work_bytes) {
    Norm p;
    if (const int rc = norm_args(n, "layer_norm_grad_bytes", &p)) return rc;
    if (!work_bytes) return taser_fail(TASER_E_ARG, "layer_norm_grad_bytes: null output");
    *work_bytes = grad_bytes(p, n->type);
    return TASER_OK;
}

extern "C" int taser_layer_norm_grad(const taser_norm* n, const float* stats, const void* dout, int64_t dout_stride, void* dx, void* dweight, void* dbias, void* work,
                                     uint64_t work_bytes, void* hip_stream) {
    Norm p;
    if (const int rc = norm_args(n, "layer_norm_grad", &p)) return rc;
    if (p.rows && (!stats || !dout || !dx)) return taser_fail(TASER_E_ARG, "layer_norm_grad: null statistics, output's gradient or dx");
    if (p.rows > 1 && dout_stride < p.width) return taser_fail(TASER_E_ARG, "layer_norm_grad: rows of the output's gradient overlap");
    p.dout_stride = dout_stride;
    const bool sums = dweight || dbias;
    if (sums && p.rows && (!work || work_bytes < grad_bytes(p, n->type))) return taser_fail(TASER_E_ARG, "layer_norm_grad: less workspace than taser_layer_norm_grad_bytes says");
    if (work && (uintptr_t)work % 16) return taser_fail(TASER_E_ARG, "layer_norm_grad: the workspace is not aligned to 16 bytes");
    if (!p.rows && !sums) return TASER_OK;
    hipStream_t stream = (hipStream_t)hip_stream;
    taser_clear_stale_hip_error();
    float* parts = sums ? (float*)work : nullptr;
    if (!p.rows) {   // sums of nothing
        TaserProfileSpan span(stream, "layer_norm_grad_join");
        norm_join_kernel<<<(unsigned)((2 * p.width + 31) / 32), 1024, 0, stream>>>(nullptr, 0, p.width, p.weight_type, dweight, dbias);
        TASER_HIP_TRY(hipGetLastError());
        return TASER_OK;
    }
    if (n->type == TASER_F32) return backward<float>(p, n->type, n->x, dout, stats, dx, dweight, dbias, parts, stream);
    if (n->type == TASER_F16) return backward<_Float16>(p, n->type, n->x, dout, stats, dx, dweight, dbias, parts, stream);
    return backward<__bf16>(p, n->type, n->x, dout, stats, dx, dweight, dbias, parts, stream);
}

// Layer norm and its gradient (taser_layer_norm, taser_layer_norm_grad).
//
//   out = xhat weight + bias,  xhat = (x - mean) rstd;  with g = dout weight:
//   dx = rstd (g - mean(g) - xhat mean(g xhat)),  dweight = sum over rows of dout xhat,  dbias = sum over rows of dout
//
// Both are bound by reading and writing rows once. A row belongs to a group of G threads, each with up to 16 of its columns in registers:
// mean first, then the squares of what is away from it (no difference of large sums). A group goes from row to row, its columns' weights and,
// in the gradient, its columns' sums of dweight and dbias staying in registers, the next row on its way; a block adds its groups' sums
// through LDS, a second launch the blocks', in an order that the sizes fix. Rows past 1024 threads' registers are read again for each
// of their passes, and dweight and dbias come from a kernel of their own, by columns.
#include "pieces.h"

namespace {

constexpr int kColumns = 16;                  // of a thread
constexpr int64_t kHeld = 1024 * kColumns;    // the longest row that is held

struct Norm {
    int64_t rows, width, x_stride, dout_stride;
    const void *weight, *bias;
    int32_t weight_type;
    float eps;
};

// Sums of two numbers over a group of G threads. Groups of more than a wave go through LDS, `turn` alternates between its two halves.
template <int G> __device__ inline void group_sums(float& a, float& b, float2 (*shared)[16], int turn) {
#pragma unroll
    for (int m = 1; m < (G < 64 ? G : 64); m <<= 1) {
        a += __shfl_xor(a, m);
        b += __shfl_xor(b, m);
    }
    if (G <= 64) return;
    const int wave = threadIdx.x >> 6, first = threadIdx.x / G * (G / 64);
    if ((threadIdx.x & 63) == 0) shared[turn & 1][wave] = make_float2(a, b);
    __syncthreads();
    a = b = 0.f;
#pragma unroll
    for (int w = 0; w < G / 64; ++w) {
        a += shared[turn & 1][first + w].x;
        b += shared[turn & 1][first + w].y;
    }
}

// Columns of this thread: piece h at (h G + lane) EACH.
template <typename T, int G, int HELD> __device__ inline void load_row(const T* row, int lane, int64_t width, TaserPiece<T> (&p)[HELD]) {
#pragma unroll
    for (int h = 0; h < HELD; ++h) taser_load_piece<T>(row, (int64_t)(h * G + lane) * kTaserEach<T>, width, (T)0.f, p[h]);
}
template <typename T, int G, int HELD> __device__ inline void load_weights(const void* from, int32_t type, int lane, int64_t width, float none, float (&w)[HELD][kTaserEach<T>]) {
#pragma unroll
    for (int h = 0; h < HELD; ++h) {
        if (from) {
            taser_load_floats<kTaserEach<T>>(from, type, (int64_t)(h * G + lane) * kTaserEach<T>, width, w[h]);
        } else {
#pragma unroll
            for (int i = 0; i < kTaserEach<T>; ++i) w[h][i] = none;
        }
    }
}

template <typename T, int G, int HELD, int THREADS> __global__ __launch_bounds__(THREADS) void norm_kernel(const Norm p, const T* x, T* out, float* stats) {
    constexpr int EACH = kTaserEach<T>, GROUPS = THREADS / G;
    __shared__ float2 shared[2][16];
    const int lane = threadIdx.x % G;
    const int64_t group = (int64_t)blockIdx.x * GROUPS + threadIdx.x / G, groups = (int64_t)gridDim.x * GROUPS, turns = (p.rows + groups - 1) / groups;
    float weight[HELD][EACH], bias[HELD][EACH];
    load_weights<T, G, HELD>(p.weight, p.weight_type, lane, p.width, 1.f, weight);
    load_weights<T, G, HELD>(p.bias, p.weight_type, lane, p.width, 0.f, bias);
    TaserPiece<T> next[HELD];
    // A group without a row of its own left takes the last one once more: it writes nothing.
    int64_t row = group;
    load_row<T, G, HELD>(x + (row < p.rows ? row : p.rows - 1) * p.x_stride, lane, p.width, next);
    const float by = 1.f / (float)p.width;
    for (int64_t turn = 0; turn < turns; ++turn, row += groups) {
        float v[HELD][EACH];
        float sum = 0.f, none = 0.f;
#pragma unroll
        for (int h = 0; h < HELD; ++h)
#pragma unroll
            for (int i = 0; i < EACH; ++i) sum += v[h][i] = (float)next[h].x[i];
        if (turn + 1 < turns) load_row<T, G, HELD>(x + (row + groups < p.rows ? row + groups : p.rows - 1) * p.x_stride, lane, p.width, next);
        group_sums<G>(sum, none, shared, 0);
        const float mean = sum * by;
        float squares = 0.f;
#pragma unroll
        for (int h = 0; h < HELD; ++h)
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                v[h][i] = (int64_t)(h * G + lane) * EACH + i < p.width ? v[h][i] - mean : 0.f;
                squares = fmaf(v[h][i], v[h][i], squares);
            }
        group_sums<G>(squares, none, shared, 1);
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
            taser_store_piece<T>(out + row * p.width, (int64_t)(h * G + lane) * EACH, p.width, y);
        }
    }
}

// Rows past 1024 threads' registers: a block each, read three times.
template <typename T> __global__ __launch_bounds__(1024) void norm_wide_kernel(const Norm p, const T* x, T* out, float* stats) {
    constexpr int EACH = kTaserEach<T>;
    __shared__ float2 shared[2][16];
    const T* from = x + (int64_t)blockIdx.x * p.x_stride;
    T* to = out + (int64_t)blockIdx.x * p.width;
    const int64_t step = 1024 * EACH;
    float sum = 0.f, none = 0.f, squares = 0.f;
    for (int64_t c = threadIdx.x * EACH; c < p.width; c += step) {
        TaserPiece<T> v;
        taser_load_piece<T>(from, c, p.width, (T)0.f, v);
#pragma unroll
        for (int i = 0; i < EACH; ++i) sum += (float)v.x[i];
    }
    group_sums<1024>(sum, none, shared, 0);
    const float mean = sum / (float)p.width;
    for (int64_t c = threadIdx.x * EACH; c < p.width; c += step) {
        TaserPiece<T> v;
        taser_load_piece<T>(from, c, p.width, (T)0.f, v);
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const float away = c + i < p.width ? (float)v.x[i] - mean : 0.f;
            squares = fmaf(away, away, squares);
        }
    }
    group_sums<1024>(squares, none, shared, 1);
    const float rstd = 1.f / sqrtf(squares / (float)p.width + p.eps);
    if (stats && threadIdx.x == 0) {
        stats[2 * (int64_t)blockIdx.x] = mean;
        stats[2 * (int64_t)blockIdx.x + 1] = rstd;
    }
    for (int64_t c = threadIdx.x * EACH; c < p.width; c += step) {
        TaserPiece<T> v;
        float weight[EACH], bias[EACH];
        taser_load_piece<T>(from, c, p.width, (T)0.f, v);
#pragma unroll
        for (int i = 0; i < EACH; ++i) weight[i] = 1.f, bias[i] = 0.f;
        if (p.weight) taser_load_floats<EACH>(p.weight, p.weight_type, c, p.width, weight);
        if (p.bias) taser_load_floats<EACH>(p.bias, p.weight_type, c, p.width, bias);
#pragma unroll
        for (int i = 0; i < EACH; ++i) v.x[i] = (T)fmaf(((float)v.x[i] - mean) * rstd, weight[i], bias[i]);
        taser_store_piece<T>(to, c, p.width, v);
    }
}

// dx, and of each block [2][width] sums of dout xhat and dout, if `parts` is given.
template <typename T, int G, int HELD, int THREADS>
__global__ __launch_bounds__(THREADS) void norm_grad_kernel(const Norm p, const T* x, const T* dout, const float* stats, T* dx, float* parts) {
    constexpr int EACH = kTaserEach<T>, GROUPS = THREADS / G, COLUMNS = HELD * EACH;
    __shared__ float2 shared[2][16];
    __shared__ float sums[GROUPS > 1 ? THREADS / 2 * COLUMNS : 1];
    const int lane = threadIdx.x % G, mine = threadIdx.x / G;
    const int64_t groups = (int64_t)gridDim.x * GROUPS, turns = (p.rows + groups - 1) / groups;
    float weight[HELD][EACH], dweight[HELD][EACH] = {}, dbias[HELD][EACH] = {};
    load_weights<T, G, HELD>(p.weight, p.weight_type, lane, p.width, 1.f, weight);
    TaserPiece<T> next_x[HELD], next_y[HELD];
    int64_t row = (int64_t)blockIdx.x * GROUPS + mine;
    float2 next_stats;
    auto load = [&](int64_t r) {
        r = r < p.rows ? r : p.rows - 1;
        load_row<T, G, HELD>(x + r * p.x_stride, lane, p.width, next_x);
        load_row<T, G, HELD>(dout + r * p.dout_stride, lane, p.width, next_y);
        next_stats = make_float2(stats[2 * r], stats[2 * r + 1]);
    };
    load(row);
    const float by = 1.f / (float)p.width;
    for (int64_t turn = 0; turn < turns; ++turn, row += groups) {
        const float mean = next_stats.x, rstd = next_stats.y;
        float xhat[HELD][EACH], y[HELD][EACH];
        float a = 0.f, b = 0.f;
#pragma unroll
        for (int h = 0; h < HELD; ++h)
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                xhat[h][i] = (int64_t)(h * G + lane) * EACH + i < p.width ? ((float)next_x[h].x[i] - mean) * rstd : 0.f;
                y[h][i] = (float)next_y[h].x[i];
                const float g = y[h][i] * weight[h][i];   // 0 past the row's end, where dout was taken as 0
                a += g;
                b = fmaf(g, xhat[h][i], b);
            }
        if (turn + 1 < turns) load(row + groups);
        group_sums<G>(a, b, shared, (int)turn);
        if (row >= p.rows) continue;   // its last turn
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
            taser_store_piece<T>(dx + row * p.width, (int64_t)(h * G + lane) * EACH, p.width, d);
        }
    }
    if (!parts) return;
    // The upper half of the groups hands its sums to the lower half, until one has them all.
    auto fold = [&](float (&of)[HELD][EACH]) {
#pragma unroll
        for (int half = GROUPS / 2; half >= 1; half >>= 1) {
            __syncthreads();
            if (mine >= half && mine < 2 * half) {
#pragma unroll
                for (int h = 0; h < HELD; ++h)
#pragma unroll
                    for (int i = 0; i < EACH; ++i) sums[(h * EACH + i) * (half * G) + (mine - half) * G + lane] = of[h][i];
            }
            __syncthreads();
            if (mine < half) {
#pragma unroll
                for (int h = 0; h < HELD; ++h)
#pragma unroll
                    for (int i = 0; i < EACH; ++i) of[h][i] += sums[(h * EACH + i) * (half * G) + mine * G + lane];
            }
        }
    };
    if (GROUPS > 1) {
        fold(dweight);
        fold(dbias);
    }
    if (mine) return;
    float* to = parts + (int64_t)blockIdx.x * 2 * p.width;
#pragma unroll
    for (int h = 0; h < HELD; ++h) {
        taser_store_as<float, EACH>(to, (int64_t)(h * G + lane) * EACH, p.width, dweight[h]);
        taser_store_as<float, EACH>(to + p.width, (int64_t)(h * G + lane) * EACH, p.width, dbias[h]);
    }
}

template <typename T> __global__ __launch_bounds__(1024) void norm_grad_wide_kernel(const Norm p, const T* x, const T* dout, const float* stats, T* dx) {
    constexpr int EACH = kTaserEach<T>;
    __shared__ float2 shared[2][16];
    const int64_t row = blockIdx.x, step = 1024 * EACH;
    const float mean = stats[2 * row], rstd = stats[2 * row + 1];
    TaserPiece<T> v, y;
    float g[EACH], a = 0.f, b = 0.f;
    auto load = [&](int64_t c) {   // g is 0 past the row's end
        taser_load_piece<T>(x + row * p.x_stride, c, p.width, (T)0.f, v);
        taser_load_piece<T>(dout + row * p.dout_stride, c, p.width, (T)0.f, y);
#pragma unroll
        for (int i = 0; i < EACH; ++i) g[i] = 1.f;
        if (p.weight) taser_load_floats<EACH>(p.weight, p.weight_type, c, p.width, g);
#pragma unroll
        for (int i = 0; i < EACH; ++i) g[i] *= (float)y.x[i];
    };
    for (int64_t c = threadIdx.x * EACH; c < p.width; c += step) {
        load(c);
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            a += g[i];
            if (c + i < p.width) b = fmaf(g[i], ((float)v.x[i] - mean) * rstd, b);
        }
    }
    group_sums<1024>(a, b, shared, 0);
    a /= (float)p.width;
    b /= (float)p.width;
    for (int64_t c = threadIdx.x * EACH; c < p.width; c += step) {
        load(c);
#pragma unroll
        for (int i = 0; i < EACH; ++i) v.x[i] = (T)(rstd * (g[i] - a - ((float)v.x[i] - mean) * rstd * b));
        taser_store_piece<T>(dx + row * p.width, c, p.width, v);
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

// Threads to a row and pieces to a thread.
struct Shape { int group, held; };
Shape shape_of(int64_t width, int32_t type) {
    const int each = type == TASER_F32 ? 4 : 8, most = kColumns / each;
    const int64_t pieces = (width + each - 1) / each;
    int group = 8;
    while (group < 64 && group < pieces) group *= 2;
    if (pieces <= group) return {group, 1};
    while (group < 1024 && (int64_t)group * most < pieces) group *= 2;
    return {group, most};
}

// Blocks that a call of so many rows has, groups of `group` threads in blocks of `threads`: two to four a compute unit.
int64_t norm_blocks(int64_t rows, int group, int threads, int64_t most) {
    const int64_t each = threads / group, blocks = (rows + each - 1) / each;
    return blocks < most ? blocks : most;
}
int grad_threads(int group) { return group <= 512 ? 512 : 1024; }
int64_t grad_blocks(const Norm& p, int32_t type) {
    const Shape s = shape_of(p.width, type);
    const int threads = grad_threads(s.group);
    return norm_blocks(p.rows, s.group, threads, threads == 512 ? 512 : 256);
}
// The wide kernels' slices of the rows.
int64_t column_slices(const Norm& p) {
    const int64_t n = (p.rows + 15) / 16;
    return n < 64 ? n : 64;
}

template <typename T, int G, int HELD> void run_norm(const Norm& p, const T* x, T* out, float* stats, hipStream_t stream) {
    constexpr int THREADS = G <= 256 ? 256 : G;
    const int64_t blocks = norm_blocks(p.rows, G, THREADS, 256 * (1024 / THREADS));
    norm_kernel<T, G, HELD, THREADS><<<(unsigned)blocks, THREADS, 0, stream>>>(p, x, out, stats);
}
template <typename T, int G, int HELD> void run_grad(const Norm& p, const T* x, const T* dout, const float* stats, T* dx, float* parts, int64_t blocks, hipStream_t stream) {
    constexpr int THREADS = G <= 512 ? 512 : 1024;
    norm_grad_kernel<T, G, HELD, THREADS><<<(unsigned)blocks, THREADS, 0, stream>>>(p, x, dout, stats, dx, parts);
}

// run(G, HELD) of the row's shape, as compile-time numbers.
template <int G> struct Group { static constexpr int value = G; };
template <int H> struct Held { static constexpr int value = H; };
template <typename T, typename F> void with_shape(Shape s, F&& run) {
    constexpr int MOST = kColumns / kTaserEach<T>;
    if (s.held == 1) {
        if (s.group == 8) run(Group<8>(), Held<1>());
        else if (s.group == 16) run(Group<16>(), Held<1>());
        else if (s.group == 32) run(Group<32>(), Held<1>());
        else run(Group<64>(), Held<1>());
    } else {
        if (s.group == 64) run(Group<64>(), Held<MOST>());
        else if (s.group == 128) run(Group<128>(), Held<MOST>());
        else if (s.group == 256) run(Group<256>(), Held<MOST>());
        else if (s.group == 512) run(Group<512>(), Held<MOST>());
        else run(Group<1024>(), Held<MOST>());
    }
}

template <typename T> int forward(const Norm& p, int32_t type, const void* x, void* out, float* stats, hipStream_t stream) {
    TaserProfileSpan span(stream, "layer_norm");
    if (p.width > kHeld) norm_wide_kernel<T><<<(unsigned)p.rows, 1024, 0, stream>>>(p, (const T*)x, (T*)out, stats);
    else with_shape<T>(shape_of(p.width, type), [&](auto g, auto h) { run_norm<T, decltype(g)::value, decltype(h)::value>(p, (const T*)x, (T*)out, stats, stream); });
    TASER_HIP_TRY(hipGetLastError());
    return TASER_OK;
}

template <typename T>
int backward(const Norm& p, int32_t type, const void* x, const void* dout, const float* stats, void* dx, void* dweight, void* dbias, float* parts, hipStream_t stream) {
    int64_t n_parts;
    {
        TaserProfileSpan span(stream, "layer_norm_grad");
        if (p.width > kHeld) {
            n_parts = column_slices(p);
            norm_grad_wide_kernel<T><<<(unsigned)p.rows, 1024, 0, stream>>>(p, (const T*)x, (const T*)dout, stats, (T*)dx);
            const int64_t across = (p.width + 64 * kTaserEach<T> - 1) / (64 * kTaserEach<T>);
            if (parts) norm_columns_kernel<T><<<dim3((unsigned)across, (unsigned)n_parts), 256, 0, stream>>>(p, (const T*)x, (const T*)dout, stats, parts);
        } else {
            n_parts = grad_blocks(p, type);
            with_shape<T>(shape_of(p.width, type), [&](auto g, auto h) {
                run_grad<T, decltype(g)::value, decltype(h)::value>(p, (const T*)x, (const T*)dout, stats, (T*)dx, parts, n_parts, stream);
            });
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

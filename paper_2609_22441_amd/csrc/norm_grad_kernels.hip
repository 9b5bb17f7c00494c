// Gradients of the norms around a block, its gate and its residual sum.
//
// 65,536 x 4,096 bf16 with gate, residual and both norms 800 us (4.29 GB at 5.4 TB/s; in pieces through the
// caches 1,999), 50,000 x 512 bf16, a layer norm alone, 49 (two launches; 154 MB at 3.4 TB/s).
#include "norm_choice.h"
#include "norm_device.h"

namespace ccj {
namespace {

constexpr int kThreads = 256;
constexpr int kWide = 1024;                        // of rows of any length

// What the gradient of a row's elements needs of the whole row.
struct RowStats {
    RowNorm post, pre;
    // Means over the row: of pre's t and t * yn, of post's F and F * fn; 0 where the norm has none.
    float t, t_yn, v, v_fn;
};

int64_t padded_cols(int32_t cols) { return ((int64_t)cols + kCols - 1) / kCols * kCols; }

// The gradient of a norm's input from that of its normalised value vn, of a block: 1 / its size r and the
// row's means. Without a norm an infinity stays where it is.
__device__ __forceinline__ void norm_back(int norm, const float (&t)[kCols], const float (&vn)[kCols],
                                          float r, float mean_t, float mean_t_vn, float (&d)[kCols]) {
    if (norm == kNormNone) {
#pragma unroll
        for (int i = 0; i < kCols; ++i)
            d[i] = t[i];
    } else {
#pragma unroll
        for (int i = 0; i < kCols; ++i)
            d[i] = r * (t[i] - mean_t - vn[i] * mean_t_vn);
    }
}

// ---- rows in registers ----

// Wavefronts on a SIMD: with at most 15 registers of a lane spilled, but for rows beyond 4,096 columns, of
// which kernels with biases spill 5 to 26 with a stream in 16 bits, 32 to 75 with one in 32, and those of
// 32-bit elements without biases 16 to 22.
template <typename T, typename S, int B, bool BIAS>
constexpr int grad_wavefronts() {
    return B == 2 ? 2 : (BIAS ? 3 : 4) - (sizeof(T) == 4);
}

// L lanes of a row hold B blocks of 8 columns each, and for all the rows that they go through the sums over
// rows of their columns; with a stream in 16 bits and more than a wavefront L at most, the workgroup's. One
// read of f, gate, x, dy and dh, one write of dx, df and dgate; four sums over the row's lanes one after
// another, two more with layer norms. Between these the vector units are what is short (65,536 x 4,096 bf16:
// 750 instructions a lane and row were 55 % of their time at 1,226 us), so that nothing is divided and no
// weight multiplied with scale for each row; and registers, of which a wavefront may have 128 for four on a
// unit: what is behind one of the sums is computed again from the elements as they were read, and vectors
// wait in LDS.
// At the end the groups of lanes of a workgroup add up their sums in order. BIAS: with post's bias or the
// sums of either bias. partial: [workgroups][kSums][padded columns].
template <typename T, typename S, int L, int B, bool TAIL, bool BIAS>
__global__ __launch_bounds__(L <= 64 ? kThreads : L, (grad_wavefronts<T, S, B, BIAS>())) void row_grad_kernel(
    NormGradArgs ga, float *partial, int64_t padded) {
    const NormArgs &a = ga.a;
    constexpr int kGroups = L <= 64 ? kThreads / L : 1;
    constexpr bool kFewer = L > 64 && sizeof(S) == 2;
    constexpr int kV = BIAS ? kSums : 2;          // of Sum, the biases come last
    __shared__ float place[2][2][L > 64 ? L / 64 : 1];
    RowSum<L, kFewer> sum(place);
    const int lane = threadIdx.x % L, lanes = kFewer ? blockDim.x : L;
    const float per = 1.0f / (float)a.cols;
    int col[B], exchange[B];
    float w[B][kCols], sums[kV][B][kCols] = {};
    // The vectors that a row's elements meet once or twice wait in LDS, where lanes' halves of a block lie
    // side by side: pre's weight, post's bias.
    typedef float four_t __attribute__((ext_vector_type(4)));
    __shared__ __attribute__((aligned(16))) four_t waiting[BIAS ? 2 : 1][B][2][L];
    auto vector = [&](int which, int i, float(&x)[kCols]) {
        const four_t low = waiting[which][i][0][lane], high = waiting[which][i][1][lane];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            x[e] = low[e];
            x[4 + e] = high[e];
        }
    };
#pragma unroll
    for (int i = 0; i < B; ++i) {
        col[i] = (lane + i * lanes) * kCols;
        exchange[i] = exchange_of(lane + i * lanes, a.cols);
        vector_block(a.post_weight, col[i], a.cols, 1.0f, w[i]);
        times(w[i], a.scale);
        if (threadIdx.x < L)
#pragma unroll
            for (int which = 0; which < (BIAS ? 2 : 1); ++which) {
                float x[kCols];
                vector_block(which ? a.post_bias : a.pre_weight, col[i], a.cols, which ? 0.0f : 1.0f, x);
                times(x, which ? a.scale : 1.0f);
                waiting[which][i][0][lane] = four_t{x[0], x[1], x[2], x[3]};
                waiting[which][i][1][lane] = four_t{x[4], x[5], x[6], x[7]};
            }
    }
    __syncthreads();
    auto fetch = [&](auto &to, auto type, const void *p, int64_t stride, int64_t row) {
        using E = decltype(type);
#pragma unroll
        for (int i = 0; i < B; ++i)
            to[i] = p ? held_block<TAIL>(row_of<E>(p, stride, row), col[i], a.cols, exchange[i])
                      : Raw<E>{};
    };
    // Three wavefronts on a unit have registers for a row in 16 bits on its way while the row before is
    // computed: layer norms of 50,000 x 512 bf16 94 us, 101 without; with a stream in 32 bits they have
    // not (131,072 x 128 79 us, 167 with it), nor have four wavefronts.
    constexpr bool kAhead = L <= 64 && B == 1 && BIAS && sizeof(S) == 2;
    Raw<T> next_f[B], next_u[B], next_dh[B];
    Raw<S> next_x[B], next_dy[B];
    const int64_t first_row = (int64_t)blockIdx.x * kGroups + group_of_lanes<L>();
    auto fetch_next = [&](int64_t row) {
        fetch(next_f, T(), a.f, a.f_stride, row);
        fetch(next_u, T(), a.gate, a.gate_stride, row);
        fetch(next_x, S(), a.x, a.x_stride, row);
        fetch(next_dh, T(), ga.dh, ga.dh_stride, row);
        fetch(next_dy, S(), ga.dy, ga.dy_stride, row);
    };
    if (kAhead && first_row < a.n)
        fetch_next(first_row);
    for (int64_t row = first_row; row < a.n; row += (int64_t)gridDim.x * kGroups) {
        Raw<T> f[B], u[B], dh[B];
        Raw<S> x[B], dy[B];
        if constexpr (kAhead) {
            f[0] = next_f[0];
            u[0] = next_u[0];
            x[0] = next_x[0];
            dh[0] = next_dh[0];
            dy[0] = next_dy[0];
            if (row + (int64_t)gridDim.x * kGroups < a.n)
                fetch_next(row + (int64_t)gridDim.x * kGroups);
        } else {
            fetch(f, T(), a.f, a.f_stride, row);
            fetch(u, T(), a.gate, a.gate_stride, row);
            fetch(x, S(), a.x, a.x_stride, row);
            fetch(dh, T(), ga.dh, ga.dh_stride, row);
            fetch(dy, S(), ga.dy, ga.dy_stride, row);
        }
#pragma unroll
        for (int i = 0; i < B; ++i)
            settle(f[i], exchange[i]);
        RowStats st = {};
        float v[B][kCols], g[B][kCols], slope[B][kCols], y[B][kCols];
#pragma unroll
        for (int i = 0; i < B; ++i)
            numbers(f[i], v[i]);
        st.post = norm_of<TAIL>(a.post, v, col, a.cols, per, a.post_eps, sum);
#pragma unroll
        for (int i = 0; i < B; ++i) {
            settle(u[i], exchange[i]);
            settle(x[i], exchange[i]);
            settle(dh[i], exchange[i]);
            settle(dy[i], exchange[i]);
            float gate[kCols], stream[kCols], b[kCols] = {};
            numbers(u[i], gate);
            numbers(x[i], stream);
            gate_block<true>(a.gate_kind, gate, g[i], slope[i]);
            normalised(a.post, v[i], st.post, v[i]);
            if (BIAS)
                vector(1, i, b);
            block_sum(stream, g[i], v[i], w[i], b, y[i]);
        }
        if (ga.dh) {
            st.pre = norm_of<TAIL>(a.pre, y, col, a.cols, per, a.pre_eps, sum);
            float s[2] = {};                      // of t * yn and t, which is 0 where the row has no column
#pragma unroll
            for (int i = 0; i < B; ++i) {
                float d[kCols], yn[kCols], q[kCols];
                vector(0, i, q);
                numbers(dh[i], d);
                normalised(a.pre, y[i], st.pre, yn);
#pragma unroll
                for (int e = 0; e < kCols; ++e) {
                    s[0] += d[e] * q[e] * yn[e];
                    sums[kPreWeight][i][e] += d[e] * yn[e];
                    if (BIAS)
                        sums[kPreBias][i][e] += d[e];
                }
                if (a.pre == kNormLayer)
#pragma unroll
                    for (int e = 0; e < kCols; ++e)
                        s[1] += d[e] * q[e];
#pragma unroll
                for (int e = 0; e < kCols; ++e)
                    again(y[i][e]);
                again(dh[i]);
            }
            if (a.pre == kNormLayer) {
                sum(s);
                st.t = s[1] * per;
                st.t_yn = s[0] * per;
            } else if (a.pre == kNormRms) {
                st.t_yn = sum(s[0]) * per;
            }
#pragma unroll
            for (int i = 0; i < B; ++i) {
                float d[kCols], t[kCols], yn[kCols], q[kCols];
                vector(0, i, q);
                numbers(dh[i], t);
                numbers(dy[i], d);
                normalised(a.pre, y[i], st.pre, yn);
#pragma unroll
                for (int e = 0; e < kCols; ++e)
                    t[e] *= q[e];
                norm_back(a.pre, t, yn, st.pre.r, st.t, st.t_yn, y[i]);
#pragma unroll
                for (int e = 0; e < kCols; ++e)
                    y[i][e] += d[e];
            }
        } else {
#pragma unroll
            for (int i = 0; i < B; ++i)
                numbers(dy[i], y[i]);
        }
        // y now holds the gradient of x.
        float s[2] = {};
#pragma unroll
        for (int i = 0; i < B; ++i) {
            if (ga.dx)
                put_held<TAIL>(row_of<S>(ga.dx, ga.dx_stride, row), col[i], a.cols, exchange[i], y[i]);
#pragma unroll
            for (int e = 0; e < kCols; ++e) {
                const float d = y[i][e] * g[i][e];
                s[0] += d * w[i][e] * v[i][e];
                sums[kPostWeight][i][e] += d * v[i][e];
                if (BIAS)
                    sums[kPostBias][i][e] += d;
            }
            if (a.post == kNormLayer)
#pragma unroll
                for (int e = 0; e < kCols; ++e)
                    s[1] += y[i][e] * g[i][e] * w[i][e];
#pragma unroll
            for (int e = 0; e < kCols; ++e)
                again(g[i][e]);
        }
        if (a.post == kNormLayer) {
            sum(s);
            st.v = s[1] * per;
            st.v_fn = s[0] * per;
        } else if (a.post == kNormRms) {
            st.v_fn = sum(s[0]) * per;
        }
#pragma unroll
        for (int i = 0; i < B; ++i) {
            float t[kCols], df[kCols], du[kCols], b[kCols] = {};
            if (BIAS)
                vector(1, i, b);
#pragma unroll
            for (int e = 0; e < kCols; ++e) {
                t[e] = y[i][e] * g[i][e] * w[i][e];
                du[e] = y[i][e] * (v[i][e] * w[i][e] + b[e]) * slope[i][e];
            }
            norm_back(a.post, t, v[i], st.post.r, st.v, st.v_fn, df);
            if (ga.dgate)
                put_held<TAIL>(row_of<T>(ga.dgate, ga.dgate_stride, row), col[i], a.cols, exchange[i],
                               du);
            put_held<TAIL>(row_of<T>(ga.df, ga.df_stride, row), col[i], a.cols, exchange[i], df);
        }
    }
#pragma unroll
    for (int i = 0; i < B; ++i) {
        times(sums[kPostWeight][i], a.scale);
        if (BIAS)
            times(sums[kPostBias][i], a.scale);
    }
    if constexpr (kGroups == 1) {
#pragma unroll
        for (int v = 0; v < kV; ++v)
#pragma unroll
            for (int i = 0; i < B; ++i)
                if (ga.sums[v] && col[i] < a.cols)
                    store_block(partial + ((int64_t)blockIdx.x * kSums + v) * padded + col[i],
                                sums[v][i]);
    } else {
        __shared__ float part[kGroups][B * L * kCols];
#pragma unroll
        for (int v = 0; v < kV; ++v) {
            if (!ga.sums[v])
                continue;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < B; ++i)
#pragma unroll
                for (int e = 0; e < kCols; ++e)
                    part[threadIdx.x / L][col[i] + e] = sums[v][i][e];
            __syncthreads();
            for (int at = threadIdx.x; at < a.cols; at += kThreads) {
                float s = 0.0f;
#pragma unroll
                for (int g = 0; g < kGroups; ++g)
                    s += part[g][at];
                partial[((int64_t)blockIdx.x * kSums + v) * padded + at] = s;
            }
        }
    }
}

// ---- rows of any length ----

// The elements of a block and their gradients, in steps that need one more sum of the row each.
template <typename T, typename S>
struct Gradient {
    float w[kCols], b[kCols], q[kCols], fn[kCols], g[kCols], slope[kCols], y[kCols], yn[kCols], dh[kCols],
        t[kCols], dy[kCols], v[kCols];
    __device__ __forceinline__ void weights(const NormArgs &a, int col) {
        vector_block(a.post_weight, col, a.cols, 1.0f, w);
        vector_block(a.post_bias, col, a.cols, 0.0f, b);
        vector_block(a.pre_weight, col, a.cols, 1.0f, q);
        times(w, a.scale);
        times(b, a.scale);
    }
    __device__ __forceinline__ void of_f(const NormArgs &a, int64_t row, int col) {
        numbers(row_block(row_of<T>(a.f, a.f_stride, row), col, a.cols), fn);
    }
    __device__ __forceinline__ void of_block(const NormArgs &a, int64_t row, int col,
                                             const RowNorm &post) {
        float u[kCols], x[kCols];
        of_f(a, row, col);
        normalised(a.post, fn, post, fn);
        numbers(a.gate ? row_block(row_of<T>(a.gate, a.gate_stride, row), col, a.cols) : Raw<T>{}, u);
        numbers(a.x ? row_block(row_of<S>(a.x, a.x_stride, row), col, a.cols) : Raw<S>{}, x);
        gate_block<true>(a.gate_kind, u, g, slope);
        block_sum(x, g, fn, w, b, y);
    }
    __device__ __forceinline__ void of_pre(const NormGradArgs &ga, int64_t row, int col,
                                           const RowNorm &pre) {
        if (!ga.dh)
            return;
        numbers(row_block(row_of<T>(ga.dh, ga.dh_stride, row), col, ga.a.cols), dh);
        normalised(ga.a.pre, y, pre, yn);
#pragma unroll
        for (int i = 0; i < kCols; ++i)
            t[i] = dh[i] * q[i];
    }
    __device__ __forceinline__ void of_sum(const NormGradArgs &ga, int64_t row, int col,
                                           const RowStats &s) {
        float d[kCols];
        numbers(ga.dy ? row_block(row_of<S>(ga.dy, ga.dy_stride, row), col, ga.a.cols) : Raw<S>{}, dy);
        if (ga.dh) {
            norm_back(ga.a.pre, t, yn, s.pre.r, s.t, s.t_yn, d);
#pragma unroll
            for (int i = 0; i < kCols; ++i)
                dy[i] += d[i];
        }
#pragma unroll
        for (int i = 0; i < kCols; ++i)
            v[i] = dy[i] * g[i] * w[i];
    }
};

// Each row's statistics, a workgroup a row: passes over the row as in the forward kernel, then one for
// the sums of either norm's gradient.
template <typename T, typename S>
__global__ __launch_bounds__(kWide) void wide_stats_kernel(NormGradArgs ga, RowStats *stats) {
    const NormArgs &a = ga.a;
    __shared__ float place[2][2][kWide / 64];
    RowSum<kWide> sum(place);
    const float per = 1.0f / (float)a.cols;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        auto over = [&](auto &&use) {
            for (int col = threadIdx.x * kCols; col < a.cols; col += kWide * kCols)
                use(col);
        };
        RowStats st = {};
        Gradient<T, S> p;
        float s[2] = {};
        if (a.post == kNormLayer) {
            over([&](int col) {
                p.of_f(a, row, col);
                s[0] += plain_sum(p.fn);
            });
            st.post.mean = sum(s[0]) * per;
        }
        if (a.post != kNormNone) {
            s[0] = 0.0f;
            over([&](int col) {
                p.of_f(a, row, col);
                s[0] += squares<true>(p.fn, st.post.mean, col, a.cols);
            });
            st.post.r = inverse_size(sum(s[0]) * per, a.post_eps);
        }
        auto forward = [&](int col) {
            p.weights(a, col);
            p.of_block(a, row, col, st.post);
        };
        if (a.pre == kNormLayer) {
            s[0] = 0.0f;
            over([&](int col) {
                forward(col);                     // y is 0 where the row has no column
                s[0] += plain_sum(p.y);
            });
            st.pre.mean = sum(s[0]) * per;
        }
        if (a.pre != kNormNone) {
            s[0] = 0.0f;
            over([&](int col) {
                forward(col);
                s[0] += squares<true>(p.y, st.pre.mean, col, a.cols);
            });
            st.pre.r = inverse_size(sum(s[0]) * per, a.pre_eps);
            s[0] = s[1] = 0.0f;
            over([&](int col) {
                forward(col);
                p.of_pre(ga, row, col, st.pre);
#pragma unroll
                for (int i = 0; i < kCols; ++i) {
                    s[0] += p.t[i];               // 0 there, too
                    s[1] += p.t[i] * p.yn[i];
                }
            });
            sum(s);
            st.t = a.pre == kNormLayer ? s[0] * per : 0.0f;
            st.t_yn = s[1] * per;
        }
        if (a.post != kNormNone) {
            s[0] = s[1] = 0.0f;
            over([&](int col) {
                forward(col);
                p.of_pre(ga, row, col, st.pre);
                p.of_sum(ga, row, col, st);
#pragma unroll
                for (int i = 0; i < kCols; ++i) {
                    s[0] += p.v[i];
                    s[1] += p.v[i] * p.fn[i];
                }
            });
            sum(s);
            st.v = a.post == kNormLayer ? s[0] * per : 0.0f;
            st.v_fn = s[1] * per;
        }
        if (threadIdx.x == 0)
            stats[row] = st;
    }
}

// The elements' gradients from the rows' statistics: a thread takes a block of columns through a strip
// of rows and keeps its sums over them. partial: [strips][kSums][padded columns].
template <typename T, typename S>
__global__ __launch_bounds__(kThreads) void wide_grad_kernel(NormGradArgs ga, const RowStats *stats,
                                                             float *partial, int64_t padded) {
    const NormArgs &a = ga.a;
    const int64_t col64 = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * kCols;
    if (col64 >= a.cols)
        return;
    const int col = (int)col64;
    const int64_t first = a.n * blockIdx.y / gridDim.y, end = a.n * (blockIdx.y + 1) / gridDim.y;
    float sums[kSums][kCols] = {};
    Gradient<T, S> p;
    p.weights(a, col);
    for (int64_t row = first; row < end; ++row) {
        const RowStats st = stats[row];
        p.of_block(a, row, col, st.post);
        p.of_pre(ga, row, col, st.pre);
        p.of_sum(ga, row, col, st);
        float df[kCols], du[kCols];
#pragma unroll
        for (int i = 0; i < kCols; ++i) {
            const float dg = p.dy[i] * p.g[i];
            du[i] = p.dy[i] * (p.fn[i] * p.w[i] + p.b[i]) * p.slope[i];
            sums[kPostWeight][i] += dg * p.fn[i];
            sums[kPostBias][i] += dg;
        }
        norm_back(a.post, p.v, p.fn, st.post.r, st.v, st.v_fn, df);
        if (ga.dh)
#pragma unroll
            for (int i = 0; i < kCols; ++i) {
                sums[kPreWeight][i] += p.dh[i] * p.yn[i];
                sums[kPreBias][i] += p.dh[i];
            }
        if (ga.dx)
            put_block(row_of<S>(ga.dx, ga.dx_stride, row), col, a.cols, p.dy);
        if (ga.dgate)
            put_block(row_of<T>(ga.dgate, ga.dgate_stride, row), col, a.cols, du);
        put_block(row_of<T>(ga.df, ga.df_stride, row), col, a.cols, df);
    }
    times(sums[kPostWeight], a.scale);
    times(sums[kPostBias], a.scale);
#pragma unroll
    for (int s = 0; s < kSums; ++s)
        if (ga.sums[s])
            store_block(partial + ((int64_t)blockIdx.y * kSums + s) * padded + col, sums[s]);
}

// ---- the sums of all strips ----

constexpr int kFoldWaves = 16;

// 64 columns of one sum: every wavefront adds every 16th partial result, in order, then one of them
// the wavefronts' in order.
__global__ __launch_bounds__(64 * kFoldWaves) void fold_kernel(NormGradArgs ga, const float *partial,
                                                               int64_t strips, int64_t padded) {
    __shared__ float part[kFoldWaves][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, s = blockIdx.y;
    const int64_t col = (int64_t)blockIdx.x * 64 + lane;
    float *const to = ga.sums[s];
    if (!to)
        return;                                   // all of the workgroup
    float sum = 0.0f;
    if (col < ga.a.cols)
#pragma unroll 16
        for (int64_t i = wave; i < strips; i += kFoldWaves)
            sum += partial[(i * kSums + s) * padded + col];
    part[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && col < ga.a.cols) {
        sum = ga.accumulate ? to[col] : 0.0f;
#pragma unroll
        for (int w = 0; w < kFoldWaves; ++w)
            sum += part[w][lane];
        to[col] = sum;
    }
}

hipError_t fold(const NormGradArgs &g, const float *partial, int64_t strips, hipStream_t stream) {
    bool any = false;
    for (const float *s : g.sums)
        any = any || s;
    if (any)
        fold_kernel<<<dim3((unsigned)((g.a.cols + 63) / 64), kSums), 64 * kFoldWaves, 0, stream>>>(
            g, partial, strips, padded_cols(g.a.cols));
    return hipGetLastError();
}

template <typename T, typename S, int L, int B = 1>
hipError_t launch_rows(const NormGradArgs &g, int lanes, hipStream_t stream) {
    const NormArgs &a = g.a;
    const int threads = L <= 64 ? kThreads : lanes;
    const int64_t padded = padded_cols(a.cols), groups = norm_grad_groups(a.n, a.cols, sizeof(S) == 4);
    float *partial = static_cast<float *>(g.workspace);
    auto even = [](const void *p, int64_t stride) { return !p || even_rows(p, stride); };
    const bool tail = !(a.cols % kCols == 0 && even(a.f, a.f_stride) && even(a.x, a.x_stride) &&
                        even(a.gate, a.gate_stride) && even(g.dy, g.dy_stride) &&
                        even(g.dh, g.dh_stride) && even(g.dx, g.dx_stride) &&
                        even(g.df, g.df_stride) && even(g.dgate, g.dgate_stride));
    const bool bias = a.post_bias || g.sums[kPostBias] || g.sums[kPreBias];
    const unsigned grid = (unsigned)groups;
    if (tail && bias)
        row_grad_kernel<T, S, L, B, true, true><<<grid, threads, 0, stream>>>(g, partial, padded);
    else if (tail)
        row_grad_kernel<T, S, L, B, true, false><<<grid, threads, 0, stream>>>(g, partial, padded);
    else if (bias)
        row_grad_kernel<T, S, L, B, false, true><<<grid, threads, 0, stream>>>(g, partial, padded);
    else
        row_grad_kernel<T, S, L, B, false, false><<<grid, threads, 0, stream>>>(g, partial, padded);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? fold(g, partial, groups, stream) : e;
}

template <typename T, typename S>
hipError_t launch_types(const NormGradArgs &g, hipStream_t stream) {
    constexpr bool kWideStream = sizeof(S) == 4;
    const NormShape shape = norm_grad_shape(g.a.cols, kWideStream);
    switch (shape.lanes * 4 + shape.blocks) {
    case 16 * 4 + 1: return launch_rows<T, S, 16>(g, shape.lanes, stream);
    case 32 * 4 + 1: return launch_rows<T, S, 32>(g, shape.lanes, stream);
    case 64 * 4 + 1: return launch_rows<T, S, 64>(g, shape.lanes, stream);
    }
    if constexpr (kWideStream) {
        switch (shape.lanes * 4 + shape.blocks) {
        case 128 * 4 + 1: return launch_rows<T, S, 128>(g, shape.lanes, stream);
        case 256 * 4 + 1: return launch_rows<T, S, 256>(g, shape.lanes, stream);
        case 512 * 4 + 1: return launch_rows<T, S, 512>(g, shape.lanes, stream);
        case 512 * 4 + 2: return launch_rows<T, S, 512, 2>(g, shape.lanes, stream);
        }
    } else {
        if (shape.blocks == 2)
            return launch_rows<T, S, 64, 2>(g, shape.lanes, stream);
        if (shape.lanes > 512)
            return launch_rows<T, S, 1024>(g, shape.lanes, stream);
        if (shape.lanes)
            return launch_rows<T, S, 512>(g, shape.lanes, stream);
    }
    const int64_t padded = padded_cols(g.a.cols), strips = norm_wide_strips(g.a.n, g.a.cols);
    RowStats *stats = static_cast<RowStats *>(g.workspace);
    float *partial = reinterpret_cast<float *>(stats + g.a.n);
    const int64_t most = 1 << 20;
    wide_stats_kernel<T, S><<<(unsigned)(g.a.n < most ? g.a.n : most), kWide, 0, stream>>>(g, stats);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return e;
    const dim3 grid((unsigned)((padded / kCols + kThreads - 1) / kThreads), (unsigned)strips);
    wide_grad_kernel<T, S><<<grid, kThreads, 0, stream>>>(g, stats, partial, padded);
    const hipError_t e2 = hipGetLastError();
    return e2 == hipSuccess ? fold(g, partial, strips, stream) : e2;
}

}  // namespace

int64_t norm_grad_workspace_bytes(int64_t n, int32_t cols) {
    if (norm_grad_shape(cols, false).lanes) {     // room for either type of the residual stream
        const int64_t narrow = norm_grad_groups(n, cols, false), wide = norm_grad_groups(n, cols, true);
        return (narrow > wide ? narrow : wide) * kSums * padded_cols(cols) * 4;
    }
    return n * (int64_t)sizeof(RowStats) + norm_wide_strips(n, cols) * kSums * padded_cols(cols) * 4;
}

hipError_t launch_norm_grad(const NormGradArgs &g, hipStream_t stream) {
    static_assert(sizeof(RowStats) % 16 == 0, "what follows the statistics is aligned to 16 bytes");
    if (g.a.n == 0)                               // sums of nothing
        return g.accumulate ? hipSuccess : fold(g, nullptr, 0, stream);
    switch (g.a.type) {
    case kF32: return launch_types<float, float>(g, stream);
    case kF16:
        return g.a.stream_type == kF32 ? launch_types<half_t, float>(g, stream)
                                       : launch_types<half_t, half_t>(g, stream);
    default:
        return g.a.stream_type == kF32 ? launch_types<bf16_t, float>(g, stream)
                                       : launch_types<bf16_t, bf16_t>(g, stream);
    }
}

}  // namespace ccj

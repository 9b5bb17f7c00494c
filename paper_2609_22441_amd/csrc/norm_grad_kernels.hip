// Gradients of the norms around a block, its gate and its residual sum.
#include "norm_choice.h"
#include "norm_device.h"

namespace ccj {
namespace {

constexpr int kThreads = 256;

// What the gradient of a row's elements needs of the whole row.
struct RowStats {
    RowNorm post, pre;
    // Means over the row: of pre's t and t * yn, of post's F and F * fn; 0 where the norm has none.
    float t, t_yn, v, v_fn;
};

int64_t padded_cols(int32_t cols) { return ((int64_t)cols + kCols - 1) / kCols * kCols; }

// The elements of a block and their gradients, in steps that need one more sum of the row each.
template <typename T, typename S>
struct Gradient : Forward<T, S> {
    float yn[kCols], t[kCols], dy[kCols], v[kCols];
    using Forward<T, S>::fn, Forward<T, S>::g, Forward<T, S>::y;
    __device__ __forceinline__ void of_pre(const Raw<T> &dh, const float (&w)[kCols],
                                           const RowNorm &pre) {
#pragma unroll
        for (int i = 0; i < kCols; ++i) {
            yn[i] = (y[i] - pre.mean) * pre.r;
            t[i] = (float)dh[i] * w[i];
        }
    }
    // dy before post's weight: Y, and Y * scale.
    __device__ __forceinline__ void of_sum(const NormGradArgs &a, const Raw<S> &d,
                                           const RowStats &s) {
#pragma unroll
        for (int i = 0; i < kCols; ++i) {
            dy[i] = (float)d[i];
            if (a.dh)
                dy[i] += a.a.pre == kNormNone ? t[i] : s.pre.r * (t[i] - s.t - yn[i] * s.t_yn);
        }
    }
    __device__ __forceinline__ void of_post(const NormGradArgs &a, const float (&w)[kCols]) {
#pragma unroll
        for (int i = 0; i < kCols; ++i)
            v[i] = dy[i] * a.a.scale * g[i] * w[i];
    }
};

// ---- rows in registers ----

// L lanes of a row hold a block of 8 columns each, and for all the rows that they go through the weights of
// their columns and the sums over rows. One read of f, gate, x, dy and dh, one write of dx, df and dgate;
// four sums over the row's lanes one after another, two more with layer norms. At the end the groups of
// lanes of a workgroup add up their sums in order. BIAS: with post's bias or the sums of either bias.
// partial: [workgroups][kSums][padded columns].
template <typename T, typename S, int L, bool TAIL, bool BIAS>
__global__ __launch_bounds__(L < kThreads ? kThreads : L) void row_grad_kernel(NormGradArgs ga,
                                                                               float *partial,
                                                                               int64_t padded) {
    const NormArgs &a = ga.a;
    constexpr int kT = L < kThreads ? kThreads : L, kGroups = kT / L;
    constexpr int kV = BIAS ? kSums : 2;          // of Sum, the biases come last
    __shared__ float place[2][L > 64 ? L / 64 : 1][2];
    RowSum<L, 2> sum{place};
    const int lane = threadIdx.x % L, col = lane * kCols, exchange = exchange_of(lane, a.cols);
    const float cols = (float)a.cols;
    float w[kCols], b[kCols] = {}, q[kCols], sums[kV][kCols] = {};
    vector_block(a.post_weight, col, a.cols, 1.0f, w);
    if (BIAS)
        vector_block(a.post_bias, col, a.cols, 0.0f, b);
    vector_block(a.pre_weight, col, a.cols, 1.0f, q);
    auto in = [&](int e) { return col + (TAIL ? e : 0) < a.cols; };
    for (int64_t row = (int64_t)blockIdx.x * kGroups + threadIdx.x / L; row < a.n;
         row += (int64_t)gridDim.x * kGroups) {
        auto held = [&](auto type, const void *p, int64_t stride) {
            using E = decltype(type);
            return p ? held_block<TAIL>(row_of<E>(p, stride, row), col, a.cols, exchange) : Raw<E>{};
        };
        Raw<T> f = held(T(), a.f, a.f_stride), u = held(T(), a.gate, a.gate_stride);
        Raw<S> x = held(S(), a.x, a.x_stride);
        Raw<T> dh = held(T(), ga.dh, ga.dh_stride);
        Raw<S> dy = held(S(), ga.dy, ga.dy_stride);
        settle(f, exchange);
        RowStats st = {};
        if (a.post == kNormLayer) {
            float s = 0.0f;
#pragma unroll
            for (int e = 0; e < kCols; ++e)
                s += (float)f[e];
            st.post.mean = sum(s) / cols;
        }
        if (a.post != kNormNone) {
            float s = 0.0f;
#pragma unroll
            for (int e = 0; e < kCols; ++e) {
                const float d = (float)f[e] - st.post.mean;
                s += in(e) ? d * d : 0.0f;
            }
            st.post.r = inverse_size(sum(s), a.cols, a.post_eps);
        }
        settle(u, exchange);
        settle(x, exchange);
        Gradient<T, S> p;
        p(a, f, u, x, st.post, w, b);
        if (a.pre == kNormLayer) {
            float s = 0.0f;
#pragma unroll
            for (int e = 0; e < kCols; ++e)
                s += p.y[e];                      // 0 where the row has no column
            st.pre.mean = sum(s) / cols;
        }
        if (a.pre != kNormNone) {
            float s = 0.0f;
#pragma unroll
            for (int e = 0; e < kCols; ++e) {
                const float d = p.y[e] - st.pre.mean;
                s += in(e) ? d * d : 0.0f;
            }
            st.pre.r = inverse_size(sum(s), a.cols, a.pre_eps);
        }
        settle(dh, exchange);
        settle(dy, exchange);
        p.of_pre(dh, q, st.pre);
        if (a.pre != kNormNone) {
            float s[2] = {};
#pragma unroll
            for (int e = 0; e < kCols; ++e) {
                s[0] += p.t[e];
                s[1] += p.t[e] * p.yn[e];
            }
            sum(s);
            st.t = a.pre == kNormLayer ? s[0] / cols : 0.0f;
            st.t_yn = s[1] / cols;
        }
        p.of_sum(ga, dy, st);
        p.of_post(ga, w);
        if (a.post != kNormNone) {
            float s[2] = {};
#pragma unroll
            for (int e = 0; e < kCols; ++e) {
                s[0] += p.v[e];
                s[1] += p.v[e] * p.fn[e];
            }
            sum(s);
            st.v = a.post == kNormLayer ? s[0] / cols : 0.0f;
            st.v_fn = s[1] / cols;
        }
        float df[kCols], du[kCols];
#pragma unroll
        for (int e = 0; e < kCols; ++e) {
            const float d = p.dy[e] * a.scale;
            df[e] = a.post == kNormNone ? p.v[e] : st.post.r * (p.v[e] - st.v - p.fn[e] * st.v_fn);
            du[e] = d * p.n[e] * p.slope[e];
            sums[kPostWeight][e] += d * p.g[e] * p.fn[e];
            sums[kPreWeight][e] += (float)dh[e] * p.yn[e];
            if (BIAS) {
                sums[kPostBias][e] += d * p.g[e];
                sums[kPreBias][e] += (float)dh[e];
            }
        }
        if (ga.dx)
            put_held<TAIL>(row_of<S>(ga.dx, ga.dx_stride, row), col, a.cols, exchange, p.dy);
        if (ga.dgate)
            put_held<TAIL>(row_of<T>(ga.dgate, ga.dgate_stride, row), col, a.cols, exchange, du);
        put_held<TAIL>(row_of<T>(ga.df, ga.df_stride, row), col, a.cols, exchange, df);
    }
    if constexpr (kGroups == 1) {
        if (col < a.cols)
#pragma unroll
            for (int v = 0; v < kV; ++v)
                if (ga.sums[v])
                    store_block(partial + ((int64_t)blockIdx.x * kSums + v) * padded + col, sums[v]);
    } else {
        __shared__ float part[kGroups][L * kCols];
#pragma unroll
        for (int v = 0; v < kV; ++v) {
            if (!ga.sums[v])
                continue;
            __syncthreads();
#pragma unroll
            for (int e = 0; e < kCols; ++e)
                part[threadIdx.x / L][col + e] = sums[v][e];
            __syncthreads();
            for (int c = threadIdx.x; c < a.cols; c += kT) {
                float s = 0.0f;
#pragma unroll
                for (int g = 0; g < kGroups; ++g)
                    s += part[g][c];
                partial[((int64_t)blockIdx.x * kSums + v) * padded + c] = s;
            }
        }
    }
}

// ---- rows of any length ----

// Each row's statistics, a workgroup a row: passes over the row as in the forward kernel, then one for
// the sums of either norm's gradient.
template <typename T, typename S>
__global__ __launch_bounds__(kThreads) void wide_stats_kernel(NormGradArgs ga, RowStats *stats) {
    const NormArgs &a = ga.a;
    __shared__ float place[2][kThreads / 64][2];
    RowSum<kThreads, 2> sum{place};
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const T *f = row_of<T>(a.f, a.f_stride, row), *u = row_of<T>(a.gate, a.gate_stride, row);
        const S *x = row_of<S>(a.x, a.x_stride, row), *dy = row_of<S>(ga.dy, ga.dy_stride, row);
        const T *dh = row_of<T>(ga.dh, ga.dh_stride, row);
        const float cols = (float)a.cols;
        auto over = [&](auto &&use) {
            for (int col = threadIdx.x * kCols; col < a.cols; col += kThreads * kCols)
                use(col);
        };
        RowStats st = {};
        if (a.post == kNormLayer) {
            float s = 0.0f;
            over([&](int col) {
                const Raw<T> v = row_block(f, col, a.cols);
#pragma unroll
                for (int i = 0; i < kCols; ++i)
                    s += (float)v[i];
            });
            st.post.mean = sum(s) / cols;
        }
        if (a.post != kNormNone) {
            float s = 0.0f;
            over([&](int col) {
                const Raw<T> v = row_block(f, col, a.cols);
#pragma unroll
                for (int i = 0; i < kCols; ++i) {
                    const float d = (float)v[i] - st.post.mean;
                    s += col + i < a.cols ? d * d : 0.0f;
                }
            });
            st.post.r = inverse_size(sum(s), a.cols, a.post_eps);
        }
        Gradient<T, S> p;
        float w[kCols], b[kCols];
        auto forward = [&](int col) {
            vector_block(a.post_weight, col, a.cols, 1.0f, w);
            vector_block(a.post_bias, col, a.cols, 0.0f, b);
            p(a, row_block(f, col, a.cols), a.gate ? row_block(u, col, a.cols) : Raw<T>{},
              a.x ? row_block(x, col, a.cols) : Raw<S>{}, st.post, w, b);
        };
        if (a.pre == kNormLayer) {
            float s = 0.0f;
            over([&](int col) {
                forward(col);
#pragma unroll
                for (int i = 0; i < kCols; ++i)
                    s += col + i < a.cols ? p.y[i] : 0.0f;
            });
            st.pre.mean = sum(s) / cols;
        }
        if (a.pre != kNormNone) {
            float s = 0.0f;
            over([&](int col) {
                forward(col);
#pragma unroll
                for (int i = 0; i < kCols; ++i) {
                    const float d = p.y[i] - st.pre.mean;
                    s += col + i < a.cols ? d * d : 0.0f;
                }
            });
            st.pre.r = inverse_size(sum(s), a.cols, a.pre_eps);
        }
        auto pre = [&](int col) {
            forward(col);
            if (ga.dh) {
                float q[kCols];
                vector_block(a.pre_weight, col, a.cols, 1.0f, q);
                p.of_pre(row_block(dh, col, a.cols), q, st.pre);
            }
        };
        if (a.pre != kNormNone) {
            float s[2] = {};
            over([&](int col) {
                pre(col);                         // dh, and with it t, is 0 behind the row's end
#pragma unroll
                for (int i = 0; i < kCols; ++i) {
                    s[0] += p.t[i];
                    s[1] += p.t[i] * (col + i < a.cols ? p.yn[i] : 0.0f);
                }
            });
            sum(s);
            st.t = a.pre == kNormLayer ? s[0] / cols : 0.0f;
            st.t_yn = s[1] / cols;
        }
        if (a.post != kNormNone) {
            float s[2] = {};
            over([&](int col) {
                pre(col);
                p.of_sum(ga, ga.dy ? row_block(dy, col, a.cols) : Raw<S>{}, st);
                p.of_post(ga, w);
#pragma unroll
                for (int i = 0; i < kCols; ++i) {
                    s[0] += col + i < a.cols ? p.v[i] : 0.0f;
                    s[1] += col + i < a.cols ? p.v[i] * p.fn[i] : 0.0f;
                }
            });
            sum(s);
            st.v = a.post == kNormLayer ? s[0] / cols : 0.0f;
            st.v_fn = s[1] / cols;
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
    float w[kCols], b[kCols], q[kCols], sums[kSums][kCols] = {};
    vector_block(a.post_weight, col, a.cols, 1.0f, w);
    vector_block(a.post_bias, col, a.cols, 0.0f, b);
    vector_block(a.pre_weight, col, a.cols, 1.0f, q);
    for (int64_t row = first; row < end; ++row) {
        const RowStats st = stats[row];
        Gradient<T, S> p;
        p(a, row_block(row_of<T>(a.f, a.f_stride, row), col, a.cols),
          a.gate ? row_block(row_of<T>(a.gate, a.gate_stride, row), col, a.cols) : Raw<T>{},
          a.x ? row_block(row_of<S>(a.x, a.x_stride, row), col, a.cols) : Raw<S>{}, st.post, w, b);
        Raw<T> dh{};
        if (ga.dh) {
            dh = row_block(row_of<T>(ga.dh, ga.dh_stride, row), col, a.cols);
            p.of_pre(dh, q, st.pre);
        }
        p.of_sum(ga, ga.dy ? row_block(row_of<S>(ga.dy, ga.dy_stride, row), col, a.cols) : Raw<S>{},
                 st);
        p.of_post(ga, w);
        float df[kCols], du[kCols];
#pragma unroll
        for (int i = 0; i < kCols; ++i) {
            const float d = p.dy[i] * a.scale;
            df[i] = a.post == kNormNone ? p.v[i]
                                        : st.post.r * (p.v[i] - st.v - p.fn[i] * st.v_fn);
            du[i] = d * p.n[i] * p.slope[i];
            sums[kPostWeight][i] += d * p.g[i] * p.fn[i];
            sums[kPostBias][i] += d * p.g[i];
            if (ga.dh) {
                sums[kPreWeight][i] += (float)dh[i] * p.yn[i];
                sums[kPreBias][i] += (float)dh[i];
            }
        }
        if (ga.dx)
            put_block(row_of<S>(ga.dx, ga.dx_stride, row), col, a.cols, p.dy);
        if (ga.dgate)
            put_block(row_of<T>(ga.dgate, ga.dgate_stride, row), col, a.cols, du);
        put_block(row_of<T>(ga.df, ga.df_stride, row), col, a.cols, df);
    }
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
#pragma unroll 8
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

template <typename T, typename S, int L>
hipError_t launch_rows(const NormGradArgs &g, hipStream_t stream) {
    const NormArgs &a = g.a;
    constexpr int kT = L < kThreads ? kThreads : L;
    const int64_t padded = padded_cols(a.cols), groups = norm_grad_groups(a.n, a.cols);
    float *partial = static_cast<float *>(g.workspace);
    auto even = [](const void *p, int64_t stride) { return !p || even_rows(p, stride); };
    const bool tail = !(a.cols % kCols == 0 && even(a.f, a.f_stride) && even(a.x, a.x_stride) &&
                        even(a.gate, a.gate_stride) && even(g.dy, g.dy_stride) &&
                        even(g.dh, g.dh_stride) && even(g.dx, g.dx_stride) &&
                        even(g.df, g.df_stride) && even(g.dgate, g.dgate_stride));
    const bool bias = a.post_bias || g.sums[kPostBias] || g.sums[kPreBias];
    const unsigned grid = (unsigned)groups;
    if (tail && bias)
        row_grad_kernel<T, S, L, true, true><<<grid, kT, 0, stream>>>(g, partial, padded);
    else if (tail)
        row_grad_kernel<T, S, L, true, false><<<grid, kT, 0, stream>>>(g, partial, padded);
    else if (bias)
        row_grad_kernel<T, S, L, false, true><<<grid, kT, 0, stream>>>(g, partial, padded);
    else
        row_grad_kernel<T, S, L, false, false><<<grid, kT, 0, stream>>>(g, partial, padded);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? fold(g, partial, groups, stream) : e;
}

template <typename T, typename S>
hipError_t launch_types(const NormGradArgs &g, hipStream_t stream) {
    switch (norm_grad_lanes(g.a.cols)) {
    case 16: return launch_rows<T, S, 16>(g, stream);
    case 64: return launch_rows<T, S, 64>(g, stream);
    case 256: return launch_rows<T, S, 256>(g, stream);
    case 512: return launch_rows<T, S, 512>(g, stream);
    case 1024: return launch_rows<T, S, 1024>(g, stream);
    }
    const int64_t padded = padded_cols(g.a.cols), strips = norm_wide_strips(g.a.n, g.a.cols);
    RowStats *stats = static_cast<RowStats *>(g.workspace);
    float *partial = reinterpret_cast<float *>(stats + g.a.n);
    const int64_t most = 1 << 20;
    wide_stats_kernel<T, S><<<(unsigned)(g.a.n < most ? g.a.n : most), kThreads, 0, stream>>>(g, stats);
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
    if (norm_grad_lanes(cols))
        return norm_grad_groups(n, cols) * kSums * padded_cols(cols) * 4;
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

// Norms after and before a block, with its gate and residual sum: rows in, rows out.
//
// Bound by memory where rows are many: 65,536 x 4,096 with x and y in 32 bits, the rest bf16, 656 us (3.76 GB
// at 5.7 TB/s), all bf16 484 to 501 (2.68 GB); 50,000 x 512 f16, a layer norm alone, 24 (a third of the time
// is what a row's two sums wait for); 64 x 4,096 3.7, the launch. In pieces through the caches the first took 887.
#include "norm_choice.h"
#include "norm_device.h"

namespace ccj {
namespace {

constexpr int kThreads = 256;
constexpr int kWide = 1024;                        // of rows of any length

// Rows that stay in registers: the lanes of a row, L or beyond 64 all of a workgroup of at most L, hold B
// blocks of 8 columns each, and weights and biases of their columns for all the rows that they go through.
// One read of f, gate and x, one write of y and h; the sums between them are over lanes, and over a
// workgroup's wavefronts through LDS. BIAS: with either bias.
// Beyond 8,192 columns a lane has 128 registers, enough for elements and stream in 16 bits (16,384 x 16,384
// 507 us, 5.3 TB/s); with a stream in 32 bits 6 of them are spilled to scratch (742, 5.1), with biases too 40
// (1,106, 3.4), in 32 bits throughout 38 and 132 (1,478 and 1,615, 3.6 and 3.3).
template <typename T, typename S, int L, int B, bool TAIL, bool BIAS>
__global__ __launch_bounds__(L <= 64 ? kThreads : L) void row_norm_kernel(NormArgs a) {
    constexpr int kGroups = L <= 64 ? kThreads / L : 1;
    __shared__ float place[2][2][L > 64 ? L / 64 : 1];
    RowSum<L, (L > 64)> sum(place);
    const int lane = L > 64 ? threadIdx.x : threadIdx.x % L, lanes = L > 64 ? blockDim.x : L;
    const float per = 1.0f / (float)a.cols;
    int col[B], exchange[B];
    float post_w[B][kCols], post_b[B][kCols] = {}, pre_w[B][kCols], pre_b[B][kCols] = {};
#pragma unroll
    for (int i = 0; i < B; ++i) {
        col[i] = (lane + i * lanes) * kCols;
        exchange[i] = exchange_of(lane + i * lanes, a.cols);
        vector_block(a.post_weight, col[i], a.cols, 1.0f, post_w[i]);
        vector_block(a.pre_weight, col[i], a.cols, 1.0f, pre_w[i]);
        if (BIAS) {
            vector_block(a.post_bias, col[i], a.cols, 0.0f, post_b[i]);
            vector_block(a.pre_bias, col[i], a.cols, 0.0f, pre_b[i]);
        }
        times(post_w[i], a.scale);
        times(post_b[i], a.scale);
    }
    for (int64_t row = (int64_t)blockIdx.x * kGroups + group_of_lanes<L>(); row < a.n;
         row += (int64_t)gridDim.x * kGroups) {
        Raw<T> f[B], u[B];
        Raw<S> x[B];
#pragma unroll
        for (int i = 0; i < B; ++i) {
            f[i] = held_block<TAIL>(row_of<T>(a.f, a.f_stride, row), col[i], a.cols, exchange[i]);
            u[i] = Raw<T>{};
            x[i] = Raw<S>{};
            if (a.gate)
                u[i] = held_block<TAIL>(row_of<T>(a.gate, a.gate_stride, row), col[i], a.cols,
                                        exchange[i]);
            if (a.x)
                x[i] = held_block<TAIL>(row_of<S>(a.x, a.x_stride, row), col[i], a.cols, exchange[i]);
        }
#pragma unroll
        for (int i = 0; i < B; ++i)
            settle(f[i], exchange[i]);
        float v[B][kCols], y[B][kCols];
#pragma unroll
        for (int i = 0; i < B; ++i)
            numbers(f[i], v[i]);
        const RowNorm post = norm_of<TAIL>(a.post, v, col, a.cols, per, a.post_eps, sum);
#pragma unroll
        for (int i = 0; i < B; ++i) {
            settle(u[i], exchange[i]);
            settle(x[i], exchange[i]);
            float g[kCols], unused[kCols], gate[kCols], stream[kCols];
            numbers(u[i], gate);
            numbers(x[i], stream);
            gate_block<false>(a.gate_kind, gate, g, unused);
            normalised(a.post, v[i], post, v[i]);
            block_sum(stream, g, v[i], post_w[i], post_b[i], y[i]);
            put_held<TAIL>(row_of<S>(a.y, a.y_stride, row), col[i], a.cols, exchange[i], y[i]);
        }
        if (!a.h)
            continue;
        const RowNorm pre = norm_of<TAIL>(a.pre, y, col, a.cols, per, a.pre_eps, sum);
#pragma unroll
        for (int i = 0; i < B; ++i) {
            float h[kCols];
            normalised(a.pre, y[i], pre, h);
#pragma unroll
            for (int e = 0; e < kCols; ++e)
                h[e] = h[e] * pre_w[i][e] + pre_b[i][e];
            put_held<TAIL>(row_of<T>(a.h, a.h_stride, row), col[i], a.cols, exchange[i], h);
        }
    }
}

// Rows of any length, a workgroup each, in pieces of 2,048 columns: a pass over f for each sum of its
// norm, a pass over x, f and the gate for each sum of y's, and one that writes. All but the first pass
// find the row in the caches.
template <typename T, typename S>
__global__ __launch_bounds__(kWide) void wide_norm_kernel(NormArgs a) {
    __shared__ float place[2][2][kWide / 64];
    RowSum<kWide> sum(place);
    const float per = 1.0f / (float)a.cols;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const T *f = row_of<T>(a.f, a.f_stride, row), *u = row_of<T>(a.gate, a.gate_stride, row);
        const S *x = row_of<S>(a.x, a.x_stride, row);
        // The sum over the row of use(col).
        auto over = [&](auto &&use) {
            float s = 0.0f;
            for (int col = threadIdx.x * kCols; col < a.cols; col += kWide * kCols)
                s += use(col);
            return sum(s);
        };
        auto block_f = [&](int col, float(&v)[kCols]) { numbers(row_block(f, col, a.cols), v); };
        RowNorm post, pre;
        if (a.post == kNormLayer)
            post.mean = over([&](int col) {
                            float v[kCols];
                            block_f(col, v);
                            return plain_sum(v);
                        }) * per;
        if (a.post != kNormNone)
            post.r = inverse_size(over([&](int col) {
                                      float v[kCols];
                                      block_f(col, v);
                                      return squares<true>(v, post.mean, col, a.cols);
                                  }) * per,
                                  a.post_eps);
        float y[kCols];
        auto forward = [&](int col) {
            float w[kCols], b[kCols], v[kCols], g[kCols], unused[kCols], gate[kCols], stream[kCols];
            vector_block(a.post_weight, col, a.cols, 1.0f, w);
            vector_block(a.post_bias, col, a.cols, 0.0f, b);
            times(w, a.scale);
            times(b, a.scale);
            block_f(col, v);
            numbers(a.gate ? row_block(u, col, a.cols) : Raw<T>{}, gate);
            numbers(a.x ? row_block(x, col, a.cols) : Raw<S>{}, stream);
            gate_block<false>(a.gate_kind, gate, g, unused);
            normalised(a.post, v, post, v);
            block_sum(stream, g, v, w, b, y);
        };
        if (a.pre == kNormLayer)
            pre.mean = over([&](int col) {
                           forward(col);          // 0 where the row has no column
                           return plain_sum(y);
                       }) * per;
        if (a.pre != kNormNone)
            pre.r = inverse_size(over([&](int col) {
                                     forward(col);
                                     return squares<true>(y, pre.mean, col, a.cols);
                                 }) * per,
                                 a.pre_eps);
        over([&](int col) {
            forward(col);
            put_block(row_of<S>(a.y, a.y_stride, row), col, a.cols, y);
            if (a.h) {
                float w[kCols], b[kCols], h[kCols];
                vector_block(a.pre_weight, col, a.cols, 1.0f, w);
                vector_block(a.pre_bias, col, a.cols, 0.0f, b);
                normalised(a.pre, y, pre, h);
#pragma unroll
                for (int i = 0; i < kCols; ++i)
                    h[i] = h[i] * w[i] + b[i];
                put_block(row_of<T>(a.h, a.h_stride, row), col, a.cols, h);
            }
            return 0.0f;
        });
    }
}

template <typename T, typename S, int L, int B>
hipError_t launch_rows(const NormArgs &a, int lanes, hipStream_t stream) {
    const int threads = L <= 64 ? kThreads : lanes, rows = L <= 64 ? kThreads / L : 1;
    const unsigned grid = (unsigned)norm_groups((a.n + rows - 1) / rows, threads);
    const bool bias = a.post_bias || a.pre_bias;
    const bool even = a.cols % kCols == 0 && even_rows(a.f, a.f_stride) && even_rows(a.y, a.y_stride) &&
                      (!a.x || even_rows(a.x, a.x_stride)) && (!a.h || even_rows(a.h, a.h_stride)) &&
                      (!a.gate || even_rows(a.gate, a.gate_stride));
    if (even && bias)
        row_norm_kernel<T, S, L, B, false, true><<<grid, threads, 0, stream>>>(a);
    else if (even)
        row_norm_kernel<T, S, L, B, false, false><<<grid, threads, 0, stream>>>(a);
    else
        row_norm_kernel<T, S, L, B, true, true><<<grid, threads, 0, stream>>>(a);
    return hipGetLastError();
}

template <typename T, typename S>
hipError_t launch_types(const NormArgs &a, hipStream_t stream) {
    const NormShape s = norm_shape(a.cols);
    if (s.blocks == 1)
        return s.lanes == 16   ? launch_rows<T, S, 16, 1>(a, s.lanes, stream)
               : s.lanes == 32 ? launch_rows<T, S, 32, 1>(a, s.lanes, stream)
               : s.lanes == 64 ? launch_rows<T, S, 64, 1>(a, s.lanes, stream)
                               : launch_rows<T, S, 256, 1>(a, s.lanes, stream);
    if (s.blocks == 2)
        return s.lanes == 64    ? launch_rows<T, S, 64, 2>(a, s.lanes, stream)
               : s.lanes <= 256 ? launch_rows<T, S, 256, 2>(a, s.lanes, stream)
               : s.lanes <= 512 ? launch_rows<T, S, 512, 2>(a, s.lanes, stream)
                                : launch_rows<T, S, 1024, 2>(a, s.lanes, stream);
    const int64_t most = 1 << 20;
    wide_norm_kernel<T, S><<<(unsigned)(a.n < most ? a.n : most), kWide, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_norm(const NormArgs &a, hipStream_t stream) {
    switch (a.type) {
    case kF32: return launch_types<float, float>(a, stream);
    case kF16:
        return a.stream_type == kF32 ? launch_types<half_t, float>(a, stream)
                                     : launch_types<half_t, half_t>(a, stream);
    default:
        return a.stream_type == kF32 ? launch_types<bf16_t, float>(a, stream)
                                     : launch_types<bf16_t, bf16_t>(a, stream);
    }
}

}  // namespace ccj

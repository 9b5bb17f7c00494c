// Norms after and before a block, with its gate and residual sum: rows in, rows out.
#include "norm_device.h"

namespace ccj {
namespace {

constexpr int kThreads = 256;

// Rows of any length, a workgroup each, in pieces of 2,048 columns: a pass over f for each sum of its
// norm, a pass over x, f and the gate for each sum of y's, and one that writes. All but the first pass
// find the row in the caches.
template <typename T, typename S>
__global__ __launch_bounds__(kThreads) void wide_norm_kernel(NormArgs a) {
    __shared__ float place[2][kThreads / 64][1];
    RowSum<kThreads, 1> sum{place};
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const T *f = row_of<T>(a.f, a.f_stride, row), *u = row_of<T>(a.gate, a.gate_stride, row);
        const S *x = row_of<S>(a.x, a.x_stride, row);
        auto over = [&](auto &&use) {
            for (int col = threadIdx.x * kCols; col < a.cols; col += kThreads * kCols)
                use(col);
        };
        RowNorm post, pre;
        if (a.post == kNormLayer) {
            float s = 0.0f;
            over([&](int col) {
                const Raw<T> v = row_block(f, col, a.cols);
#pragma unroll
                for (int i = 0; i < kCols; ++i)
                    s += (float)v[i];
            });
            post.mean = sum(s) / (float)a.cols;
        }
        if (a.post != kNormNone) {
            float s = 0.0f;
            over([&](int col) {
                const Raw<T> v = row_block(f, col, a.cols);
#pragma unroll
                for (int i = 0; i < kCols; ++i) {
                    const float d = (float)v[i] - post.mean;
                    s += col + i < a.cols ? d * d : 0.0f;
                }
            });
            post.r = inverse_size(sum(s), a.cols, a.post_eps);
        }
        Forward<T, S> p;
        auto forward = [&](int col) {
            float w[kCols], b[kCols];
            vector_block(a.post_weight, col, a.cols, 1.0f, w);
            vector_block(a.post_bias, col, a.cols, 0.0f, b);
            p(a, row_block(f, col, a.cols), a.gate ? row_block(u, col, a.cols) : Raw<T>{},
              a.x ? row_block(x, col, a.cols) : Raw<S>{}, post, w, b);
        };
        if (a.pre == kNormLayer) {
            float s = 0.0f;
            over([&](int col) {
                forward(col);
#pragma unroll
                for (int i = 0; i < kCols; ++i)
                    s += col + i < a.cols ? p.y[i] : 0.0f;
            });
            pre.mean = sum(s) / (float)a.cols;
        }
        if (a.pre != kNormNone) {
            float s = 0.0f;
            over([&](int col) {
                forward(col);
#pragma unroll
                for (int i = 0; i < kCols; ++i) {
                    const float d = p.y[i] - pre.mean;
                    s += col + i < a.cols ? d * d : 0.0f;
                }
            });
            pre.r = inverse_size(sum(s), a.cols, a.pre_eps);
        }
        over([&](int col) {
            forward(col);
            put_block(row_of<S>(a.y, a.y_stride, row), col, a.cols, p.y);
            if (a.h) {
                float w[kCols], b[kCols], h[kCols];
                vector_block(a.pre_weight, col, a.cols, 1.0f, w);
                vector_block(a.pre_bias, col, a.cols, 0.0f, b);
#pragma unroll
                for (int i = 0; i < kCols; ++i)
                    h[i] = (p.y[i] - pre.mean) * pre.r * w[i] + b[i];
                put_block(row_of<T>(a.h, a.h_stride, row), col, a.cols, h);
            }
        });
    }
}

template <typename T, typename S>
hipError_t launch_types(const NormArgs &a, hipStream_t stream) {
    const int64_t most = 1 << 20;
    wide_norm_kernel<T, S><<<(unsigned)(a.n < most ? a.n : most), kThreads, 0, stream>>>(a);
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

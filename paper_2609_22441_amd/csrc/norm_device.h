// Device helpers of the block norms: sums over the lanes of a row, and the elementwise parts of the
// norms, the gate and their gradients, on blocks of 8 columns.
#pragma once

#include "layers_device.h"

namespace ccj {
namespace {

// ---- sums over a row's lanes ----

template <int CONTROL>
__device__ __forceinline__ float plus_lanes(float x) {
    return x + __uint_as_float((uint32_t)__builtin_amdgcn_mov_dpp((int)__float_as_uint(x), CONTROL,
                                                                  0xf, 0xf, true));
}

// The sum over LANES = 16 or 64 consecutive lanes, in each of them, in the same order for all.
template <int LANES>
__device__ __forceinline__ float lanes_sum(float x) {
    constexpr int kHalfMirror = 0x141, kMirror = 0x140;
    x = plus_lanes<quad_perm(1, 0, 3, 2)>(x);
    x = plus_lanes<quad_perm(2, 3, 0, 1)>(x);
    x = plus_lanes<kHalfMirror>(x);               // lane 7 - i of each 8
    x = plus_lanes<kMirror>(x);                   // lane 15 - i of each 16
    if (LANES == 64) {
        x += __shfl_xor(x, 16);
        x += __shfl_xor(x, 32);
    }
    return x;
}

// Sums of N numbers over the L lanes of a row; of more than a wavefront through LDS, whose two places
// take turns: a wavefront that writes to one again has passed a barrier that all reached after they
// had read it.
template <int L, int N>
struct RowSum {
    static constexpr int kWaves = L > 64 ? L / 64 : 1;
    float (*place)[kWaves][N];
    int turn = 0;
    __device__ __forceinline__ void operator()(float (&x)[N]) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            x[i] = lanes_sum<(L < 64 ? L : 64)>(x[i]);
        if constexpr (L > 64) {
            if ((threadIdx.x & 63) == 0)
#pragma unroll
                for (int i = 0; i < N; ++i)
                    place[turn][threadIdx.x >> 6][i] = x[i];
            __syncthreads();
#pragma unroll
            for (int i = 0; i < N; ++i) {
                x[i] = 0.0f;
#pragma unroll
                for (int w = 0; w < kWaves; ++w)
                    x[i] += place[turn][w][i];
            }
            turn ^= 1;
        }
    }
    __device__ __forceinline__ float operator()(float a) {
        float x[N] = {a};
        (*this)(x);
        return x[0];
    }
};

// ---- blocks of 8 columns ----

// Block at `col` of a vector of `cols` floats, `other` without a vector, 0 behind the end.
__device__ __forceinline__ void vector_block(const float *v, int col, int cols, float other,
                                             float (&x)[kCols]) {
    if (v && col + kCols <= cols) {
        const Raw<float> r = load_block(v + col);
#pragma unroll
        for (int i = 0; i < kCols; ++i)
            x[i] = r[i];
    } else {
#pragma unroll
        for (int i = 0; i < kCols; ++i)
            x[i] = col + i >= cols ? 0.0f : v ? v[col + i] : other;
    }
}

// A block of a row that its lanes hold: where lanes exchange pieces of 32-bit elements, settle() puts
// them in place. TAIL: rows have a last block of fewer columns, or are not aligned to 16 bytes.
template <bool TAIL, typename T>
__device__ __forceinline__ Raw<T> held_block(const T *row, int col, int cols, int exchange) {
    if (col + kCols <= cols)
        return load_pieces<!TAIL>(row + col, exchange);
    return TAIL && col < cols ? load_block(row + col, cols - col) : Raw<T>{};
}

// Block at `col` of a row, zeros behind its end.
template <typename T>
__device__ __forceinline__ Raw<T> row_block(const T *p, int col, int cols) {
    return col + kCols <= cols ? load_block(p + col) : load_block(p + col, cols - col);
}

template <typename T>
__device__ __forceinline__ void put_block(T *p, int col, int cols, const float (&x)[kCols]) {
    if (col + kCols <= cols)
        store_block(p + col, x);
    else
        store_block(p + col, x, cols - col);
}

template <bool TAIL, typename T>
__device__ __forceinline__ void put_held(T *row, int col, int cols, int exchange,
                                         const float (&x)[kCols]) {
    if (!TAIL && col < cols)
        stream_block(row + col, x, exchange);
    else if (TAIL && col < cols)
        put_block(row, col, cols, x);
}

// A row's norm: (v - mean) * r.
struct RowNorm {
    float mean = 0.0f, r = 1.0f;
};

// 1 / sqrt(sum / cols + eps), once per row: correctly rounded root and quotient.
__device__ __forceinline__ float inverse_size(float sum, int cols, float eps) {
    return 1.0f / sqrtf(sum / (float)cols + eps);
}

// The gate and its derivative. exp of a magnitude's negative does not overflow, and 1 - g of a sigmoid
// near 1 is e / (1 + e), without cancellation. The reciprocal is within one unit in the last place
// (a division's ten instructions for each element would be a sixth of what a row's bytes leave time
// for).
template <typename T>
__device__ __forceinline__ void gate_block(int kind, const Raw<T> &u, float (&g)[kCols],
                                           float (&slope)[kCols]) {
#pragma unroll
    for (int i = 0; i < kCols; ++i) {
        const float v = (float)u[i];
        if (kind == kGateSigmoid) {
            const float e = __expf(-fabsf(v)), r = __builtin_amdgcn_rcpf(1.0f + e);
            g[i] = v < 0.0f ? e * r : r;
            slope[i] = e * r * r;
        } else {
            g[i] = kind == kGateLinear ? v : 1.0f;
            slope[i] = 1.0f;
        }
    }
}

template <typename T>
__device__ __forceinline__ const T *row_of(const void *p, int64_t stride, int64_t row) {
    return (const T *)((const char *)p + row * stride);
}

template <typename T>
__device__ __forceinline__ T *row_of(void *p, int64_t stride, int64_t row) {
    return (T *)((char *)p + row * stride);
}

// y of a block, and f normalised, from their parts.
template <typename T, typename S>
struct Forward {
    float fn[kCols], n[kCols], g[kCols], slope[kCols], y[kCols];
    __device__ __forceinline__ void operator()(const NormArgs &a, const Raw<T> &f, const Raw<T> &u,
                                               const Raw<S> &x, const RowNorm &post,
                                               const float (&w)[kCols], const float (&b)[kCols]) {
        gate_block(a.gate_kind, u, g, slope);
#pragma unroll
        for (int i = 0; i < kCols; ++i) {
            fn[i] = ((float)f[i] - post.mean) * post.r;
            n[i] = fn[i] * w[i] + b[i];
            y[i] = (float)x[i] + a.scale * g[i] * n[i];
        }
    }
};

}  // namespace
}  // namespace ccj

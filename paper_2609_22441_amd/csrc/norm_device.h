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

constexpr int kHalfMirror = 0x141, kMirror = 0x140;       // lane 7 - i of each 8, 15 - i of each 16

// The sum over LANES consecutive lanes, a power of two up to 64, in each of them: a tree whose additions
// are the same for all.
template <int LANES>
__device__ __forceinline__ float lanes_sum(float x) {
    if (LANES >= 2)
        x = plus_lanes<quad_perm(1, 0, 3, 2)>(x);
    if (LANES >= 4)
        x = plus_lanes<quad_perm(2, 3, 0, 1)>(x);
    if (LANES >= 8)
        x = plus_lanes<kHalfMirror>(x);
    if (LANES >= 16)
        x = plus_lanes<kMirror>(x);
    // Of two copies, exchanging the odd 16 lanes (the upper 32) of one with the even (lower) ones of the
    // other leaves both summands in every lane.
    if (LANES >= 32) {
        const auto y = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                        false);
        x = __uint_as_float(y[0]) + __uint_as_float(y[1]);
    }
    if (LANES >= 64) {
        const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                        false);
        x = __uint_as_float(y[0]) + __uint_as_float(y[1]);
    }
    return x;
}

// Sums of up to 2 numbers over the L lanes of a row, in each of them; of more than a wavefront, which are
// the workgroup's and with FEWER possibly not all L, through LDS, whose two places take turns: a wavefront
// that writes to one again has passed a barrier that all reached after they had read it. The places of
// wavefronts that the workgroup does not have are 0.
template <int L, bool FEWER = false>
struct RowSum {
    static constexpr int kWaves = L > 64 ? L / 64 : 1;
    float (*place)[2][kWaves];
    int turn = 0;
    __device__ __forceinline__ explicit RowSum(float (&p)[2][2][kWaves]) : place(p) {
        if constexpr (L > 64 && FEWER) {
            if (threadIdx.x < 4 * kWaves)
                (&p[0][0][0])[threadIdx.x] = 0.0f;
            __syncthreads();
        }
    }
    template <int N>
    __device__ __forceinline__ void operator()(float (&x)[N]) {
        static_assert(N <= 2, "");
#pragma unroll
        for (int i = 0; i < N; ++i)
            x[i] = lanes_sum<(L < 64 ? L : 64)>(x[i]);
        if constexpr (L > 64) {
            if ((threadIdx.x & 63) == 0)
#pragma unroll
                for (int i = 0; i < N; ++i)
                    place[turn][i][threadIdx.x >> 6] = x[i];
            __syncthreads();
#pragma unroll
            for (int i = 0; i < N; ++i)
                x[i] = lanes_sum<kWaves>(place[turn][i][threadIdx.x % kWaves]);
            turn ^= 1;
        }
    }
    __device__ __forceinline__ float operator()(float a) {
        float x[1] = {a};
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
// them in place. TAIL: rows have a last block of fewer columns, or are not aligned to 16 bytes; the elements
// of such a block are asked for after what was asked for before is here, once a matrix (50,000 x 1,001 bf16
// 123 us and its gradient 243, x 1,000 98 and 165; in 999 x 97 of 32 bits 1.4 of the gradient's 8.8).
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

// 1 / sqrt(mean + eps), within one unit in the last place: every lane computes it, and a correctly rounded
// root and quotient are 25 instructions.
__device__ __forceinline__ float inverse_size(float mean, float eps) {
    return __builtin_amdgcn_rsqf(mean + eps);
}

// A gate and its derivative, for a block. exp of a magnitude's negative does not overflow, and 1 - g of a
// sigmoid near 1 is e / (1 + e), without cancellation. The reciprocal is within one unit in the last place
// (a division's ten instructions for each element would be a sixth of what a row's bytes leave time
// for). The kind is asked for once, not for each element.
template <bool SLOPE>
__device__ __forceinline__ void gate_block(int kind, const float (&u)[kCols], float (&g)[kCols],
                                           float (&slope)[kCols]) {
    if (kind == kGateSigmoid) {
#pragma unroll
        for (int i = 0; i < kCols; ++i) {
            const float e = __expf(-fabsf(u[i])), r = __builtin_amdgcn_rcpf(1.0f + e), er = e * r;
            g[i] = u[i] < 0.0f ? er : r;
            if (SLOPE)
                slope[i] = er * r;
        }
    } else {
#pragma unroll
        for (int i = 0; i < kCols; ++i) {
            g[i] = kind == kGateLinear ? u[i] : 1.0f;
            if (SLOPE)
                slope[i] = 1.0f;
        }
    }
}

template <typename T>
__device__ __forceinline__ void numbers(const Raw<T> &x, float (&v)[kCols]) {
#pragma unroll
    for (int i = 0; i < kCols; ++i)
        v[i] = (float)x[i];
}

// What is computed from x on is computed from it again: the compiler would keep the results of the first
// time in registers, of which rows on their way need more.
__device__ __forceinline__ void again(float &x) { asm volatile("" : "+v"(x)); }

template <typename T>
__device__ __forceinline__ void again(Raw<T> &x) {
#pragma unroll
    for (int i = 0; i < Raw<T>::kWords; ++i)
        asm volatile("" : "+v"(x.w[i]));
}

template <typename T>
__device__ __forceinline__ const T *row_of(const void *p, int64_t stride, int64_t row) {
    return (const T *)((const char *)p + row * stride);
}

template <typename T>
__device__ __forceinline__ T *row_of(void *p, int64_t stride, int64_t row) {
    return (T *)((char *)p + row * stride);
}

// y of a block from f normalised; weight and bias times scale.
__device__ __forceinline__ void block_sum(const float (&x)[kCols], const float (&g)[kCols],
                                          const float (&fn)[kCols], const float (&w)[kCols],
                                          const float (&b)[kCols], float (&y)[kCols]) {
#pragma unroll
    for (int i = 0; i < kCols; ++i)
        y[i] = x[i] + g[i] * (fn[i] * w[i] + b[i]);
}

__device__ __forceinline__ void times(float (&v)[kCols], float scale) {
#pragma unroll
    for (int i = 0; i < kCols; ++i)
        v[i] *= scale;
}

// A block normalised: (v - mean) * r, the mean being 0 but in a layer norm.
__device__ __forceinline__ void normalised(int kind, const float (&v)[kCols], const RowNorm &n,
                                           float (&vn)[kCols]) {
    if (kind == kNormLayer) {
#pragma unroll
        for (int i = 0; i < kCols; ++i)
            vn[i] = (v[i] - n.mean) * n.r;
    } else {
#pragma unroll
        for (int i = 0; i < kCols; ++i)
            vn[i] = v[i] * n.r;
    }
}

// The sum of (v - mean)^2 over the columns that a row has of a block at `col`. TAIL: a block may have
// some of its columns.
template <bool TAIL>
__device__ __forceinline__ float squares(const float (&v)[kCols], float mean, int col, int cols) {
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < kCols; ++i) {
        const float d = v[i] - mean;
        s += !TAIL || col + i < cols ? d * d : 0.0f;
    }
    return TAIL || col < cols ? s : 0.0f;
}

__device__ __forceinline__ float plain_sum(const float (&v)[kCols]) {
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < kCols; ++i)
        s += v[i];
    return s;
}

// The norm of a row whose lanes hold B blocks: v is 0 where the row has no column. per: 1 / columns.
template <bool TAIL, int B, typename Sum>
__device__ __forceinline__ RowNorm norm_of(int kind, const float (&v)[B][kCols], const int (&col)[B],
                                           int cols, float per, float eps, Sum &sum) {
    RowNorm n;
    float s = 0.0f;
    if (kind == kNormLayer) {
#pragma unroll
        for (int i = 0; i < B; ++i)
            s += plain_sum(v[i]);
        n.mean = sum(s) * per;
        s = 0.0f;
#pragma unroll
        for (int i = 0; i < B; ++i)
            s += squares<TAIL>(v[i], n.mean, col[i], cols);
    } else if (kind == kNormRms) {
#pragma unroll
        for (int i = 0; i < B; ++i)
#pragma unroll
            for (int e = 0; e < kCols; ++e)
                s += v[i][e] * v[i][e];
    }
    if (kind != kNormNone)
        n.r = inverse_size(sum(s) * per, eps);
    return n;
}

// Which of a workgroup's rows a thread works on, as a scalar where all lanes of its wavefront do.
template <int L>
__device__ __forceinline__ int group_of_lanes() {
    const int group = threadIdx.x / L;
    return L >= 64 ? __builtin_amdgcn_readfirstlane(group) : group;
}

}  // namespace
}  // namespace ccj

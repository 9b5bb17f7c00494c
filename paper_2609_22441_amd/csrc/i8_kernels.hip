// 8-bit integers with a scale per row: quantisation of rows, and the product of two such matrices.
#include "layers_device.h"

namespace ccj {
namespace {

typedef int int4_t __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;

// ---- quantisation ----

// A row's largest magnitude, as the bits of a non-negative float: their order as integers is that of
// the values, infinities and NaN above all numbers.
constexpr uint32_t kInfinity = 0x7f800000u;

struct RowScale {
    float inverse;       // 127 / most, of a row scaled by `raise`
    float raise;         // 2^64 for rows so small that 127 / most would overflow, else 1
    float scale;         // most / 127, or NaN
};

__device__ __forceinline__ RowScale row_scale(uint32_t most_bits) {
    const float most = __uint_as_float(most_bits);
    RowScale s;
    s.raise = most < 0x1p-60f ? 0x1p64f : 1.0f;
    s.inverse = most_bits == 0 || most_bits >= kInfinity ? 0.0f : 127.0f / (most * s.raise);
    s.scale = most_bits >= kInfinity ? __uint_as_float(0x7fc00000u) : most / 127.0f;
    return s;
}

// Eight values to 8 bits. A row with a NaN or an infinity has the factor 0 and gets zeros.
__device__ __forceinline__ uint64_t eight_bits(const float (&x)[kCols], const RowScale &s) {
    uint64_t q = 0;
#pragma unroll
    for (int i = 0; i < kCols; ++i) {
        const int v = s.inverse == 0.0f ? 0 : (int)rintf(x[i] * s.raise * s.inverse);
        q |= (uint64_t)(uint8_t)v << (8 * i);
    }
    return q;
}

// A group of L lanes per row (L = 16, 64 or the workgroup).
template <typename T, int L>
__global__ __launch_bounds__(kThreads) void quantize_kernel(QuantizeArgs a) {
    __shared__ uint32_t wave_most[kThreads / 64];
    const int64_t row = (int64_t)blockIdx.x * (kThreads / L) + threadIdx.x / L;
    const int lane = threadIdx.x % L;
    if (L < kThreads && row >= a.n)
        return;
    const T *x = (const T *)((const char *)a.x + row * a.x_stride);
    const int blocks = blocks_of(a.cols), padded = (a.cols + 15) / 16 * 2;   // blocks of 8 columns
    uint32_t most = 0;
    for (int b = lane; b < blocks; b += L) {
        const int count = a.cols - b * kCols;
        const Raw<T> r = count >= kCols ? load_block(x + b * kCols)
                                        : load_block(x + b * kCols, count);
#pragma unroll
        for (int i = 0; i < kCols; ++i)
            most = max(most, __float_as_uint((float)r[i]) & 0x7fffffffu);
    }
#pragma unroll
    for (int s = 1; s < (L < 64 ? L : 64); s <<= 1)
        most = max(most, __shfl_xor(most, s));
    if (L > 64) {
        if ((threadIdx.x & 63) == 0)
            wave_most[threadIdx.x >> 6] = most;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kThreads / 64; ++w)
            most = max(most, wave_most[w]);
    }
    const RowScale s = row_scale(most);
    if (lane == 0)
        a.scales[row] = s.scale;
    int8_t *q = a.q + row * a.q_stride;
    for (int b = lane; b < padded; b += L) {
        const int count = a.cols - b * kCols;
        const Raw<T> r = count >= kCols ? load_block(x + b * kCols)
                                        : load_block(x + b * kCols, count);
        float v[kCols];
#pragma unroll
        for (int i = 0; i < kCols; ++i)
            v[i] = (float)r[i];
        *(uint64_t *)(q + b * kCols) = eight_bits(v, s);
    }
}

template <typename T>
void launch_quantize_type(const QuantizeArgs &a, hipStream_t stream) {
    if (a.cols <= 16 * kCols)
        quantize_kernel<T, 16><<<(unsigned)((a.n + 15) / 16), kThreads, 0, stream>>>(a);
    else if (a.cols <= 64 * kCols)
        quantize_kernel<T, 64><<<(unsigned)((a.n + 3) / 4), kThreads, 0, stream>>>(a);
    else
        quantize_kernel<T, kThreads><<<(unsigned)a.n, kThreads, 0, stream>>>(a);
}

// ---- product ----

template <typename TO>
__device__ __forceinline__ float finish(int sum, float scale_a, float scale_b, float bias,
                                        bool relu) {
    const float y = (float)sum * scale_a * scale_b + bias;
    return relu && y < 0.0f ? 0.0f : y;           // a NaN stays one
}

// Tiles of 64 x 64 results, 64 bytes of k at a time through LDS; four wavefronts of 32 x 32.
// The weights are the matrix instruction's first operand, so that a lane holds four consecutive
// columns of one output row.
template <typename TO>
__global__ __launch_bounds__(kThreads) void product_kernel(ProductArgs p) {
    constexpr int kTile = 64, kStep = 64, kPitch = kStep + 16;
    __shared__ __attribute__((aligned(16))) int8_t sa[kTile * kPitch], sb[kTile * kPitch];
    const int64_t tiles_n = (p.n + kTile - 1) / kTile;
    const int64_t m0 = blockIdx.x / tiles_n * kTile, n0 = blockIdx.x % tiles_n * kTile;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int row = threadIdx.x >> 2, part = (threadIdx.x & 3) * 16;
    const int8_t *ga = p.a + (m0 + row) * p.a_stride + part;
    const int8_t *gb = p.b + (n0 + row) * p.b_stride + part;
    int4_t acc[2][2] = {};
    for (int64_t k0 = 0; k0 < p.k; k0 += kStep) {
        const bool in = k0 + part < p.k;
        int4_t va = {}, vb = {};
        if (in && m0 + row < p.m)
            va = *(const int4_t *)(ga + k0);
        if (in && n0 + row < p.n)
            vb = *(const int4_t *)(gb + k0);
        __syncthreads();
        *(int4_t *)(sa + row * kPitch + part) = va;
        *(int4_t *)(sb + row * kPitch + part) = vb;
        __syncthreads();
        int4_t fa[2], fb[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            fa[i] = *(const int4_t *)(sa + ((wave >> 1) * 32 + i * 16 + (lane & 15)) * kPitch +
                                      (lane >> 4) * 16);
            fb[i] = *(const int4_t *)(sb + ((wave & 1) * 32 + i * 16 + (lane & 15)) * kPitch +
                                      (lane >> 4) * 16);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[j], fa[i], acc[i][j], 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int64_t m = m0 + (wave >> 1) * 32 + i * 16 + (lane & 15);
        if (m >= p.m)
            continue;
        const float scale_a = p.a_scales[m];
        TO *out = (TO *)((char *)p.out + m * p.out_stride);
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int64_t n = n0 + (wave & 1) * 32 + j * 16 + (lane >> 4) * 4 + r;
                if (n < p.n)
                    out[n] = (TO)finish<TO>(acc[i][j][r], scale_a, p.b_scales[n],
                                            p.bias ? p.bias[n] : 0.0f, p.relu);
            }
    }
}

template <typename TO>
void launch_product_type(const ProductArgs &p, hipStream_t stream) {
    const int64_t tiles = (p.m + 63) / 64 * ((p.n + 63) / 64);
    product_kernel<TO><<<(unsigned)tiles, kThreads, 0, stream>>>(p);
}

}  // namespace

hipError_t launch_quantize(const QuantizeArgs &a, hipStream_t stream) {
    if (a.type == kF32)
        launch_quantize_type<float>(a, stream);
    else if (a.type == kF16)
        launch_quantize_type<half_t>(a, stream);
    else
        launch_quantize_type<bf16_t>(a, stream);
    return hipGetLastError();
}

hipError_t launch_product(const ProductArgs &p, hipStream_t stream) {
    if (p.out_type == kF32)
        launch_product_type<float>(p, stream);
    else if (p.out_type == kF16)
        launch_product_type<half_t>(p, stream);
    else
        launch_product_type<bf16_t>(p, stream);
    return hipGetLastError();
}

}  // namespace ccj

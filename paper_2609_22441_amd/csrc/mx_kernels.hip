// Rows in microscaled 4-bit floating point: to 4 bits, back, and the product of two such matrices.
#include "layers_device.h"

namespace ccj {
namespace {

typedef int int4_t __attribute__((ext_vector_type(4)));
typedef int int8_words __attribute__((ext_vector_type(8)));
typedef float float4_t __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int64_t kGrid = 1 << 20;                // workgroups at most; each then takes several tiles

// ---- rows to 4 bits and back ----

struct MxLaunch {
    MxRowsArgs a;
    Divider div;
    int32_t blocks;                               // of 8 columns, per row
    int64_t tiles;
};

// Row and block of 8 columns of the units of a tile: U for each thread, kThreads apart.
struct Unit {
    int64_t row;
    uint32_t block;
};

template <int U>
__device__ __forceinline__ void units_of(const MxLaunch &l, int64_t tile, Unit (&unit)[U]) {
    const int64_t first = tile * (kThreads * U);
    const int64_t row0 = first < UINT32_MAX ? (int64_t)((uint32_t)first / (uint32_t)l.blocks)
                                            : first / l.blocks;
    const uint32_t rem = (uint32_t)(first - row0 * l.blocks);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t local = rem + threadIdx.x + u * kThreads, r = l.div(local);
        unit[u] = {row0 + r, local - r * l.blocks};
    }
}

constexpr uint32_t kInfinity = 0x7f800000u;
constexpr uint32_t kNanScale = 255;

// A scale's biased exponent from the bits of a block's largest magnitude. Rounding to one bit of
// mantissa carries into the exponent from 1.75 on.
__device__ __forceinline__ uint32_t scale_byte(uint32_t most) {
    return most >= kInfinity ? kNanScale : (uint32_t)max((int)((most + 0x200000u) >> 23) - 2, 0);
}

__device__ __forceinline__ float scale_value(uint32_t byte) {
    return __uint_as_float(byte == kNanScale ? 0x7fc00000u : byte ? byte << 23 : 0x400000u);
}

template <typename T>
__device__ __forceinline__ uint32_t top_of(const Raw<T> &x) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < kCols; ++i)
        top = max(top, __float_as_uint((float)x[i]) & 0x7fffffffu);
    return top;
}

template <int CONTROL>
__device__ __forceinline__ uint32_t max_with(uint32_t x) {
    return max(x, (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CONTROL, 0xf, 0xf, true));
}

// The largest of four lanes that hold a block of 32 values.
__device__ __forceinline__ uint32_t block_top(uint32_t x) {
    return max_with<quad_perm(2, 3, 0, 1)>(max_with<quad_perm(1, 0, 3, 2)>(x));
}

// Eight values to 4 bits. The conversion divides by the scale, a power of two (2^-127 too), and rounds
// to nearest, ties to even; beyond 6 it gives 6.
template <typename T>
__device__ __forceinline__ uint32_t four_bits(const Raw<T> &x, uint32_t byte) {
    const float scale = scale_value(byte);
    uint32_t q = 0;
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, (float)x[0], (float)x[1], scale, 0);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, (float)x[2], (float)x[3], scale, 1);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, (float)x[4], (float)x[5], scale, 2);
    q = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(q, (float)x[6], (float)x[7], scale, 3);
    return byte == kNanScale ? 0 : q;
}

// A thread takes 8 columns, four neighbours a block of 32 with its scale.
template <typename T, int U>
__global__ __launch_bounds__(kThreads) void quantize_kernel(MxLaunch l) {
    const MxRowsArgs &a = l.a;
    for (int64_t tile = blockIdx.x; tile < l.tiles; tile += gridDim.x) {
        Unit unit[U];
        units_of(l, tile, unit);
        Raw<T> x[U];
        int exchange[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int col = unit[u].block * kCols;
            const T *p = (const T *)((const char *)a.x + min(unit[u].row, a.n - 1) * a.x_stride) + col;
            exchange[u] = exchange_of(unit[u].block, a.cols);
            x[u] = col + kCols <= a.cols ? load_pieces<true>(p, exchange[u])
                                         : load_block(p, a.cols - col);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            settle(x[u], exchange[u]);
            const uint32_t byte = scale_byte(block_top(top_of(x[u])));
            if (unit[u].row >= a.n)
                continue;
            const uint32_t block = unit[u].block;
            *(uint32_t *)(a.q + unit[u].row * a.q_stride + block * 4) = four_bits(x[u], byte);
            uint8_t *scales = a.scales + unit[u].row * a.scales_stride;
            if (block % 4 == 0)
                scales[block / 4] = (uint8_t)byte;
            if (block + 1 == (uint32_t)l.blocks)  // zeros up to 16 bytes, 4 at a time
                for (uint32_t i = (uint32_t)l.blocks / 4; i % 16; i += 4)
                    *(uint32_t *)(scales + i) = 0;
        }
    }
}

template <typename T, bool TAIL, int U>
__global__ __launch_bounds__(kThreads) void dequantize_kernel(MxLaunch l) {
    const MxRowsArgs &a = l.a;
    for (int64_t tile = blockIdx.x; tile < l.tiles; tile += gridDim.x) {
        Unit unit[U];
        units_of(l, tile, unit);
        uint32_t q[U], byte[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t row = min(unit[u].row, a.n - 1);
            q[u] = *(const uint32_t *)(a.q + row * a.q_stride + unit[u].block * 4);
            byte[u] = a.scales[row * a.scales_stride + unit[u].block / 4];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (unit[u].row >= a.n)
                continue;
            const float scale = scale_value(byte[u]);
            const auto v0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q[u], scale, 0);
            const auto v1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q[u], scale, 1);
            const auto v2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q[u], scale, 2);
            const auto v3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q[u], scale, 3);
            float y[kCols] = {v0[0], v0[1], v1[0], v1[1], v2[0], v2[1], v3[0], v3[1]};
            if (byte[u] == kNanScale)
#pragma unroll
                for (int i = 0; i < kCols; ++i)
                    y[i] = scale;
            const int col = unit[u].block * kCols;
            T *p = (T *)((char *)const_cast<void *>(a.x) + unit[u].row * a.x_stride) + col;
            // Lanes 4 or 8 i on are in one row where its blocks are a multiple of 4 or 8, and then all
            // here: a tile starts at a multiple of 8 blocks as well.
            if (TAIL && col + kCols > a.cols)
                store_block(p, y, a.cols - col);
            else if (TAIL)
                store_block(p, y);
            else
                stream_block(p, y, l.blocks % 4 ? kAlone : l.blocks % 8 ? kFour : kEight);
        }
    }
}

MxLaunch rows_launch(const MxRowsArgs &a, int32_t blocks, int per_thread) {
    const int64_t per = (int64_t)kThreads * per_thread;
    return {a, Divider(blocks), blocks, (a.n * blocks + per - 1) / per};
}

unsigned grid_of(int64_t tiles) { return (unsigned)(tiles < kGrid ? tiles : kGrid); }

// One block per thread until the chip is full, then four.
bool few_blocks(int64_t rows, int32_t blocks) { return rows * blocks < (int64_t)1 << 19; }

template <typename T>
hipError_t quantize_type(const MxRowsArgs &a, hipStream_t stream) {
    const int32_t blocks = (int32_t)(mx_padded(a.cols) / kCols);
    if (few_blocks(a.n, blocks)) {
        const MxLaunch l = rows_launch(a, blocks, 1);
        quantize_kernel<T, 1><<<grid_of(l.tiles), kThreads, 0, stream>>>(l);
    } else {
        const MxLaunch l = rows_launch(a, blocks, 4);
        quantize_kernel<T, 4><<<grid_of(l.tiles), kThreads, 0, stream>>>(l);
    }
    return hipGetLastError();
}

template <typename T, bool TAIL>
hipError_t dequantize_tail(const MxRowsArgs &a, hipStream_t stream) {
    const int32_t blocks = blocks_of(a.cols);
    if (few_blocks(a.n, blocks)) {
        const MxLaunch l = rows_launch(a, blocks, 1);
        dequantize_kernel<T, TAIL, 1><<<grid_of(l.tiles), kThreads, 0, stream>>>(l);
    } else {
        const MxLaunch l = rows_launch(a, blocks, 4);
        dequantize_kernel<T, TAIL, 4><<<grid_of(l.tiles), kThreads, 0, stream>>>(l);
    }
    return hipGetLastError();
}

template <typename T>
hipError_t dequantize_type(const MxRowsArgs &a, hipStream_t stream) {
    return a.cols % kCols == 0 && even_rows(a.x, a.x_stride) ? dequantize_tail<T, false>(a, stream)
                                                             : dequantize_tail<T, true>(a, stream);
}

// ---- product ----

__device__ __forceinline__ float finish(float sum, float bias, bool relu) {
    const float y = sum + bias;
    return relu ? __builtin_elementwise_maximum(y, 0.0f) : y;         // a NaN stays one
}

__device__ __forceinline__ int8_words operand(int4_t x) {
    return int8_words{x[0], x[1], x[2], x[3], 0, 0, 0, 0};
}

// D += A B over 128 of k, of 16 rows each: lane l holds the 32 values of row l % 16 in block l / 16 and
// their scale in byte BYTE. 4: E2M1.
template <int BYTE>
__device__ __forceinline__ float4_t multiply16(int4_t a, int4_t b, float4_t c, int scale_a,
                                               int scale_b) {
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(a), operand(b), c, 4, 4, BYTE,
                                                            scale_a, BYTE, scale_b);
}

constexpr int kSkinnyWaves = 8;

// A workgroup has 16 x 16 results and its 8 wavefronts share out k, in slabs of 512 values; fragments
// come from memory to registers as the matrix instruction takes them. A lane's four blocks of a slab
// follow each other, 64 bytes and one word of scales; the sum over k may take its blocks in any order.
// The wavefronts' sums meet in LDS.
template <typename TO>
__global__ __launch_bounds__(64 * kSkinnyWaves) void skinny_kernel(MxProductArgs p) {
    constexpr int kSlab = 256;                    // bytes
    __shared__ __attribute__((aligned(16))) float part[kSkinnyWaves][256];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t tiles_n = (uint32_t)((p.n + 15) / 16);
    const int64_t m0 = (int64_t)(blockIdx.x / tiles_n) * 16, n0 = (int64_t)(blockIdx.x % tiles_n) * 16;
    const int bytes = (int)(p.k / 2), piece = (lane >> 4) * 64;
    const int64_t row_a = min(m0 + (lane & 15), p.m - 1), row_b = min(n0 + (lane & 15), p.n - 1);
    const uint8_t *a = p.a + row_a * p.a_stride, *b = p.b + row_b * p.b_stride;
    const uint8_t *sa = p.a_scales + row_a * p.a_scales_stride;
    const uint8_t *sb = p.b_scales + row_b * p.b_scales_stride;
    float4_t acc = {};
    for (int k0 = wave * kSlab; k0 < bytes; k0 += kSkinnyWaves * kSlab) {
        // Pieces past k repeat the row's first one; of a they count as zeros, and their scales as 0.
        const int at = k0 + piece;
        const bool in = at < bytes;
        int4_t fa[4], fb[4];
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            fb[c] = *(const int4_t *)(b + (in ? at : 0) + c * 16);
            fa[c] = *(const int4_t *)(a + (in ? at : 0) + c * 16);
        }
        int scale_a = *(const int *)(sa + (in ? at / 16 : 0)), scale_b = *(const int *)(sb + (in ? at / 16 : 0));
        scale_a = in ? scale_a : 0;
        scale_b = in ? scale_b : 0;
#pragma unroll
        for (int c = 0; c < 4; ++c)
            fa[c] = in ? fa[c] : int4_t{};
        acc = multiply16<0>(fb[0], fa[0], acc, scale_b, scale_a);
        acc = multiply16<1>(fb[1], fa[1], acc, scale_b, scale_a);
        acc = multiply16<2>(fb[2], fa[2], acc, scale_b, scale_a);
        acc = multiply16<3>(fb[3], fa[3], acc, scale_b, scale_a);
    }
    *(float4_t *)&part[wave][lane * 4] = acc;
    __syncthreads();
    // Lane l's register r: row l % 16, column 4 (l / 16) + r.
    if (threadIdx.x < 256) {
        const int row = threadIdx.x >> 4, col = threadIdx.x & 15;
        float sum = 0.0f;
#pragma unroll
        for (int w = 0; w < kSkinnyWaves; ++w)
            sum += part[w][((col >> 2) * 16 + row) * 4 + (col & 3)];
        const int64_t m = m0 + row, n = n0 + col;
        if (m < p.m && n < p.n)
            ((TO *)((char *)p.out + m * p.out_stride))[n] =
                (TO)finish(sum, p.bias ? p.bias[n] : 0.0f, p.relu);
    }
}

template <typename TO>
hipError_t launch_skinny(const MxProductArgs &p, hipStream_t stream) {
    const int64_t tiles = (p.m + 15) / 16 * ((p.n + 15) / 16);
    if (tiles * (64 * kSkinnyWaves) > (int64_t)UINT32_MAX)
        return hipErrorInvalidConfiguration;
    skinny_kernel<TO><<<(unsigned)tiles, 64 * kSkinnyWaves, 0, stream>>>(p);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_mx_quantize(const MxRowsArgs &a, hipStream_t stream) {
    switch (a.type) {
    case kF32: return quantize_type<float>(a, stream);
    case kF16: return quantize_type<half_t>(a, stream);
    default: return quantize_type<bf16_t>(a, stream);
    }
}

hipError_t launch_mx_dequantize(const MxRowsArgs &a, hipStream_t stream) {
    switch (a.type) {
    case kF32: return dequantize_type<float>(a, stream);
    case kF16: return dequantize_type<half_t>(a, stream);
    default: return dequantize_type<bf16_t>(a, stream);
    }
}

hipError_t launch_mx_product(const MxProductArgs &p, hipStream_t stream) {
    switch (p.out_type) {
    case kF32: return launch_skinny<float>(p, stream);
    case kF16: return launch_skinny<half_t>(p, stream);
    default: return launch_skinny<bf16_t>(p, stream);
    }
}

hipError_t launch_mx_linear(const MxRowsArgs &x, const MxProductArgs &p, hipStream_t stream) {
    const hipError_t e = launch_mx_quantize(x, stream);
    return e == hipSuccess ? launch_mx_product(p, stream) : e;
}

}  // namespace ccj

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

__device__ __forceinline__ float finish(int sum, float scale_a, float scale_b, float bias,
                                        bool relu) {
    const float y = (float)sum * scale_a * scale_b + bias;
    return relu && y < 0.0f ? 0.0f : y;           // a NaN stays one
}

typedef int int16_tile __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(1))) const void global_void;
typedef __attribute__((address_space(3))) void lds_void;

__device__ const int4_t kZeros = {0, 0, 0, 0};    // read in the place of columns past k

constexpr int kStep = 64;                         // bytes of k per stage

// s_waitcnt's operand for at most `vm` vector loads outstanding and no LDS operation.
constexpr int wait_loads(int vm) { return (vm & 15) | (vm >> 4) << 14 | 7 << 4; }

// The order of memory accesses around a barrier is the source's.
__device__ __forceinline__ void stage_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Where 16-byte chunk c (0 to 3) of row r lies among the four of the row's 64 bytes: any 8 or 16
// consecutive rows have the chunks of one c in different banks.
__device__ __forceinline__ int swizzled(int row, int chunk) {
    return chunk ^ (((row >> 2) & 1) << 1 | (((row >> 1) ^ (row >> 3)) & 1));
}

// Tiles of TM rows of a by TN of b, WM x WN wavefronts. Stages of 64 bytes of k go from memory to
// LDS without passing through registers, three ahead of the one that is multiplied: each has the time
// of three stages' matrix instructions to arrive. 32 x 32 x 32 instructions: per result they read
// their operands from registers half as often as 16 x 16 x 64 ones. The weights are the first operand,
// so that a lane holds four consecutive columns of one output row; the results pass through LDS once
// more, to be written in whole rows of the wavefront's columns.
template <typename TO, int TM, int TN, int WM, int WN, int kStages>
__global__ __launch_bounds__(64 * WM * WN, 2) void tile_kernel(ProductArgs p, uint32_t tiles_m,
                                                            uint32_t tiles_n) {
    constexpr int kWaves = WM * WN, kT = 64 * kWaves;
    constexpr int kMB = TM / WM / 32, kNB = TN / WN / 32;        // 32 x 32 blocks of a wavefront
    constexpr int kLoadsA = TM * kStep / 16 / kT, kLoadsB = TN * kStep / 16 / kT;
    constexpr int kLoads = kLoadsA + kLoadsB;
    constexpr int kStageBytes = (TM + TN) * kStep;
    // A wavefront's results of 32 rows, 16 bytes more per row against bank conflicts.
    constexpr int kPitch = kNB * 32 * sizeof(TO) + 16;
    static_assert(kLoadsA >= 1 && kLoadsB >= 1 && 32 * kPitch * kWaves <= kStages * kStageBytes, "");
    __shared__ __attribute__((aligned(1024))) int8_t lds[kStages * kStageBytes];
    __shared__ __attribute__((aligned(16))) float scale_b[TN], bias[TN];

    // Workgroups go round the 8 XCDs; each gets consecutive tiles, in groups of 8 rows of tiles, so
    // that those it works on together share their rows of a and b in its L2.
    uint32_t id = blockIdx.x;
    {
        const uint32_t total = tiles_m * tiles_n, share = total / 8, more = total % 8;
        const uint32_t xcd = id % 8;
        id = xcd * share + min(xcd, more) + id / 8;
    }
    const uint32_t group = id / (8 * tiles_n), rows = min(8u, tiles_m - group * 8);
    const uint32_t in = id - group * 8 * tiles_n;
    const int64_t m0 = (int64_t)(group * 8 + in % rows) * TM, n0 = (int64_t)(in / rows) * TN;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / WN, wn = wave % WN;
    // Thread t moves 16 bytes of row t / 4 (and every kT / 4 rows on) to LDS byte 16 t.
    const int row = threadIdx.x >> 2, chunk = swizzled(row & 15, threadIdx.x & 3);
    const int8_t *from[kLoads];
#pragma unroll
    for (int i = 0; i < kLoadsA; ++i)             // rows past the last repeat it: not written
        from[i] = p.a + min(m0 + row + i * (kT / 4), p.m - 1) * p.a_stride + chunk * 16;
#pragma unroll
    for (int i = 0; i < kLoadsB; ++i)
        from[kLoadsA + i] = p.b + min(n0 + row + i * (kT / 4), p.n - 1) * p.b_stride + chunk * 16;
    for (int i = threadIdx.x; i < TN; i += kT) {
        const int64_t n = min(n0 + i, p.n - 1);
        scale_b[i] = p.b_scales[n];
        bias[i] = p.bias ? p.bias[n] : 0.0f;
    }
    const int steps = (int)((p.k + kStep - 1) / kStep);
    int8_t *const mine_of_stage = lds + wave * 1024;
    auto fetch = [&](int step) {
        int8_t *to = mine_of_stage + (step % kStages) * kStageBytes;
        if ((step + 1) * kStep > p.k) {           // the last one, of columns past k too
            const bool in_k = step * kStep + chunk * 16 < p.k;
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                from[i] = in_k ? from[i] : (const int8_t *)&kZeros;
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int at = i < kLoadsA ? i * kT * 16 : TM * kStep + (i - kLoadsA) * kT * 16;
            __builtin_amdgcn_global_load_lds((global_void *)from[i], (lds_void *)(to + at), 16, 0, 0);
            from[i] += kStep;
        }
    };
    int16_tile acc[kMB][kNB] = {};
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s)
        if (s < steps)
            fetch(s);
    // A fragment: lane l holds 16 bytes of row l % 32, chunk l / 32 of a half of the stage's k.
    const int frow = lane & 31;
    const int8_t *const sa = lds + (wm * (TM / WM) + frow) * kStep;
    const int8_t *const sb = lds + (TM + wn * (TN / WN) + frow) * kStep;
    const int at[2] = {swizzled(frow & 15, lane >> 5) * 16, swizzled(frow & 15, 2 + (lane >> 5)) * 16};
    int4_t fa[2][kMB], fb[2][kNB];                // of both halves of a stage
    auto read = [&](int h, int step) {
        const int stage = step % kStages * kStageBytes;
#pragma unroll
        for (int j = 0; j < kNB; ++j)
            fb[h][j] = *(const int4_t *)(sb + stage + j * 32 * kStep + at[h]);
#pragma unroll
        for (int i = 0; i < kMB; ++i)
            fa[h][i] = *(const int4_t *)(sa + stage + i * 32 * kStep + at[h]);
    };
    auto multiply = [&](int h) {
#pragma unroll
        for (int i = 0; i < kMB; ++i)
#pragma unroll
            for (int j = 0; j < kNB; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(fb[h][j], fa[h][i], acc[i][j], 0,
                                                                  0, 0);
        // One read after each of the first matrix instructions, so that none of them waits for it.
#pragma unroll
        for (int i = 0; i < kMB + kNB && i < kMB * kNB; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // The fragments that one half's matrix instructions take are read while the other half's run; so
    // a step begins with its first half in registers and reads into the next stage at its end.
    if (steps >= kStages - 1)
        __builtin_amdgcn_s_waitcnt(wait_loads((kStages - 2) * kLoads));
    else
        __builtin_amdgcn_s_waitcnt(wait_loads(0));
    stage_barrier();
    if (steps > 0)
        read(0, 0);
    for (int step = 0; step < steps; ++step) {
        if (step + kStages - 2 < steps)
            __builtin_amdgcn_s_waitcnt(wait_loads((kStages - 3) * kLoads));
        else
            __builtin_amdgcn_s_waitcnt(wait_loads(0));
        // Every wavefront's loads of the next stage are in LDS, and the stage whose place is fetched
        // into has been read by all.
        stage_barrier();
        __builtin_amdgcn_sched_barrier(0);
        read(1, step);
        multiply(0);
        if (step + kStages - 1 < steps)
            fetch(step + kStages - 1);
        __builtin_amdgcn_sched_barrier(0);
        read(0, step + 1);                        // past the last step: not used
        multiply(1);
    }
    stage_barrier();                              // the stages' LDS now holds results

    int8_t *mine = lds + wave * 32 * kPitch;
    const int64_t wave_m = m0 + wm * (TM / WM), wave_n = n0 + wn * (TN / WN);
    constexpr int kEach = 16 / sizeof(TO), kLanes = kNB * 32 / kEach;       // lanes per output row
#pragma unroll
    for (int i = 0; i < kMB; ++i) {
        const int64_t m = wave_m + i * 32 + frow;
        const float scale_a = p.a_scales[min(m, p.m - 1)];
#pragma unroll
        for (int j = 0; j < kNB; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                // Registers 4 g to 4 g + 3: columns 8 g + 4 (lane / 32) and the three after it.
                const int col = j * 32 + g * 8 + (lane >> 5) * 4;
                typedef float floats __attribute__((ext_vector_type(4)));
                typedef TO values __attribute__((ext_vector_type(4)));
                floats y;
                const floats sb = *(const floats *)(scale_b + wn * (TN / WN) + col);
                const floats bb = *(const floats *)(bias + wn * (TN / WN) + col);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    y[r] = finish(acc[i][j][g * 4 + r], scale_a, sb[r], bb[r], p.relu);
                *(values *)(mine + frow * kPitch + col * sizeof(TO)) =
                    __builtin_convertvector(y, values);
            }
        // The wavefront's own rows: its LDS writes come before its reads.
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int r = 0; r < 32; r += 64 / kLanes) {
            const int at = r + lane / kLanes, col = lane % kLanes * kEach;
            const int64_t to_m = wave_m + i * 32 + at, n = wave_n + col;
            if (to_m < p.m && n < p.n) {
                const words_t w = (words_t) * (const int4_t *)(mine + at * kPitch + col * sizeof(TO));
                TO *out = (TO *)((char *)p.out + to_m * p.out_stride) + n;
                if (n + kEach <= p.n) {
                    *(words_t *)out = w;
                } else {
                    TO v[kEach];
                    __builtin_memcpy(v, &w, 16);
                    for (int e = 0; n + e < p.n; ++e)
                        out[e] = v[e];
                }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

template <typename TO, int TM, int TN, int WM, int WN, int kStages>
hipError_t launch_tiles(const ProductArgs &p, hipStream_t stream) {
    const int64_t tm = (p.m + TM - 1) / TM, tn = (p.n + TN - 1) / TN;
    if (tm * tn * (64 * WM * WN) > (int64_t)UINT32_MAX)
        return hipErrorInvalidConfiguration;
    tile_kernel<TO, TM, TN, WM, WN, kStages><<<(unsigned)(tm * tn), 64 * WM * WN, 0, stream>>>(
        p, (uint32_t)tm, (uint32_t)tn);
    return hipGetLastError();
}

template <typename TO>
hipError_t launch_product_type(const ProductArgs &p, hipStream_t stream) {
    if (p.m > 128 * 12 && p.n > 128 * 12)
        return launch_tiles<TO, 256, 256, 2, 4, 4>(p, stream);
    return launch_tiles<TO, 128, 128, 2, 2, 4>(p, stream);
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
    switch (p.out_type) {
    case kF32: return launch_product_type<float>(p, stream);
    case kF16: return launch_product_type<half_t>(p, stream);
    default: return launch_product_type<bf16_t>(p, stream);
    }
}

}  // namespace ccj

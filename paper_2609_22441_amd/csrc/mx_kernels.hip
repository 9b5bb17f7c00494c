// Rows in microscaled 4-bit floating point: to 4 bits, back, and the product of two such matrices.
//
// To 4 bits and back are bound by memory: 16,384 x 8,192 bf16 59 us (339 MB, 5.8 TB/s) and 49 (339 MB, 6.9;
// part of its input is in the caches). Large products are bound by power and by the way from L2 to LDS, as far
// as an earlier step of the kernel with parts left out shows, and leave the matrix units idle while they
// write: 16,384 x 8,192 x 8,192 515 us (4,270 TFLOP/s; matrix instructions on values in registers make 6,300),
// 8,192 x 16,384 x 4,096 280 (3,930, 268 MB of output follow the sums). Those of few rows by the launch and
// the weights' way: 1 x 4,096 x 4,096 with the quantisation 4.4 us, 9.4 MB at 2.1 TB/s.
#include <type_traits>

#include "layers_device.h"
#include "mx_choice.h"

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

// Block at `col` of a row, zeros behind its end.
template <typename T>
__device__ __forceinline__ Raw<T> row_block(const T *p, int col, int cols) {
    return col + kCols <= cols ? load_block(p + col) : load_block(p + col, cols - col);
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

typedef float float16_tile __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) void lds_void;

// The same over 64 of k, of 32 rows each: lane l holds the values of row l % 32 in block l / 32.
template <int BYTE>
__device__ __forceinline__ float16_tile multiply32(int4_t a, int4_t b, float16_tile c, int scale_a,
                                                   int scale_b) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(a), operand(b), c, 4, 4, BYTE,
                                                           scale_a, BYTE, scale_b);
}

constexpr int kStep = 128;                        // bytes of k per stage: 256 values, 8 scales

// Rows of a matrix from one on: offsets into them are 32 bits, and nothing behind them is read whatever
// the offset.
constexpr int64_t kMaxStride = 1 << 24;           // 255 rows of it and one more: below 2^32

struct Rows {
    const uint8_t *p;
    uint32_t bytes;
    __device__ Rows(const uint8_t *matrix, int64_t stride, int64_t first, int rows, int width)
        : p(matrix + first * stride), bytes((uint32_t)((rows - 1) * stride + width)) {}
    // 16 bytes a lane to LDS, in the order of the lanes. In assembly, as the compiler would wait for
    // all such loads before any read of LDS, and with them for the stage that was asked for last; the
    // kernel's own waits are what orders them. The operand registers are ready after 5 wait states
    // whatever wrote them, m0 after one.
    __device__ __forceinline__ void to_lds(uint8_t *lds, uint32_t at, int more) const {
        const uint64_t address = (uint64_t)(uintptr_t)p;
        const int4_t buffer = {(int)(uint32_t)address, (int)(uint32_t)(address >> 32) & 0xffff,
                               (int)bytes, 0x20000};
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                     :
                     : "s"((uint32_t)(uintptr_t)(lds_void *)lds), "v"(at), "s"(buffer), "s"(more)
                     : "memory", "m0");
    }
};

// s_waitcnt's operand for at most `vm` vector loads outstanding and no LDS operation.
constexpr int wait_loads(int vm) { return (vm & 15) | (vm >> 4) << 14 | 7 << 4; }

// The order of memory accesses around a barrier is the source's.
__device__ __forceinline__ void stage_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Where 16-byte chunk c (0 to 7) of row r lies among the eight of the row's 128 bytes: any 16
// consecutive rows have the chunks of one c in different banks.
__device__ __forceinline__ int swizzled(int row, int chunk) { return chunk ^ ((row >> 1) & 7); }

// Tiles of TM rows of a by TN of b, WM x WN wavefronts. A stage of k is 128 bytes of every row, a whole
// cache line: half of one at a time would be fetched twice from L2, as the caches next to the unit hold
// less than the stages on the way (16,384 x 8,192 x 8,192 598 us with four stages of 64 bytes, 534 with two
// of 128, 515 with a stage's fragments in registers before its place is fetched into). It goes from memory to LDS without passing through registers, while
// the stage before it is multiplied; the scales of two stages go with the first of them, 16 bytes a
// row. The weights are the first operand, so that a lane holds four consecutive columns of one output
// row; the results pass through LDS once more, to be written in whole rows of the wavefront's columns.
//
// SPLIT groups of WM x WN wavefronts take every SPLIT-th stage of k each, for tiles too few to fill the
// chip; their sums meet in LDS, in the groups' order.
template <typename TO, int TM, int TN, int WM, int WN, int SPLIT>
__global__ __launch_bounds__(64 * WM * WN * SPLIT, 2) void tile_kernel(MxProductArgs p,
                                                                       uint32_t tiles_m,
                                                                       uint32_t tiles_n) {
    constexpr int kWaves = WM * WN, kT = 64 * kWaves;            // of a group
    constexpr int kMB = TM / WM / 32, kNB = TN / WN / 32;        // 32 x 32 blocks of a wavefront
    constexpr int kLoadsA = TM * kStep / 16 / kT, kLoadsB = TN * kStep / 16 / kT;
    constexpr int kLoads = kLoadsA + kLoadsB;
    constexpr int kStageBytes = (TM + TN) * kStep;
    // Rows of scales are fetched in kScaleLoads rounds by the wavefronts that they suffice for.
    constexpr int kScaleRows = TM + TN, kScaleLoads = (kScaleRows + kT - 1) / kT;
    constexpr int kScaleBytes = kScaleRows * 16;
    static_assert(kScaleRows % 64 == 0 && kLoadsA >= 1 && kLoadsB >= 1, "");
    // A wavefront's results of 32 rows, 16 bytes more per row against bank conflicts.
    constexpr int kPitch = kNB * 32 * sizeof(TO) + 16;
    constexpr int kGroupBytes = 2 * (kStageBytes + kScaleBytes);
    constexpr int kSums = kWaves * kMB * kNB * 4096;             // bytes of a group's sums
    static_assert(SPLIT == 1 || kSums <= kGroupBytes, "");
    constexpr int kStaged = SPLIT * kGroupBytes, kOutput = 32 * kPitch * kWaves;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[kStaged > kOutput ? kStaged : kOutput];
    __shared__ __attribute__((aligned(16))) float bias[TN];

    // Workgroups go round the 8 XCDs; each gets consecutive tiles, in groups of 4 rows of tiles, so
    // that those it works on together share their rows of a and b in its L2.
    uint32_t id = blockIdx.x;
    {
        const uint32_t total = tiles_m * tiles_n, share = total / 8, more = total % 8;
        const uint32_t xcd = id % 8;
        id = xcd * share + min(xcd, more) + id / 8;
    }
    const uint32_t group = id / (4 * tiles_n), rows = min(4u, tiles_m - group * 4);
    const uint32_t in = id - group * 4 * tiles_n;
    const int64_t m0 = (int64_t)(group * 4 + in % rows) * TM, n0 = (int64_t)(in / rows) * TN;

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % kWaves;
    const int split = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / kWaves;
    const int wm = wave / WN, wn = wave % WN;
    // Thread t of a group moves 16 bytes of row t / 8 (and every kT / 8 rows on) to LDS byte 16 t, and
    // 16 scales of row t (and every kT rows on).
    const int thread = threadIdx.x % kT, row = thread >> 3, chunk = swizzled(row & 15, thread & 7);
    const int bytes = (int)(p.k / 2), scale_width = (bytes + 255) / 256 * 16;
    const int rows_a = (int)min(p.m - m0, (int64_t)TM), rows_b = (int)min(p.n - n0, (int64_t)TN);
    const Rows a(p.a, p.a_stride, m0, rows_a, bytes), b(p.b, p.b_stride, n0, rows_b, bytes);
    const Rows a_scales(p.a_scales, p.a_scales_stride, m0, rows_a, scale_width);
    const Rows b_scales(p.b_scales, p.b_scales_stride, n0, rows_b, scale_width);
    uint32_t from[kLoads], from_scales[kScaleLoads];
#pragma unroll
    for (int i = 0; i < kLoadsA; ++i)             // rows past the last repeat it: not written
        from[i] = (uint32_t)min(row + i * (kT / 8), rows_a - 1) * (uint32_t)p.a_stride + chunk * 16;
#pragma unroll
    for (int i = 0; i < kLoadsB; ++i)
        from[kLoadsA + i] =
            (uint32_t)min(row + i * (kT / 8), rows_b - 1) * (uint32_t)p.b_stride + chunk * 16;
#pragma unroll
    for (int i = 0; i < kScaleLoads; ++i) {
        const int at = thread + i * kT;           // rows of a, then of b; past them the last
        from_scales[i] = at < TM ? (uint32_t)min(at, rows_a - 1) * (uint32_t)p.a_scales_stride
                                 : (uint32_t)min(at - TM, rows_b - 1) * (uint32_t)p.b_scales_stride;
    }
    for (int i = threadIdx.x; i < TN; i += kT * SPLIT)
        bias[i] = p.bias ? p.bias[min(n0 + i, p.n - 1)] : 0.0f;
    // Stages of k, the last perhaps half of one; how many of them are this group's, and a group's most.
    const int all = (bytes + kStep - 1) / kStep;
    const int steps = (all + SPLIT - 1 - split) / SPLIT, most = (all + SPLIT - 1) / SPLIT;
    uint8_t *const stages = lds + split * kGroupBytes;
    uint8_t *const scale_places = stages + 2 * kStageBytes;
    auto fetch = [&](int step) {
        const int stage = step * SPLIT + split;
        if (SPLIT > 1 || step % 2 == 0) {
            uint8_t *to = scale_places + (SPLIT > 1 ? step : step / 2) % 2 * kScaleBytes + wave * 1024;
#pragma unroll
            for (int i = 0; i < kScaleLoads; ++i)
                if (wave * 64 + i * kT < kScaleRows)
                    (wave * 64 + i * kT < TM ? a_scales : b_scales)
                        .to_lds(to + i * kT * 16, from_scales[i], stage / 2 * 16);
        }
        uint8_t *to = stages + wave * 1024 + step % 2 * kStageBytes;
        if ((stage + 1) * kStep > bytes) {        // half a stage, in the place of the other the same again
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                from[i] -= chunk & 4 ? 64 : 0;
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int place = i < kLoadsA ? i * kT * 16 : TM * kStep + (i - kLoadsA) * kT * 16;
            (i < kLoadsA ? a : b).to_lds(to + place, from[i], stage * kStep);
        }
    };
    float16_tile acc[kMB][kNB] = {};
    if (0 < steps)
        fetch(0);
    if (1 < steps)
        fetch(1);
    // A fragment: lane l holds 16 bytes of row l % 32. The sum over k may take a stage's eight chunks in
    // any order: a lane takes numbers 4 (l / 32) to 4 (l / 32) + 3, whose scales are one word.
    const int frow = lane & 31, upper = lane >> 5;
    const uint8_t *const sa = stages + (wm * (TM / WM) + frow) * kStep;
    const uint8_t *const sb = stages + (TM + wn * (TN / WN) + frow) * kStep;
    const uint8_t *const ca = scale_places + (wm * (TM / WM) + frow) * 16 + upper * 4;
    const uint8_t *const cb = scale_places + (TM + wn * (TN / WN) + frow) * 16 + upper * 4;
    int4_t fa[4][kMB], fb[4][kNB];                // of a stage's quarters
    int ea[kMB], eb[kNB], next_a[kMB], next_b[kNB];       // scales of a stage and of the next
    auto read = [&](auto quarter, int step) {
        constexpr int h = decltype(quarter)::value;
        const int at = step % 2 * kStageBytes + swizzled(frow & 15, upper * 4 + h) * 16;
#pragma unroll
        for (int j = 0; j < kNB; ++j)
            fb[h][j] = *(const int4_t *)(sb + at + j * 32 * kStep);
#pragma unroll
        for (int i = 0; i < kMB; ++i)
            fa[h][i] = *(const int4_t *)(sa + at + i * 32 * kStep);
    };
    auto read_scales = [&](int step) {
        const int stage = step * SPLIT + split;
        const int place = (SPLIT > 1 ? step : step / 2) % 2 * kScaleBytes + stage % 2 * 8;
#pragma unroll
        for (int j = 0; j < kNB; ++j)
            next_b[j] = *(const int *)(cb + place + j * 32 * 16);
#pragma unroll
        for (int i = 0; i < kMB; ++i)
            next_a[i] = *(const int *)(ca + place + i * 32 * 16);
    };
    // Of half a stage, the upper lanes' values have no part: with scales of 2^-127 on both sides their
    // products, below 2^-243 in all, do not reach 32 bits.
    auto take_scales = [&](int step) {
        const bool in_k = (step * SPLIT + split) * kStep + upper * 64 < bytes;
#pragma unroll
        for (int j = 0; j < kNB; ++j)
            eb[j] = in_k ? next_b[j] : 0;
#pragma unroll
        for (int i = 0; i < kMB; ++i)
            ea[i] = in_k ? next_a[i] : 0;
    };
    auto multiply = [&](auto quarter) {
        constexpr int h = decltype(quarter)::value;
#pragma unroll
        for (int i = 0; i < kMB; ++i)
#pragma unroll
            for (int j = 0; j < kNB; ++j)
                acc[i][j] = multiply32<h>(fb[h][j], fa[h][i], acc[i][j], eb[j], ea[i]);
        // The reads of LDS between the first quarter's and the last one's matrix instructions.
        if (h == 0 || h == 3)
#pragma unroll
            for (int i = 0; i < kMB * kNB; ++i) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                __builtin_amdgcn_sched_group_barrier(0x100, h == 0 ? 3 : 2, 0);
            }
        __builtin_amdgcn_sched_barrier(0);
    };
    // The matrix instructions above stay above: nothing in the program keeps them from moving down past
    // the barrier to the next use of their results, behind the reads that they are to overlap.
    auto pin = [&] {
#pragma unroll
        for (int i = 0; i < kMB; ++i)
#pragma unroll
            for (int j = 0; j < kNB; ++j)
                asm volatile("" : "+v"(acc[i][j]));
    };
    using std::integral_constant;
    if (steps > 1)                                // the first stage and its scales are here
        __builtin_amdgcn_s_waitcnt(wait_loads(kLoads));
    else
        __builtin_amdgcn_s_waitcnt(wait_loads(0));
    stage_barrier();
    // A step begins with its first quarter in registers. While that is multiplied the others are read,
    // so that the stage's place is free, and the stage after the next on its way, before three quarters
    // of the matrix instructions; the next stage, which was asked for a step ago, is here by then.
    read(integral_constant<int, 0>(), 0);
    read_scales(0);
    take_scales(0);
    for (int step = 0; step < most; ++step) {
        const bool mine = SPLIT == 1 || step < steps;            // else others of the workgroup go on
        if (mine) {
            __builtin_amdgcn_sched_barrier(0);
            read(integral_constant<int, 1>(), step);
            read(integral_constant<int, 2>(), step);
            read(integral_constant<int, 3>(), step);
            multiply(integral_constant<int, 0>());
            pin();
        }
        __builtin_amdgcn_s_waitcnt(wait_loads(0));
        stage_barrier();
        if (mine) {
            if (step + 2 < steps)
                fetch(step + 2);
            __builtin_amdgcn_sched_barrier(0);
            multiply(integral_constant<int, 1>());
            multiply(integral_constant<int, 2>());
            read(integral_constant<int, 0>(), step + 1);         // past the last step: not used
            read_scales(step + 1);
            multiply(integral_constant<int, 3>());
            take_scales(step + 1);
        }
    }
    stage_barrier();                              // the stages' LDS now holds results
    if constexpr (SPLIT > 1) {
        if (split)
#pragma unroll
            for (int b = 0; b < kMB * kNB; ++b)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    *(float4_t *)(stages + ((wave * kMB * kNB + b) * 4 + g) * 1024 + lane * 16) =
                        float4_t{acc[b / kNB][b % kNB][4 * g], acc[b / kNB][b % kNB][4 * g + 1],
                                 acc[b / kNB][b % kNB][4 * g + 2], acc[b / kNB][b % kNB][4 * g + 3]};
        __syncthreads();
        if (split)
            return;
#pragma unroll
        for (int s = 1; s < SPLIT; ++s)
#pragma unroll
            for (int b = 0; b < kMB * kNB; ++b)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const float4_t v = *(const float4_t *)(stages + s * kGroupBytes +
                                                           ((wave * kMB * kNB + b) * 4 + g) * 1024 +
                                                           lane * 16);
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        acc[b / kNB][b % kNB][4 * g + r] += v[r];
                }
    }

    uint8_t *mine = lds + wave * 32 * kPitch;
    const int64_t wave_m = m0 + wm * (TM / WM), wave_n = n0 + wn * (TN / WN);
    constexpr int kEach = 16 / sizeof(TO), kLanes = kNB * 32 / kEach;       // lanes per output row
#pragma unroll
    for (int i = 0; i < kMB; ++i) {
#pragma unroll
        for (int j = 0; j < kNB; ++j)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                // Registers 4 g to 4 g + 3: columns 8 g + 4 (lane / 32) and the three after it.
                const int col = j * 32 + g * 8 + upper * 4;
                typedef TO out4_t __attribute__((ext_vector_type(4)));
                float4_t y;
                const float4_t bb = *(const float4_t *)(bias + wn * (TN / WN) + col);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    y[r] = finish(acc[i][j][g * 4 + r], bb[r], p.relu);
                *(out4_t *)(mine + frow * kPitch + col * sizeof(TO)) =
                    __builtin_convertvector(y, out4_t);
            }
        // The wavefront's own rows: its LDS writes come before its reads.
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int r = 0; r < 32; r += 64 / kLanes) {
            const int at_row = r + lane / kLanes, col = lane % kLanes * kEach;
            const int64_t to_m = wave_m + i * 32 + at_row, n = wave_n + col;
            if (to_m < p.m && n < p.n) {
                const words_t w = (words_t) * (const int4_t *)(mine + at_row * kPitch + col * sizeof(TO));
                TO *out = (TO *)((char *)p.out + to_m * p.out_stride) + n;
                if (n + kEach <= p.n) {
                    __builtin_nontemporal_store(w, (words_t *)out);
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

constexpr int kSkinnyWaves = 8;

// A workgroup has 16 x 16 results and its 8 wavefronts share out k, in slabs of 512 values; fragments
// come from memory to registers as the matrix instruction takes them. A lane's four blocks of a slab
// follow each other, 64 bytes and one word of scales; the sum over k may take its blocks in any order.
// The wavefronts' sums meet in LDS. TWO: two slabs of a wavefront are on their way at a time, for rows of
// more than one slab each.
//
// QUANT: the rows of a (at most 16) are put in 4 bits from x in the kernel, by every workgroup again: a
// few KiB from L2 on the weights' way, against a launch of their own.
template <typename TO, bool QUANT, bool TWO>
__global__ __launch_bounds__(64 * kSkinnyWaves) void skinny_kernel(MxProductArgs p, MxRowsArgs x,
                                                                   Divider div) {
    constexpr int kT = 64 * kSkinnyWaves, kSlab = 256, kStep = kSkinnyWaves * kSlab;   // threads; bytes
    extern __shared__ __attribute__((aligned(16))) uint8_t quantized[];
    __shared__ __attribute__((aligned(16))) float part[kSkinnyWaves][256];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t tiles_n = (uint32_t)((p.n + 15) / 16);
    const int64_t m0 = (int64_t)(blockIdx.x / tiles_n) * 16, n0 = (int64_t)(blockIdx.x % tiles_n) * 16;
    const int bytes = (int)(p.k / 2), piece = (lane >> 4) * 64;
    const int64_t row_a = min(m0 + (lane & 15), p.m - 1), row_b = min(n0 + (lane & 15), p.n - 1);
    // Rows in LDS are 16 bytes longer, against bank conflicts; their scales lie behind them.
    const int pitch = bytes + 16, scale_pitch = bytes / 16 + 4;
    uint8_t *const quantized_scales = quantized + (QUANT ? p.m * pitch : 0);
    const uint8_t *a = QUANT ? quantized + row_a * pitch : p.a + row_a * p.a_stride;
    const uint8_t *sa = QUANT ? quantized_scales + row_a * scale_pitch
                              : p.a_scales + row_a * p.a_scales_stride;
    const uint8_t *b = p.b + row_b * p.b_stride;
    const uint8_t *sb = p.b_scales + row_b * p.b_scales_stride;
    // Pieces past k repeat the row's first one, with scales of 2^-127 on both sides: their products,
    // below 2^-243 in all, do not reach 32 bits.
    auto read = [&](const uint8_t *from, const uint8_t *scales, int4_t (&f)[4], int &scale, int k0) {
        const int at = k0 + piece < bytes ? k0 + piece : 0;
#pragma unroll
        for (int c = 0; c < 4; ++c)
            f[c] = *(const int4_t *)(from + at + c * 16);
        scale = *(const int *)(scales + at / 16);
        scale = k0 + piece < bytes ? scale : 0;
    };
    int4_t fa[4], fb[4], ga[4], gb[4];
    int scale_fa, scale_fb, scale_ga, scale_gb;
    const int first = wave * kSlab;
    auto read_b = [&](int k0) {
        read(b, sb, fb, scale_fb, k0);
        if (TWO && k0 + kStep < bytes)
            read(b, sb, gb, scale_gb, k0 + kStep);
    };
    if (first < bytes)
        read_b(first);
    if constexpr (QUANT) {
        constexpr int kU = 4;                     // blocks of 8 columns of a thread on their way
        const int blocks = bytes / 4, units = (int)p.m * blocks;
        for (int unit0 = threadIdx.x; unit0 < units; unit0 += kT * kU) {
            Raw<TO> v[kU];
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                const int unit = min(unit0 + u * kT, units - 4 + (int)(threadIdx.x & 3));
                const int row = div(unit), col = (unit - row * blocks) * kCols;
                v[u] = row_block((const TO *)((const char *)x.x + row * x.x_stride), col, x.cols);
            }
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                const uint32_t byte = scale_byte(block_top(top_of(v[u])));
                const int unit = unit0 + u * kT;
                if (unit < units) {
                    const int row = div(unit), block = unit - row * blocks;
                    *(uint32_t *)(quantized + row * pitch + block * 4) = four_bits(v[u], byte);
                    if (block % 4 == 0)
                        quantized_scales[row * scale_pitch + block / 4] = (uint8_t)byte;
                }
            }
        }
        __syncthreads();
    }
    float4_t acc = {};
    auto add = [&](const int4_t (&x)[4], int scale_x, const int4_t (&y)[4], int scale_y) {
        acc = multiply16<0>(x[0], y[0], acc, scale_x, scale_y);
        acc = multiply16<1>(x[1], y[1], acc, scale_x, scale_y);
        acc = multiply16<2>(x[2], y[2], acc, scale_x, scale_y);
        acc = multiply16<3>(x[3], y[3], acc, scale_x, scale_y);
    };
    for (int k0 = first; k0 < bytes; k0 += (TWO ? 2 : 1) * kStep) {
        const bool two = TWO && k0 + kStep < bytes;
        if (k0 != first)
            read_b(k0);
        read(a, sa, fa, scale_fa, k0);
        if (two)
            read(a, sa, ga, scale_ga, k0 + kStep);
        add(fb, scale_fb, fa, scale_fa);
        if (two)
            add(gb, scale_gb, ga, scale_ga);
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

template <typename TO, int TM, int TN, int WM, int WN, int SPLIT>
hipError_t launch_tiles(const MxProductArgs &p, hipStream_t stream) {
    const int64_t tm = (p.m + TM - 1) / TM, tn = (p.n + TN - 1) / TN;
    if (tm * tn * (64 * WM * WN * SPLIT) > (int64_t)UINT32_MAX)
        return hipErrorInvalidConfiguration;
    tile_kernel<TO, TM, TN, WM, WN, SPLIT>
        <<<(unsigned)(tm * tn), 64 * WM * WN * SPLIT, 0, stream>>>(p, (uint32_t)tm, (uint32_t)tn);
    return hipGetLastError();
}

// Of rows that lie far apart there may be more tiles than a launch has room for: several launches then, of
// as many columns as fit and of as many rows as these leave room for.
template <typename TO>
hipError_t launch_skinny(const MxProductArgs &all, hipStream_t stream) {
    const auto kernel = all.k > kMxOneSlab ? skinny_kernel<TO, false, true> : skinny_kernel<TO, false, false>;
    const int64_t most = UINT32_MAX / (64 * kSkinnyWaves);       // tiles
    for (int64_t n0 = 0; n0 < all.n; n0 += most * 16) {
        MxProductArgs p = all;
        p.n = all.n - n0 < most * 16 ? all.n - n0 : most * 16;
        p.b = all.b + n0 * all.b_stride;
        p.b_scales = all.b_scales + n0 * all.b_scales_stride;
        p.bias = all.bias ? all.bias + n0 : nullptr;
        const int64_t rows = most / mx_tiles(1, p.n, 16, 16) * 16;
        for (int64_t m0 = 0; m0 < all.m; m0 += rows) {
            p.m = all.m - m0 < rows ? all.m - m0 : rows;
            p.a = all.a + m0 * all.a_stride;
            p.a_scales = all.a_scales + m0 * all.a_scales_stride;
            p.out = (char *)all.out + m0 * all.out_stride + n0 * (int64_t)sizeof(TO);
            kernel<<<(unsigned)mx_tiles(p.m, p.n, 16, 16), 64 * kSkinnyWaves, 0, stream>>>(p, MxRowsArgs{},
                                                                                          Divider(1));
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess)
                return e;
        }
    }
    return hipSuccess;
}

template <typename TO>
hipError_t launch_product_type(const MxProductArgs &p, hipStream_t stream) {
    for (int64_t stride : {p.m > 1 ? p.a_stride : 0, p.n > 1 ? p.b_stride : 0,
                           p.m > 1 ? p.a_scales_stride : 0, p.n > 1 ? p.b_scales_stride : 0})
        if (p.k > 0 && stride > kMaxStride)       // rows of no columns: nothing is read
            return launch_skinny<TO>(p, stream);
    switch (mx_product_choice(p.m, p.n, p.k)) {
    case kMxSkinny: return launch_skinny<TO>(p, stream);
    case kMxTile64: return launch_tiles<TO, 64, 64, 2, 2, 2>(p, stream);
    case kMxTile128: return launch_tiles<TO, 128, 128, 2, 2, 1>(p, stream);
    default: return launch_tiles<TO, 256, 256, 2, 4, 1>(p, stream);
    }
}

template <typename T>
hipError_t launch_linear_type(const MxRowsArgs &x, const MxProductArgs &p, hipStream_t stream) {
    if (mx_quantize_inside(p.m, p.n, p.k)) {
        const int64_t tiles = mx_tiles(p.m, p.n, 16, 16);
        const auto kernel = p.k > kMxOneSlab ? skinny_kernel<T, true, true> : skinny_kernel<T, true, false>;
        kernel<<<(unsigned)tiles, 64 * kSkinnyWaves, mx_quantize_lds(p.m, p.k), stream>>>(
            p, x, Divider((uint32_t)(p.k / kCols)));
        return hipGetLastError();
    }
    const hipError_t e = quantize_type<T>(x, stream);
    return e == hipSuccess ? launch_product_type<T>(p, stream) : e;
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
    case kF32: return launch_product_type<float>(p, stream);
    case kF16: return launch_product_type<half_t>(p, stream);
    default: return launch_product_type<bf16_t>(p, stream);
    }
}

hipError_t launch_mx_linear(const MxRowsArgs &x, const MxProductArgs &p, hipStream_t stream) {
    switch (x.type) {
    case kF32: return launch_linear_type<float>(x, p, stream);
    case kF16: return launch_linear_type<half_t>(x, p, stream);
    default: return launch_linear_type<bf16_t>(x, p, stream);
    }
}

}  // namespace ccj

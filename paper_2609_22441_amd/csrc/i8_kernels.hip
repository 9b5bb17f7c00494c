// 8-bit integers with a scale per row: quantisation of rows, and the product of two such matrices.
//
// Quantisation moves bytes: 16,384 x 8,192 bf16 75 us (403 MB, 5.3 TB/s). Large products are bound by the
// matrix instructions: 8,192^3 469 us (2,345 TOPS), 8,192 x 16,384 x 4,096 522 (2,106; 268 MB of output
// follow the sums), linear 16,384 x 8,192 x 8,192 1,018 with the quantisation. Short ones by their output
// (50,000 x 512 x 96 20.9 us, 15 of them the product's), those of few rows by the weights and the launch
// (1 x 4,096 x 4,096 7.5 us).
#include "i8_choice.h"
#include "layers_device.h"

namespace ccj {
namespace {

typedef int int4_t __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kSkinnyWaves = 8;

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

// The largest magnitude of a block.
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

// The largest of 16 or 64 lanes' numbers, in all of them: within 16 lanes without LDS.
template <int LANES>
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
    constexpr int kHalfMirror = 0x141, kMirror = 0x140;
    x = max_with<quad_perm(1, 0, 3, 2)>(x);
    x = max_with<quad_perm(2, 3, 0, 1)>(x);
    x = max_with<kHalfMirror>(x);                 // lane 7 - i of each 8
    x = max_with<kMirror>(x);                     // lane 15 - i of each 16
    if (LANES == 64) {
        x = max(x, __shfl_xor(x, 16));
        x = max(x, __shfl_xor(x, 32));
    }
    return x;
}

// Eight values to 8 bits. A row with a NaN or an infinity has the factor 0 and gets zeros.
template <typename T>
__device__ __forceinline__ uint64_t eight_bits(const Raw<T> &x, const RowScale &s) {
    float v[kCols];
#pragma unroll
    for (int i = 0; i < kCols; ++i)
        v[i] = (float)x[i];
    if (s.raise != 1.0f)
#pragma unroll
        for (int i = 0; i < kCols; ++i)
            v[i] *= s.raise;
    uint32_t q[2] = {};
#pragma unroll
    for (int i = 0; i < kCols; ++i)
        q[i / 4] |= ((uint32_t)(int)rintf(v[i] * s.inverse) & 0xff) << (i % 4 * 8);
    return s.inverse == 0.0f ? 0 : (uint64_t)q[1] << 32 | q[0];
}

// A group of L lanes per row (L = 16, 64 or the workgroup), a lane with up to B blocks, which stay in
// registers between the search for the largest and the rounding: one read of x, one write of q. Rows
// longer than L * B blocks (B = 0) are read twice, the second time from the caches. Short rows go R at
// a time, all of their loads on the way together.
template <typename T, int L, int B, int R>
__global__ __launch_bounds__(kThreads) void quantize_kernel(QuantizeArgs a) {
    __shared__ uint32_t wave_most[kThreads / 64];
    const int lane = threadIdx.x % L;
    const int blocks = blocks_of(a.cols), padded = (a.cols + 15) / 16 * 2;   // blocks of 8 columns
    constexpr int kHeld = B ? B : 1, kRows = kThreads / L * R;
    static_assert(R == 1 || (B && L <= 64), "");
    for (int64_t row0 = (int64_t)blockIdx.x * kRows + threadIdx.x / L; row0 < a.n;
         row0 += (int64_t)gridDim.x * kRows) {
        auto value = [&](int64_t row, int block) {
            const T *x = (const T *)((const char *)a.x + row * a.x_stride) + block * kCols;
            const int count = a.cols - block * kCols;
            return count >= kCols ? load_once(x) : load_block(x, count);
        };
        Raw<T> held[R][kHeld];
        uint32_t most[R] = {};
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t row = min(row0 + r * (kThreads / L), a.n - 1);
            if (B) {
#pragma unroll
                for (int i = 0; i < kHeld; ++i)
                    held[r][i] = lane + i * L < blocks ? value(row, lane + i * L) : Raw<T>{};
            } else {
#pragma unroll 4
                for (int b = lane; b < blocks; b += L)
                    most[r] = max(most[r], top_of(value(row, b)));
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int64_t row = row0 + r * (kThreads / L);
            if (B)
#pragma unroll
                for (int i = 0; i < kHeld; ++i)
                    most[r] = max(most[r], top_of(held[r][i]));
            uint32_t top = wave_max<(L < 64 ? L : 64)>(most[r]);
            if (L > 64) {
                __syncthreads();
                if ((threadIdx.x & 63) == 0)
                    wave_most[threadIdx.x >> 6] = top;
                __syncthreads();
#pragma unroll
                for (int w = 0; w < kThreads / 64; ++w)
                    top = max(top, wave_most[w]);
            }
            if (row >= a.n)
                break;
            const RowScale s = row_scale(top);
            if (lane == 0)
                a.scales[row] = s.scale;
            uint64_t *q = (uint64_t *)(a.q + row * a.q_stride);
            if (B) {
#pragma unroll
                for (int i = 0; i < kHeld; ++i)
                    if (lane + i * L < padded)
                        q[lane + i * L] = eight_bits(held[r][i], s);
            } else {
                for (int b = lane; b < padded; b += L)
                    q[b] = eight_bits(value(row, b), s);
            }
        }
    }
}

template <typename T, int L, int B, int R = 1>
void launch_quantize_rows(const QuantizeArgs &a, hipStream_t stream) {
    constexpr int kRows = kThreads / L * R;
    const int64_t groups = (a.n + kRows - 1) / kRows, most = 1 << 22;
    quantize_kernel<T, L, B, R><<<(unsigned)(groups < most ? groups : most), kThreads, 0, stream>>>(a);
}

template <typename T>
void launch_quantize_type(const QuantizeArgs &a, hipStream_t stream) {
    const int blocks = (a.cols + 15) / 16 * 2;
    if (blocks <= 16)
        launch_quantize_rows<T, 16, 1, 2>(a, stream);
    else if (blocks <= 32)
        launch_quantize_rows<T, 16, 2, 2>(a, stream);
    else if (blocks <= 64)
        launch_quantize_rows<T, 64, 1, 2>(a, stream);
    else if (blocks <= 128)
        launch_quantize_rows<T, 64, 2, 2>(a, stream);
    else if (blocks <= 512)
        launch_quantize_rows<T, kThreads, 2>(a, stream);
    else if (blocks <= 2048)
        launch_quantize_rows<T, kThreads, 8>(a, stream);
    else
        launch_quantize_rows<T, kThreads, 0>(a, stream);
}

// ---- product ----

__device__ __forceinline__ float finish(int sum, float scale_a, float scale_b, float bias,
                                        bool relu) {
    const float y = (float)sum * scale_a * scale_b + bias;
    return relu ? __builtin_elementwise_maximum(y, 0.0f) : y;         // a NaN stays one
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
//
// SPLIT groups of WM x WN wavefronts take every SPLIT-th stage of k each, for tiles too few to fill the
// chip; their integer sums meet in LDS.
//
// With two stages k is at most both of them, and all of it is fetched at once: short products are
// bound by their output, and a quarter of the LDS lets four workgroups overlap their loads and stores
// on a unit.
//
// QUANT, of short k too and one tile of columns: the tile's rows are quantised from x on their way to
// LDS, so that no 8-bit rows are written to memory and read back.
template <typename TO, int TM, int TN, int WM, int WN, int SPLIT, int kStages, bool QUANT>
__global__ __launch_bounds__(64 * WM * WN * SPLIT, 2) void tile_kernel(ProductArgs p, uint32_t tiles_m,
                                                                       uint32_t tiles_n,
                                                                       LinearArgs x) {
    constexpr int kWaves = WM * WN, kT = 64 * kWaves;            // of a group
    constexpr int kMB = TM / WM / 32, kNB = TN / WN / 32;        // 32 x 32 blocks of a wavefront
    constexpr int kLoadsA = TM * kStep / 16 / kT, kLoadsB = TN * kStep / 16 / kT;
    constexpr int kLoads = kLoadsA + kLoadsB;
    constexpr int kStageBytes = (TM + TN) * kStep;
    // A wavefront's results of 32 rows, 16 bytes more per row against bank conflicts.
    constexpr int kPitch = kNB * 32 * sizeof(TO) + 16;
    constexpr bool kWhole = kStages == 2;
    static_assert(kWhole || (kStages >= 3 && !QUANT), "");
    constexpr int kSums = kWaves * kMB * kNB * 4096;             // bytes of a group's sums
    static_assert(kLoadsA >= 1 && kLoadsB >= 1 && (SPLIT == 1 || kSums <= kStages * kStageBytes), "");
    constexpr int kStaged = SPLIT * kStages * kStageBytes, kOutput = 32 * kPitch * kWaves;
    __shared__ __attribute__((aligned(1024))) int8_t lds[kStaged > kOutput ? kStaged : kOutput];
    __shared__ __attribute__((aligned(16))) float scale_b[TN], bias[TN], scale_q[QUANT ? TM : 1];

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
    // Thread t of a group moves 16 bytes of row t / 4 (and every kT / 4 rows on) to LDS byte 16 t.
    const int row = (threadIdx.x % kT) >> 2, chunk = swizzled(row & 15, threadIdx.x & 3);
    const int8_t *from[kLoads];
#pragma unroll
    for (int i = 0; i < (QUANT ? 0 : kLoadsA); ++i)      // rows past the last repeat it: not written
        from[i] = p.a + min(m0 + row + i * (kT / 4), p.m - 1) * p.a_stride + chunk * 16 +
                  split * kStep;
#pragma unroll
    for (int i = 0; i < kLoadsB; ++i)
        from[kLoadsA + i] = p.b + min(n0 + row + i * (kT / 4), p.n - 1) * p.b_stride + chunk * 16 +
                            split * kStep;
    for (int i = threadIdx.x; i < TN; i += kT * SPLIT) {
        const int64_t n = min(n0 + i, p.n - 1);
        scale_b[i] = p.b_scales[n];
        bias[i] = p.bias ? p.bias[n] : 0.0f;
    }
    // Steps of every group; the last may lie past k for some.
    const int steps = (int)((p.k + kStep * SPLIT - 1) / (kStep * SPLIT));
    int8_t *const stages = lds + split * kStages * kStageBytes;
    auto fetch = [&](int step) {
        int8_t *to = stages + wave * 1024 + (step % kStages) * kStageBytes;
        const int k0 = (step * SPLIT + split) * kStep;
        if (k0 + kStep > p.k) {                   // the last one, of columns past k too
            const bool in_k = k0 + chunk * 16 < p.k;
#pragma unroll
            for (int i = QUANT ? kLoadsA : 0; i < kLoads; ++i)
                from[i] = in_k ? from[i] : (const int8_t *)&kZeros;
        }
#pragma unroll
        for (int i = QUANT ? kLoadsA : 0; i < kLoads; ++i) {
            const int at = i < kLoadsA ? i * kT * 16 : TM * kStep + (i - kLoadsA) * kT * 16;
            __builtin_amdgcn_global_load_lds((global_void *)from[i], (lds_void *)(to + at), 16, 0, 0);
            from[i] += kStep * SPLIT;
        }
    };
    int16_tile acc[kMB][kNB] = {};
#pragma unroll
    for (int s = 0; s < (kWhole ? kStages : kStages - 1); ++s)
        if (s < steps)
            fetch(s);
    if constexpr (QUANT) {
        static_assert(SPLIT == 1, "");
        constexpr int kLanesQ = 16, kGroups = kT / kLanesQ, kRowsQ = TM / kGroups;
        constexpr int kBlocksQ = kStages * kStep / kCols / kLanesQ;           // blocks of a lane
        const int lane_q = threadIdx.x % kLanesQ, group_q = threadIdx.x / kLanesQ;
        const int blocks = blocks_of(x.cols);
        for (int r0 = 0; r0 < kRowsQ; r0 += 4) {
            Raw<TO> held[4][kBlocksQ];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int64_t m = min(m0 + group_q + (r0 + r) * kGroups, p.m - 1);
                const TO *of = (const TO *)((const char *)x.x + m * x.x_stride);
#pragma unroll
                for (int i = 0; i < kBlocksQ; ++i) {
                    const int block = lane_q + i * kLanesQ, count = x.cols - block * kCols;
                    held[r][i] = Raw<TO>{};
                    if (block < blocks)
                        held[r][i] = count >= kCols ? load_block(of + block * kCols)
                                                    : load_block(of + block * kCols, count);
                }
            }
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int at_row = group_q + (r0 + r) * kGroups;
                uint32_t most = 0;
#pragma unroll
                for (int i = 0; i < kBlocksQ; ++i)
                    most = max(most, top_of(held[r][i]));
                const RowScale s = row_scale(wave_max<kLanesQ>(most));
                if (lane_q == 0)
                    scale_q[at_row] = s.scale;
#pragma unroll
                for (int i = 0; i < kBlocksQ; ++i) {
                    const int block = lane_q + i * kLanesQ;      // of 8 bytes; zeros past the row's
                    if (block < steps * (kStep / kCols))
                        *(uint64_t *)(stages + block / 8 * kStageBytes + at_row * kStep +
                                      swizzled(at_row & 15, block % 8 / 2) * 16 + block % 2 * 8) =
                            eight_bits(held[r][i], s);
                }
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // before the barrier below
    }
    // A fragment: lane l holds 16 bytes of row l % 32, chunk l / 32 of a half of the stage's k.
    const int frow = lane & 31;
    const int8_t *const sa = stages + (wm * (TM / WM) + frow) * kStep;
    const int8_t *const sb = stages + (TM + wn * (TN / WN) + frow) * kStep;
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
    if (!kWhole && steps >= kStages - 1)
        __builtin_amdgcn_s_waitcnt(wait_loads((kStages - 2) * kLoads));
    else
        __builtin_amdgcn_s_waitcnt(wait_loads(0));
    stage_barrier();
    if (steps > 0)
        read(0, 0);
    for (int step = 0; step < steps; ++step) {
        if constexpr (!kWhole) {
            if (step + kStages - 2 < steps)
                __builtin_amdgcn_s_waitcnt(wait_loads((kStages - 3) * kLoads));
            else
                __builtin_amdgcn_s_waitcnt(wait_loads(0));
            // Every wavefront's loads of the next stage are in LDS, and the stage whose place is
            // fetched into has been read by all.
            stage_barrier();
        }
        __builtin_amdgcn_sched_barrier(0);
        read(1, step);
        multiply(0);
        if (!kWhole && step + kStages - 1 < steps)
            fetch(step + kStages - 1);
        __builtin_amdgcn_sched_barrier(0);
        read(0, step + 1);                        // past the last step: not used
        multiply(1);
    }
    stage_barrier();                              // the stages' LDS now holds results
    if constexpr (SPLIT > 1) {
        if (split)
#pragma unroll
            for (int b = 0; b < kMB * kNB; ++b)
#pragma unroll
                for (int g = 0; g < 4; ++g)
                    *(int4_t *)(stages + ((wave * kMB * kNB + b) * 4 + g) * 1024 + lane * 16) =
                        int4_t{acc[b / kNB][b % kNB][4 * g], acc[b / kNB][b % kNB][4 * g + 1],
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
                    const int4_t v = *(const int4_t *)(stages + s * kStages * kStageBytes +
                                                       ((wave * kMB * kNB + b) * 4 + g) * 1024 +
                                                       lane * 16);
#pragma unroll
                    for (int r = 0; r < 4; ++r)
                        acc[b / kNB][b % kNB][4 * g + r] += v[r];
                }
    }

    int8_t *mine = lds + wave * 32 * kPitch;
    const int64_t wave_m = m0 + wm * (TM / WM), wave_n = n0 + wn * (TN / WN);
    constexpr int kEach = 16 / sizeof(TO), kLanes = kNB * 32 / kEach;       // lanes per output row
#pragma unroll
    for (int i = 0; i < kMB; ++i) {
        const int64_t m = wave_m + i * 32 + frow;
        const float scale_a = QUANT ? scale_q[wm * (TM / WM) + i * 32 + frow]
                                    : p.a_scales[min(m, p.m - 1)];
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
                    // Past the caches, which then keep a and b: 8,192 x 16,384 x 4,096 500 us, 543
                    // with other stores.
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

// Few results: the weights' bytes are the work, and the way to fast ones is many loads in flight. A
// workgroup has 16 x 16 results and its 8 wavefronts share out k, in slabs of 256 bytes; fragments come
// from memory to registers as the matrix instruction takes them (lane l: row l % 16). The sum over k
// may take its products in any order, so lane l's four pieces of a slab are 64 bytes in a row, and
// four lanes read 256. The wavefronts' sums meet in LDS.
//
// QUANT: the rows of a (at most 16) are quantised from x in the kernel, by every workgroup again: a few
// KiB from L2 on the weights' way, against a launch of their own.
template <typename TO, bool QUANT>
__global__ __launch_bounds__(64 * kSkinnyWaves) void skinny_kernel(ProductArgs p, LinearArgs x) {
    constexpr int kSlab = 256, kT = 64 * kSkinnyWaves;
    extern __shared__ __attribute__((aligned(16))) int8_t quantized[];     // rows of k + 16 bytes
    __shared__ __attribute__((aligned(16))) int part[kSkinnyWaves][256];
    __shared__ uint32_t most[16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t tiles_n = (uint32_t)((p.n + 15) / 16);
    const int64_t m0 = (int64_t)(blockIdx.x / tiles_n) * 16, n0 = (int64_t)(blockIdx.x % tiles_n) * 16;
    const int k = (int)p.k, piece = (lane >> 4) * 64, rows = (int)min(p.m - m0, (int64_t)16);
    const int8_t *b = p.b + min(n0 + (lane & 15), p.n - 1) * p.b_stride;
    const int8_t *a = QUANT ? quantized + min(lane & 15, rows - 1) * (k + 16)
                            : p.a + (m0 + min(lane & 15, rows - 1)) * p.a_stride;
    int4_t fb[4], fa[4];
    // Pieces past k repeat the row's first ones; those of a count as zeros.
    auto read = [&](const int8_t *from, int4_t (&f)[4], int k0) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int at = k0 + piece + c * 16;
            f[c] = *(const int4_t *)(from + (at < k ? at : 0));
        }
    };
    int4_t acc = {};
    const int first = wave * kSlab;
    if (first < k)
        read(b, fb, first);
    if constexpr (QUANT) {
        if (threadIdx.x < 16)
            most[threadIdx.x] = 0;
        __syncthreads();
        const int blocks = blocks_of(x.cols), padded = k / kCols;
        auto value = [&](int row, int block) {
            const TO *from = (const TO *)((const char *)x.x + row * x.x_stride) + block * kCols;
            const int count = x.cols - block * kCols;
            return count >= kCols ? load_block(from) : load_block(from, count);
        };
        for (int row = 0; row < rows; ++row) {
            uint32_t top = 0;
            for (int block = threadIdx.x; block < blocks; block += kT)
                top = max(top, top_of(value(row, block)));
            top = wave_max<64>(top);
            if (lane == 0)
                atomicMax(&most[row], top);
        }
        __syncthreads();
        for (int row = 0; row < rows; ++row) {
            const RowScale s = row_scale(most[row]);
            for (int block = threadIdx.x; block < padded; block += kT)
                *(uint64_t *)(quantized + row * (k + 16) + block * kCols) =
                    eight_bits(value(row, block), s);
        }
        __syncthreads();
    }
    for (int k0 = first; k0 < k; k0 += kSkinnyWaves * kSlab) {
        if (k0 != first)
            read(b, fb, k0);
        read(a, fa, k0);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            if (k0 + piece + c * 16 >= k)
                fa[c] = int4_t{};
            acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[c], fa[c], acc, 0, 0, 0);
        }
    }
    *(int4_t *)&part[wave][lane * 4] = acc;
    __syncthreads();
    // Lane l's register r: row l % 16, column 4 (l / 16) + r.
    if (threadIdx.x < 256) {
        const int row = threadIdx.x >> 4, col = threadIdx.x & 15;
        int sum = 0;
#pragma unroll
        for (int w = 0; w < kSkinnyWaves; ++w)
            sum += part[w][((col >> 2) * 16 + row) * 4 + (col & 3)];
        const int64_t m = m0 + row, n = n0 + col;
        if (m < p.m && n < p.n) {
            const float scale_a = QUANT ? row_scale(most[row]).scale : p.a_scales[m];
            ((TO *)((char *)p.out + m * p.out_stride))[n] =
                (TO)finish(sum, scale_a, p.b_scales[n], p.bias ? p.bias[n] : 0.0f, p.relu);
        }
    }
}

template <typename TO, int TM, int TN, int WM, int WN, int SPLIT, int STAGES = 4,
          bool QUANT = false>
hipError_t launch_tiles(const ProductArgs &p, hipStream_t stream, const LinearArgs &x = {}) {
    const int64_t tm = (p.m + TM - 1) / TM, tn = (p.n + TN - 1) / TN;
    if (tm * tn * (64 * WM * WN * SPLIT) > (int64_t)UINT32_MAX)
        return hipErrorInvalidConfiguration;
    tile_kernel<TO, TM, TN, WM, WN, SPLIT, STAGES, QUANT>
        <<<(unsigned)(tm * tn), 64 * WM * WN * SPLIT, 0, stream>>>(p, (uint32_t)tm, (uint32_t)tn, x);
    return hipGetLastError();
}

template <typename TO, bool QUANT>
hipError_t launch_skinny(const ProductArgs &p, const LinearArgs &x, hipStream_t stream) {
    const int64_t tiles = tiles_of(p.m, p.n, 16, 16);
    skinny_kernel<TO, QUANT><<<(unsigned)tiles, 64 * kSkinnyWaves, QUANT ? p.m * (p.k + 16) : 0,
                               stream>>>(p, x);
    return hipGetLastError();
}

template <typename TO>
hipError_t launch_product_type(const ProductArgs &p, hipStream_t stream) {
    switch (product_choice(p.m, p.n, p.k)) {
    case kSkinny: return launch_skinny<TO, false>(p, LinearArgs{}, stream);
    case kTile64: return launch_tiles<TO, 64, 64, 2, 2, 4>(p, stream);
    case kTile128x64: return launch_tiles<TO, 128, 64, 2, 2, 2>(p, stream);
    case kTile128Split: return launch_tiles<TO, 128, 128, 2, 2, 2>(p, stream);
    case kTileShort: return launch_tiles<TO, 128, 128, 2, 2, 1, 2>(p, stream);
    case kTile128: return launch_tiles<TO, 128, 128, 2, 2, 1>(p, stream);
    default: return launch_tiles<TO, 256, 256, 2, 4, 1>(p, stream);
    }
}

template <typename T>
hipError_t launch_linear_type(const LinearArgs &x, const ProductArgs &p, hipStream_t stream) {
    if (quantize_inside(p.m, p.n, p.k))
        return launch_skinny<T, true>(p, x, stream);
    if (quantize_in_tile(p.m, p.n, p.k))
        return launch_tiles<T, 128, 128, 2, 2, 1, 2, true>(p, stream, x);
    const QuantizeArgs q{x.x, x.q, x.scales, x.x_stride, p.a_stride, p.m, x.cols, x.type};
    launch_quantize_type<T>(q, stream);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? launch_product_type<T>(p, stream) : e;
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

hipError_t launch_linear(const LinearArgs &x, const ProductArgs &p, hipStream_t stream) {
    switch (x.type) {
    case kF32: return launch_linear_type<float>(x, p, stream);
    case kF16: return launch_linear_type<half_t>(x, p, stream);
    default: return launch_linear_type<bf16_t>(x, p, stream);
    }
}

hipError_t launch_product(const ProductArgs &p, hipStream_t stream) {
    switch (p.out_type) {
    case kF32: return launch_product_type<float>(p, stream);
    case kF16: return launch_product_type<half_t>(p, stream);
    default: return launch_product_type<bf16_t>(p, stream);
    }
}

}  // namespace ccj

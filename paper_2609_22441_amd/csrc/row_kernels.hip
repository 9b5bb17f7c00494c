// Rows in, rows out: embedding lookup (rows of a table by id, scaled) and dropout, alone or on the
// looked-up rows.
//
// Per element one product and, with dropout, one comparison of 16 random bits: both operators are
// bound by the bytes they move. A thread takes one block of 8 columns: 16 or 32 contiguous bytes
// each way, and the eight numbers of one draw of the generator, whose counter is (row, block), so
// no thread draws bits that another one needs. Blocks are numbered through the rows, so that
// rows of any width fill the wavefronts; the row of a block is a division by the launch's blocks
// per row, done as a multiplication.
#include "layers_device.h"

namespace ccj {
namespace {

constexpr int kRowThreads = 256;
constexpr int64_t kRowGrid = 1 << 20;             // workgroups at most; each then takes several tiles

struct RowLaunch {
    RowArgs a;
    Divider div;
    int32_t blocks;                               // per row
    int64_t tiles;
};

struct NoIds {};

// ID: int32_t, int64_t, or NoIds (row t's source is row t). TAIL: cols is not a multiple of 8. U:
// blocks per thread, whose loads are in flight together.
template <typename TI, typename TO, typename ID, bool DROP, bool RES, bool TAIL, int U>
__global__ __launch_bounds__(kRowThreads) void row_kernel(RowLaunch l) {
    const RowArgs &a = l.a;
    constexpr bool kIds = !__is_same(ID, NoIds);
    for (int64_t tile = blockIdx.x; tile < l.tiles; tile += gridDim.x) {
        const int64_t first = tile * (kRowThreads * U);
        const int64_t row0 = first < UINT32_MAX ? (int64_t)((uint32_t)first / (uint32_t)l.blocks)
                                                : first / l.blocks;
        const uint32_t rem = (uint32_t)(first - row0 * l.blocks);
        int64_t row[U], src[U];
        uint32_t block[U];
        bool live[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t local = rem + threadIdx.x + u * kRowThreads;
            const uint32_t r = l.div(local);
            row[u] = row0 + r;
            block[u] = local - r * l.blocks;
            live[u] = row[u] < a.n;
            src[u] = row[u];
            if constexpr (kIds)
                src[u] = live[u] ? (int64_t)static_cast<const ID *>(a.ids)[row[u]] : -1;
        }
        Raw<TI> x[U];
        Raw<TO> res[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int col = block[u] * kCols;
            const bool read = kIds ? src[u] >= 0 && src[u] < a.src_rows : live[u];
            x[u] = Raw<TI>{};
            if (read) {
                const TI *p = (const TI *)((const char *)a.src + src[u] * a.src_stride) + col;
                if (TAIL && col + kCols > a.cols)
                    x[u] = load_block(p, a.cols - col);
                else
                    x[u] = load_block(p);
            }
            if (RES && live[u]) {
                const TO *p = (const TO *)((const char *)a.res + row[u] * a.res_stride) + col;
                if (TAIL && col + kCols > a.cols)
                    res[u] = load_block(p, a.cols - col);
                else
                    res[u] = load_block(p);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (!live[u])
                continue;
            const int col = block[u] * kCols;
            float y[kCols];
            Bits bits;
            if (DROP)
                bits = draw_bits(a.mask, row[u], block[u]);
#pragma unroll
            for (int i = 0; i < kCols; ++i) {
                y[i] = (float)x[u].v[i] * a.factor;
                if (DROP)
                    y[i] = bits.kept(i, a.mask.threshold) ? y[i] : 0.0f;
                if (RES)
                    y[i] += (float)res[u].v[i];
            }
            TO *p = (TO *)((char *)a.out + row[u] * a.out_stride) + col;
            if (TAIL && col + kCols > a.cols)
                store_block(p, y, a.cols - col);
            else
                store_block(p, y);
        }
    }
}

template <typename TI, typename TO, typename ID, bool DROP, bool RES, bool TAIL>
hipError_t launch_tail(const RowArgs &a, hipStream_t stream) {
    const int blocks = blocks_of(a.cols);
    const int64_t total = a.n * blocks;
    // One block per thread until the chip is full, then four.
    const bool small = total < (int64_t)1 << 19;
    const int64_t per = (int64_t)kRowThreads * (small ? 1 : 4);
    RowLaunch l{a, Divider(blocks), blocks, (total + per - 1) / per};
    const dim3 grid((unsigned)(l.tiles < kRowGrid ? l.tiles : kRowGrid));
    if (small)
        row_kernel<TI, TO, ID, DROP, RES, TAIL, 1><<<grid, kRowThreads, 0, stream>>>(l);
    else
        row_kernel<TI, TO, ID, DROP, RES, TAIL, 4><<<grid, kRowThreads, 0, stream>>>(l);
    return hipGetLastError();
}

template <typename TI, typename TO, typename ID, bool DROP, bool RES>
hipError_t launch_drop(const RowArgs &a, hipStream_t stream) {
    return a.cols % kCols ? launch_tail<TI, TO, ID, DROP, RES, true>(a, stream)
                          : launch_tail<TI, TO, ID, DROP, RES, false>(a, stream);
}

template <typename TI, typename TO>
hipError_t launch_lookup(const RowArgs &a, hipStream_t stream) {
    const bool drop = a.mask.threshold != kThresholdOne;
    if (a.id_bytes == 4)
        return drop ? launch_drop<TI, TO, int32_t, true, false>(a, stream)
                    : launch_drop<TI, TO, int32_t, false, false>(a, stream);
    return drop ? launch_drop<TI, TO, int64_t, true, false>(a, stream)
                : launch_drop<TI, TO, int64_t, false, false>(a, stream);
}

template <typename T>
hipError_t launch_dropout(const RowArgs &a, hipStream_t stream) {
    return a.res ? launch_drop<T, T, NoIds, true, true>(a, stream)
                 : launch_drop<T, T, NoIds, true, false>(a, stream);
}

}  // namespace

hipError_t launch_rows(const RowArgs &a, hipStream_t stream) {
    if (!a.ids) {
        switch (a.src_type) {
        case kF32: return launch_dropout<float>(a, stream);
        case kF16: return launch_dropout<half_t>(a, stream);
        default: return launch_dropout<bf16_t>(a, stream);
        }
    }
    if (a.src_type == kF32)
        switch (a.out_type) {
        case kF32: return launch_lookup<float, float>(a, stream);
        case kF16: return launch_lookup<float, half_t>(a, stream);
        default: return launch_lookup<float, bf16_t>(a, stream);
        }
    return a.src_type == kF16 ? launch_lookup<half_t, half_t>(a, stream)
                              : launch_lookup<bf16_t, bf16_t>(a, stream);
}

}  // namespace ccj

// Rows in, rows out: embedding lookup (rows of a table by id, scaled) and dropout, alone or on the
// looked-up rows.
//
// Per element one product and, with dropout, one comparison of 16 random bits: both operators are
// bound by the bytes they move. A thread takes one block of 8 columns: 16 or 32 contiguous bytes
// each way, and the eight numbers of one draw of the generator, whose counter is (row, block), so
// no thread draws bits that another one needs. Blocks are numbered through the rows, so that
// rows of any width fill the wavefronts; the row of a block is a division by the launch's blocks
// per row, done as a multiplication.
//
// Dropout with residual, 131,072 x 4,096 bf16: 483 us, 3.2 GB at 6.7 TB/s. Lookup of as many rows of a
// table of that size with Zipf frequencies, with dropout: 278 us, 1.07 GB written and as much read, all but
// 0.2 GB of it from the caches; without dropout 265, so the generator is not what bounds it. 64 rows of
// 1,024: 5 us, the launch.
#include "layers_device.h"

namespace ccj {
namespace {

constexpr int kRowThreads = 256;
constexpr int64_t kRowGrid = 1 << 20;             // workgroups at most; each then takes several tiles

constexpr int kWideBlocks = 64;

struct RowLaunch {
    RowArgs a;
    Divider div;
    int32_t blocks;                               // per row
    int32_t segments;                             // of 64 blocks, per row (wide rows)
    bool by_segment;
    int64_t tiles;
};

struct NoIds {};

template <bool DROP, bool RES, typename TI, typename TO>
__device__ __forceinline__ void row_values(const RowArgs &a, const Raw<TI> &x, const Raw<TO> &res,
                                           int64_t row, uint32_t block, bool found,
                                           float (&y)[kCols]) {
    Bits bits;
    if (DROP)
        bits = draw_bits(a.mask, row, block);
#pragma unroll
    for (int i = 0; i < kCols; ++i) {
        const bool keep = DROP ? found && bits.kept(i, a.mask.threshold) : found;
        y[i] = keep ? (float)x[i] * a.factor : 0.0f;
        if (RES)
            y[i] += (float)res[i];
    }
}

// ID: int32_t, int64_t, or NoIds (row t's source is row t). TAIL: cols is not a multiple of 8, or a
// matrix not aligned to 16 bytes. U: blocks per thread, whose loads are in flight together.
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
        bool found[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t local = rem + threadIdx.x + u * kRowThreads;
            const uint32_t r = l.div(local);
            row[u] = row0 + r;
            block[u] = local - r * l.blocks;
            src[u] = min(row[u], a.n - 1);
            found[u] = true;
            if constexpr (kIds) {
                src[u] = static_cast<const ID *>(a.ids)[src[u]];
                found[u] = src[u] >= 0 && src[u] < a.src_rows;
                src[u] = found[u] ? src[u] : 0;
            }
        }
        Raw<TI> x[U];
        Raw<TO> res[U];
        int exchange[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int col = block[u] * kCols;
            // Lanes 4 or 8 i on are in one row where its blocks are a multiple of 4 or 8, and then all
            // here: a tile starts at a multiple of 8 blocks as well.
            exchange[u] = TAIL || l.blocks % 4 ? kAlone : l.blocks % 8 ? kFour : kEight;
            x[u] = load_most<TAIL, !kIds>((const TI *)((const char *)a.src + src[u] * a.src_stride), col,
                                   a.cols, exchange[u]);
            if (RES)
                res[u] = load_most<TAIL, true>(
                    (const TO *)((const char *)a.res + min(row[u], a.n - 1) * a.res_stride), col,
                    a.cols, exchange[u]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (row[u] >= a.n)
                continue;
            const int col = block[u] * kCols;
            load_rest<TAIL>(x[u], (const TI *)((const char *)a.src + src[u] * a.src_stride), col,
                            a.cols, exchange[u]);
            if (RES)
                load_rest<TAIL>(res[u], (const TO *)((const char *)a.res + row[u] * a.res_stride),
                                col, a.cols, exchange[u]);
            float y[kCols];
            row_values<DROP, RES>(a, x[u], res[u], row[u], block[u], found[u], y);
            TO *p = (TO *)((char *)a.out + row[u] * a.out_stride) + col;
            if (TAIL && col + kCols > a.cols)
                store_block(p, y, a.cols - col);
            else if (TAIL)
                store_block(p, y);
            else
                stream_block(p, y, exchange[u]);
        }
    }
}

// The same for rows of kWideBlocks blocks or more: a wavefront takes 64 blocks of U rows, so that
// rows, ids and addresses are the wavefront's (scalar) and a lane keeps its columns. Four wavefronts
// of a workgroup take segments that follow each other; where the rows are read in order and have a
// multiple of 8 segments, rows that follow each other of one segment, so that each XCD reads and
// writes one segment of all rows: 485 us against 520 (dropout and residual, 131,072 x 4,096 bf16). For
// looked-up rows it is 282 against 277, and with 2 segments (1,000 columns) 73 against 53.
template <typename TI, typename TO, typename ID, bool DROP, bool RES, bool TAIL, int U>
__global__ __launch_bounds__(kRowThreads) void wide_kernel(RowLaunch l) {
    const RowArgs &a = l.a;
    constexpr bool kIds = !__is_same(ID, NoIds);
    for (int64_t tile = blockIdx.x; tile < l.tiles; tile += gridDim.x) {
        const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        // Segment and group of U rows: wavefront by wavefront, or workgroup by workgroup.
        const uint32_t number = l.by_segment ? (uint32_t)tile
                                             : (uint32_t)tile * (kRowThreads / 64) + wave;
        const uint32_t round = l.div(number);
        const uint32_t block = (number - round * l.segments) * 64 + (threadIdx.x & 63);
        const int64_t row0 = (l.by_segment ? (int64_t)round * (kRowThreads / 64) + wave : round) * U;
        if (row0 >= a.n || block >= (uint32_t)l.blocks)
            continue;
        const int col = block * kCols;
        const int exchange = exchange_of(block, a.cols);
        int64_t src[U];
        const TI *from[U];
        bool found[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            src[u] = min(row0 + u, a.n - 1);
            if constexpr (kIds)
                src[u] = constant<ID>(a.ids)[src[u]];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            found[u] = !kIds || (src[u] >= 0 && src[u] < a.src_rows);
            from[u] = (const TI *)((const char *)a.src + (found[u] ? src[u] : 0) * a.src_stride);
        }
        Raw<TI> x[U];
        Raw<TO> res[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            x[u] = load_most<TAIL, !kIds>(from[u], col, a.cols, exchange);
            if (RES)
                res[u] = load_most<TAIL, true>(
                    (const TO *)((const char *)a.res + min(row0 + u, a.n - 1) * a.res_stride), col,
                    a.cols, exchange);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t row = row0 + u;
            if (row >= a.n)
                break;
            load_rest<TAIL>(x[u], from[u], col, a.cols, exchange);
            if (RES)
                load_rest<TAIL>(res[u], (const TO *)((const char *)a.res + row * a.res_stride), col,
                                a.cols, exchange);
            float y[kCols];
            row_values<DROP, RES>(a, x[u], res[u], row, block, found[u], y);
            TO *p = (TO *)((char *)a.out + row * a.out_stride) + col;
            if (TAIL && col + kCols > a.cols)
                store_block(p, y, a.cols - col);
            else if (TAIL)
                store_block(p, y);
            else
                stream_block(p, y, exchange);
        }
    }
}

template <typename TI, typename TO, typename ID, bool DROP, bool RES, bool TAIL>
hipError_t launch_tail(const RowArgs &a, hipStream_t stream) {
    const int blocks = blocks_of(a.cols);
    const int64_t total = a.n * blocks;
    if (blocks >= kWideBlocks && total >= (int64_t)1 << 19) {
        const int segments = (blocks + 63) / 64;
        constexpr int kRows = 2;
        const bool by_segment = __is_same(ID, NoIds) && segments % 8 == 0;
        const int64_t groups = (a.n + kRows - 1) / kRows;
        const int64_t tiles = by_segment ? (groups + 3) / 4 * segments : (groups * segments + 3) / 4;
        RowLaunch l{a, Divider(segments), blocks, segments, by_segment, tiles};
        const dim3 grid((unsigned)(l.tiles < kRowGrid ? l.tiles : kRowGrid));
        wide_kernel<TI, TO, ID, DROP, RES, TAIL, kRows><<<grid, kRowThreads, 0, stream>>>(l);
        return hipGetLastError();
    }
    // One block per thread until the chip is full, then four.
    const bool small = total < (int64_t)1 << 19;
    const int64_t per = (int64_t)kRowThreads * (small ? 1 : 4);
    RowLaunch l{a, Divider(blocks), blocks, 0, false, (total + per - 1) / per};
    const dim3 grid((unsigned)(l.tiles < kRowGrid ? l.tiles : kRowGrid));
    if (small)
        row_kernel<TI, TO, ID, DROP, RES, TAIL, 1><<<grid, kRowThreads, 0, stream>>>(l);
    else
        row_kernel<TI, TO, ID, DROP, RES, TAIL, 4><<<grid, kRowThreads, 0, stream>>>(l);
    return hipGetLastError();
}

template <typename TI, typename TO, typename ID, bool DROP, bool RES>
hipError_t launch_drop(const RowArgs &a, hipStream_t stream) {
    const bool even = a.cols % kCols == 0 && even_rows(a.src, a.src_stride) &&
                      even_rows(a.out, a.out_stride) && (!RES || even_rows(a.res, a.res_stride));
    return even ? launch_tail<TI, TO, ID, DROP, RES, false>(a, stream)
                : launch_tail<TI, TO, ID, DROP, RES, true>(a, stream);
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

hipError_t launch_rows(const RowArgs &args, hipStream_t stream) {
    RowArgs a = args;
    if (a.ids && a.src_rows == 0) {
        // No id is found: rows of zeros, as a dropout that drops everything writes in place.
        a.src = a.out;
        a.src_stride = a.out_stride;
        a.src_type = a.out_type;
        a.ids = nullptr;
        a.mask.threshold = 0;
    }
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

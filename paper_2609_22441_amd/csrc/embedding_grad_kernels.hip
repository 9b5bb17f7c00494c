// Gradient of an embedding lookup: the output gradient's rows, summed by id.
//
// The sum over the tokens of one id needs either atomic additions, whose order and so whose result
// changes from run to run, or the tokens in order of their ids. Here (id, token) pairs are sorted
// (stable, least significant digit first; an id outside the table sorts past its last row), and the
// rows are then read once each, in the order of the sorted pairs:
//
//   sum    the sorted tokens are cut into chunks of equal length, whatever the ids are, so that an
//          id that takes most of the tokens is shared out as evenly as ids that occur once. A group
//          of lanes adds a chunk's rows in 32 bits, run by run; a run that lies inside the chunk is
//          finished and written, one that crosses an edge of it is kept as a partial sum. Further
//          workgroups of the same launch write zeros into the rows that no id points at.
//   join   the partial sums of each run that crosses edges are added in the order of the chunks.
//
// The work is bound by the bytes of grad_out and grad_table: pairs are 8 bytes a token, partial
// sums at most 8 bytes a column of every chunk.
#include <algorithm>

#include "layers_device.h"

namespace ccj {
namespace {

// ---- sorted pairs ----

struct Pair {
    uint32_t key, token;
};

constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kMaxDigitBits = 9;
constexpr int kMaxDigits = 1 << kMaxDigitBits;
constexpr int kMinTile = 2048;          // pairs per workgroup of a digit pass
constexpr int kMaxTiles = 256;          // every workgroup reads the counts of all tiles
constexpr int64_t kMaxChunks = 1 << 18; // chunks times column tiles: the joins' grid stays launchable

struct SortShape {
    int32_t passes, digit_bits;         // digit passes, bits of each
    int32_t tiles;
    int64_t tile;                       // pairs per tile, a multiple of kSortThreads
};

SortShape sort_shape(int64_t n, int64_t rows) {
    SortShape s;
    int bits = 1;
    while (rows >> bits)                // keys 0 to rows: the last is every id outside the table
        ++bits;
    s.passes = (bits + kMaxDigitBits - 1) / kMaxDigitBits;
    s.digit_bits = (bits + s.passes - 1) / s.passes;
    const int64_t even = (n + kMaxTiles - 1) / kMaxTiles;
    s.tile = std::max<int64_t>(kMinTile, (even + kSortThreads - 1) / kSortThreads * kSortThreads);
    s.tiles = (int32_t)((n + s.tile - 1) / s.tile);
    return s;
}

__device__ __forceinline__ uint32_t key_of(int64_t id, int64_t rows) {
    return (uint32_t)(id >= 0 && id < rows ? id : rows);
}

template <typename ID>
struct FromIds {
    const ID *ids;
    int64_t rows;
    __device__ Pair operator()(int64_t i) const {
        return Pair{key_of((int64_t)ids[i], rows), (uint32_t)i};
    }
};

struct FromPairs {
    const Pair *p;
    __device__ Pair operator()(int64_t i) const { return p[i]; }
};

// Counts of each digit value in every tile: counts[tile][digit].
template <typename Source>
__global__ __launch_bounds__(kSortThreads) void digit_counts(Source source, int64_t n, int64_t tile,
                                                             int shift, int digits,
                                                             uint32_t *counts) {
    __shared__ uint32_t hist[kMaxDigits];
    for (int d = threadIdx.x; d < digits; d += kSortThreads)
        hist[d] = 0;
    __syncthreads();
    const int64_t first = blockIdx.x * tile, last = min(n, first + tile);
    for (int64_t i = first + threadIdx.x; i < last; i += kSortThreads)
        atomicAdd(&hist[(source(i).key >> shift) & (digits - 1)], 1u);
    __syncthreads();
    for (int d = threadIdx.x; d < digits; d += kSortThreads)
        counts[(int64_t)blockIdx.x * digits + d] = hist[d];
}

// Exclusive prefix sum of `x` over threads 0 to `count` - 1 (a multiple of 64 or below 64), by the
// whole workgroup; `sums` is scratch.
__device__ __forceinline__ uint32_t prefix(uint32_t x, int count, uint32_t (&sums)[kSortWaves]) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t inclusive = x;
#pragma unroll
    for (int s = 1; s < 64; s <<= 1) {
        const uint32_t y = __shfl_up(inclusive, s);
        if (lane >= s)
            inclusive += y;
    }
    if (lane == 63)
        sums[wave] = inclusive;
    __syncthreads();
    uint32_t before = 0;
    for (int w = 0; w < wave && w * 64 < count; ++w)
        before += sums[w];
    __syncthreads();
    return before + inclusive - x;
}

// One digit pass: tile `blockIdx.x` moves its pairs to their places among all tiles' pairs of the
// digit, in their order. Each wavefront takes a contiguous part of the tile.
template <typename Source>
__global__ __launch_bounds__(kSortThreads) void digit_scatter(Source source, int64_t n,
                                                              int64_t tile, int shift,
                                                              int digit_bits,
                                                              const uint32_t *counts, int tiles,
                                                              Pair *out) {
    __shared__ uint32_t place[kSortWaves][kMaxDigits];     // next place of a digit, by wavefront
    __shared__ uint32_t part[2][kSortThreads];             // sums over some tiles: all, earlier ones
    __shared__ uint32_t sums[kSortWaves];
    const int digits = 1 << digit_bits;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int i = threadIdx.x; i < kSortWaves * digits; i += kSortThreads)
        place[i >> digit_bits][i & (digits - 1)] = 0;
    // Every thread adds up one digit's counts over a share of the tiles.
    const int shares = kSortThreads >> digit_bits;
    {
        const int d = threadIdx.x & (digits - 1), share = threadIdx.x >> digit_bits;
        uint32_t all = 0, earlier = 0;
#pragma unroll 8
        for (int t = share; t < tiles; t += shares) {
            const uint32_t c = counts[(int64_t)t * digits + d];
            all += c;
            earlier += t < (int)blockIdx.x ? c : 0;
        }
        part[0][threadIdx.x] = all;
        part[1][threadIdx.x] = earlier;
    }
    __syncthreads();
    // The wavefronts' own counts.
    const int64_t begin = blockIdx.x * tile, end = min(n, begin + tile);
    const int64_t span = (tile / kSortWaves + 63) / 64 * 64;
    const int64_t from = min(end, begin + wave * span), to = min(end, from + span);
    for (int64_t i = from + lane; i < to; i += 64)
        atomicAdd(&place[wave][(source(i).key >> shift) & (digits - 1)], 1u);
    uint32_t all = 0, earlier = 0;
    if ((int)threadIdx.x < digits)
        for (int s = 0; s < shares; ++s) {
            all += part[0][(s << digit_bits) + threadIdx.x];
            earlier += part[1][(s << digit_bits) + threadIdx.x];
        }
    const uint32_t start = prefix(all, digits, sums) + earlier;      // also a barrier
    if ((int)threadIdx.x < digits) {
        uint32_t next = start;
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t c = place[w][threadIdx.x];
            place[w][threadIdx.x] = next;
            next += c;
        }
    }
    __syncthreads();
    for (int64_t base = from; base < to; base += 64) {
        const int64_t i = base + lane;
        const bool live = i < to;
        const Pair p = live ? source(i) : Pair{0, 0};
        const uint32_t d = (p.key >> shift) & (digits - 1);
        // Lanes of the same digit value.
        uint64_t peers = __ballot(live);
        for (int b = 0; b < digit_bits; ++b) {
            const uint64_t set = __ballot((d >> b) & 1);
            peers &= ((d >> b) & 1) ? set : ~set;
        }
        const uint32_t rank = __popcll(peers & (((uint64_t)1 << lane) - 1));
        const uint32_t first = live ? place[wave][d] : 0;
        // The wavefront's reads of its counters come before the additions below, which come before
        // the next round's reads: LDS operations of one wavefront keep their order.
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (live && rank == 0)
            place[wave][d] = first + __popcll(peers);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (live)
            out[first + rank] = p;
    }
}

// ---- sums of runs ----

struct Runs {
    const Pair *pairs;
    float *partial;              // [chunks][2][width]: sums of the runs open at a chunk's start, end
    int64_t n, chunk, chunks;
    int32_t width;               // floats per partial row, a multiple of 8
    int32_t blocks;              // column blocks per row
    int32_t tiles;               // of 64 blocks or fewer each
};

template <typename T>
__device__ __forceinline__ void write_row(const GradArgs &a, uint32_t key, int col,
                                          const float (&sum)[kCols]) {
    T *p = (T *)((char *)a.table + (int64_t)key * a.table_stride) + col;
    const int count = min(kCols, a.cols - col);
    float y[kCols];
#pragma unroll
    for (int i = 0; i < kCols; ++i)
        y[i] = sum[i] * a.factor;
    if (a.accumulate) {
        const Raw<T> old = count == kCols ? load_block(p) : load_block(p, count);
#pragma unroll
        for (int i = 0; i < kCols; ++i)
            y[i] += (float)old[i];
    }
    if (count == kCols)
        store_block(p, y);
    else
        store_block(p, y, count);
}

// Workgroups [0, sum_groups) add up chunks, a group of L lanes per chunk and tile of L column
// blocks; the others write zeros into `strip` rows each.
template <typename TG, typename TT, int L, bool DROP, bool TAIL>
__global__ __launch_bounds__(256) void sum_kernel(GradArgs a, Runs r, int64_t sum_groups,
                                                  int strip) {
    if (blockIdx.x >= sum_groups) {
        __shared__ uint8_t empty[256];
        const int64_t row0 = (blockIdx.x - sum_groups) * strip;
        const int count = (int)min((int64_t)strip, a.rows - row0);
        if ((int)threadIdx.x < count) {
            const uint32_t key = (uint32_t)(row0 + threadIdx.x);
            int64_t lo = 0, hi = r.n;                  // the first pair whose key is not below
            while (lo < hi) {
                const int64_t mid = (lo + hi) >> 1;
                if (r.pairs[mid].key < key)
                    lo = mid + 1;
                else
                    hi = mid;
            }
            empty[threadIdx.x] = lo == r.n || r.pairs[lo].key != key;
        }
        __syncthreads();
        for (int64_t i = threadIdx.x; i < (int64_t)count * r.blocks; i += 256) {
            const int row = (int)(i / r.blocks), block = (int)(i - (int64_t)row * r.blocks);
            if (empty[row]) {
                TT *p = (TT *)((char *)a.table + (row0 + row) * a.table_stride) + block * kCols;
                const float zero[kCols] = {};
                if (TAIL && (block + 1) * kCols > a.cols)
                    store_block(p, zero, a.cols - block * kCols);
                else
                    store_block(p, zero);
            }
        }
        return;
    }
    constexpr int kAhead = 8;                  // rows in flight per lane
    const int64_t group = (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L;
    const int64_t c = group / r.tiles;
    const int block = (int)(group - c * r.tiles) * L + (int)(threadIdx.x % L);
    if (c >= r.chunks || block >= r.blocks)
        return;
    const int col = block * kCols;
    const int64_t i0 = c * r.chunk, i1 = min(r.n, i0 + r.chunk);
    const bool head = i0 > 0 && r.pairs[i0 - 1].key == r.pairs[i0].key;
    const bool tail = i1 < r.n && r.pairs[i1].key == r.pairs[i1 - 1].key;
    uint32_t current = r.pairs[i0].key;
    bool first = true;
    float sum[kCols] = {};
    auto finish = [&](bool open) {
        if (current < (uint64_t)a.rows) {
            if (open)
                store_block(r.partial + (c * 2 + (first && head ? 0 : 1)) * r.width + col, sum);
            else
                write_row<TT>(a, current, col, sum);
        }
    };
    for (int64_t i = i0; i < i1 && r.pairs[i].key < (uint64_t)a.rows; i += kAhead) {
        Pair p[kAhead];
        Raw<TG> x[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            p[j] = r.pairs[min(i + j, i1 - 1)];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const TG *g = (const TG *)((const char *)a.grad + (int64_t)p[j].token * a.grad_stride) +
                          col;
            if (TAIL && col + kCols > a.cols)
                x[j] = load_block(g, a.cols - col);
            else
                x[j] = load_block(g);
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (i + j >= i1)
                break;
            if (p[j].key != current) {
                finish(first && head);
                current = p[j].key;
                first = false;
#pragma unroll
                for (int k = 0; k < kCols; ++k)
                    sum[k] = 0.0f;
            }
            Bits bits;
            if (DROP)
                bits = draw_bits(a.mask, p[j].token, block);
#pragma unroll
            for (int k = 0; k < kCols; ++k) {
                const float v = (float)x[j][k];
                sum[k] += !DROP || bits.kept(k, a.mask.threshold) ? v : 0.0f;
            }
        }
    }
    finish((first && head) || tail);
}

// A workgroup per chunk and tile of L column blocks: where a run starts in the chunk and goes on
// past its end, adds up the run's partial sums. Lane groups take every (256 / L)-th chunk of the
// run, and the first adds their sums in order.
template <typename TT, int L>
__global__ __launch_bounds__(256) void join_kernel(GradArgs a, Runs r) {
    constexpr int kGroups = 256 / L;
    const int64_t c = blockIdx.x / r.tiles;
    const int64_t i0 = c * r.chunk, i1 = min(r.n, i0 + r.chunk);
    const uint32_t key = r.pairs[i1 - 1].key;
    const bool goes_on = i1 < r.n && r.pairs[i1].key == key && key < (uint64_t)a.rows;
    const bool starts = i0 == 0 || r.pairs[i0].key != key || r.pairs[i0 - 1].key != key;
    if (!goes_on || !starts)
        return;
    int64_t lo = i1, hi = r.n;                         // the first pair past the run
    while (lo < hi) {
        const int64_t mid = (lo + hi) >> 1;
        if (r.pairs[mid].key <= key)
            lo = mid + 1;
        else
            hi = mid;
    }
    const int64_t end = (lo - 1) / r.chunk;            // the run's last chunk
    const int lane = threadIdx.x % L, group = threadIdx.x / L;
    const int block = (int)(blockIdx.x - c * r.tiles) * L + lane;
    const int col = block * kCols;
    float sum[kCols] = {};
    if (block < r.blocks)
        for (int64_t d = c + group; d <= end; d += kGroups) {
            // The run is open at its first chunk's end and at the later ones' start.
            const Raw<float> x = load_block(r.partial + (d * 2 + (d == c ? 1 : 0)) * r.width + col);
#pragma unroll
            for (int k = 0; k < kCols; ++k)
                sum[k] += x[k];
        }
    __shared__ float part[256][kCols + 1];
#pragma unroll
    for (int k = 0; k < kCols; ++k)
        part[threadIdx.x][k] = sum[k];
    __syncthreads();
    if (group == 0 && block < r.blocks) {
        for (int g = 1; g < kGroups; ++g)
#pragma unroll
            for (int k = 0; k < kCols; ++k)
                sum[k] += part[g * L + lane][k];
        write_row<TT>(a, key, col, sum);
    }
}

// ---- layout of the workspace ----

int64_t round16(int64_t x) { return (x + 15) & ~(int64_t)15; }

struct Plan {
    SortShape sort;
    int64_t chunk, chunks;
    int32_t lanes, tiles, width;
    int64_t counts, pairs0, pairs1, partial, bytes;      // offsets and the total size
};

Plan plan(int64_t n, int64_t rows, int32_t cols) {
    Plan p = {};
    p.sort = sort_shape(n, rows);
    const int blocks = blocks_of(cols);
    p.lanes = blocks <= 4 ? 4 : blocks <= 16 ? 16 : 64;
    p.tiles = (blocks + p.lanes - 1) / p.lanes;
    p.width = blocks * kCols;
    // Chunks of 64 tokens, in which the partial sums are at most 1/16 of 16-bit rows' bytes (1/32 of
    // 32-bit ones'); shorter ones while the chip has fewer than 4 wavefronts per SIMD of them.
    p.chunk = 64;
    while (p.chunk > 8 && n / p.chunk * p.tiles * p.lanes < 4 * 1024 * 64)
        p.chunk /= 2;
    while (n / p.chunk * p.tiles > kMaxChunks)
        p.chunk *= 2;
    p.chunks = (n + p.chunk - 1) / p.chunk;
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t here = at;
        at += round16(bytes);
        return here;
    };
    p.counts = take((int64_t)p.sort.tiles << p.sort.digit_bits << 2);
    p.pairs0 = take(n * (int64_t)sizeof(Pair));
    p.pairs1 = take(p.sort.passes > 1 ? n * (int64_t)sizeof(Pair) : 0);
    p.partial = take(p.chunks * 2 * p.width * 4);
    p.bytes = at;
    return p;
}

template <typename Source>
void launch_pass(Source source, const Plan &p, int64_t n, int pass, uint32_t *counts, Pair *out,
                 hipStream_t stream) {
    const int shift = pass * p.sort.digit_bits;
    digit_counts<<<p.sort.tiles, kSortThreads, 0, stream>>>(source, n, p.sort.tile, shift,
                                                            1 << p.sort.digit_bits, counts);
    digit_scatter<<<p.sort.tiles, kSortThreads, 0, stream>>>(source, n, p.sort.tile, shift,
                                                             p.sort.digit_bits, counts,
                                                             p.sort.tiles, out);
}

template <typename TG, typename TT, int L, bool DROP, bool TAIL>
void launch_sum(const GradArgs &a, const Runs &r, hipStream_t stream) {
    const int64_t sum_groups = (r.chunks * r.tiles + 256 / L - 1) / (256 / L);
    // Strips of rows of about 64 KiB.
    const int64_t row_bytes = (int64_t)a.cols * sizeof(TT);
    const int strip = (int)std::max<int64_t>(1, std::min<int64_t>(256, 65536 / row_bytes));
    const int64_t strips = a.accumulate ? 0 : (a.rows + strip - 1) / strip;
    if (sum_groups + strips > 0)
        sum_kernel<TG, TT, L, DROP, TAIL><<<(unsigned)(sum_groups + strips), 256, 0, stream>>>(
            a, r, sum_groups, strip);
    if (r.chunks > 1)
        join_kernel<TT, L><<<(unsigned)(r.chunks * r.tiles), 256, 0, stream>>>(a, r);
}

template <typename TG, typename TT, int L>
void launch_drop(const GradArgs &a, const Runs &r, hipStream_t stream) {
    const bool drop = a.mask.threshold != kThresholdOne, tail = a.cols % kCols;
    if (drop)
        tail ? launch_sum<TG, TT, L, true, true>(a, r, stream)
             : launch_sum<TG, TT, L, true, false>(a, r, stream);
    else
        tail ? launch_sum<TG, TT, L, false, true>(a, r, stream)
             : launch_sum<TG, TT, L, false, false>(a, r, stream);
}

template <typename TG, typename TT>
void launch_lanes(const GradArgs &a, const Runs &r, int lanes, hipStream_t stream) {
    if (lanes == 4)
        launch_drop<TG, TT, 4>(a, r, stream);
    else if (lanes == 16)
        launch_drop<TG, TT, 16>(a, r, stream);
    else
        launch_drop<TG, TT, 64>(a, r, stream);
}

}  // namespace

int64_t grad_workspace_bytes(int64_t n, int64_t rows, int32_t cols) {
    return plan(n, rows, cols).bytes;
}

hipError_t launch_embedding_grad(const GradArgs &a, hipStream_t stream) {
    const Plan p = plan(a.n, a.rows, a.cols);
    char *ws = static_cast<char *>(a.workspace);
    uint32_t *counts = (uint32_t *)(ws + p.counts);
    Pair *pairs[2] = {(Pair *)(ws + p.pairs0), (Pair *)(ws + p.pairs1)};
    for (int pass = 0; a.n > 0 && pass < p.sort.passes; ++pass) {
        Pair *out = pairs[pass & 1];
        if (pass)
            launch_pass(FromPairs{pairs[(pass - 1) & 1]}, p, a.n, pass, counts, out, stream);
        else if (a.id_bytes == 4)
            launch_pass(FromIds<int32_t>{(const int32_t *)a.ids, a.rows}, p, a.n, 0, counts, out,
                        stream);
        else
            launch_pass(FromIds<int64_t>{(const int64_t *)a.ids, a.rows}, p, a.n, 0, counts, out,
                        stream);
    }
    const Runs r{pairs[(p.sort.passes - 1) & 1], (float *)(ws + p.partial), a.n, p.chunk, p.chunks,
                 p.width, blocks_of(a.cols), p.tiles};
    if (a.grad_type == kF32)
        launch_lanes<float, float>(a, r, p.lanes, stream);
    else if (a.grad_type == kF16 && a.table_type == kF32)
        launch_lanes<half_t, float>(a, r, p.lanes, stream);
    else if (a.grad_type == kF16)
        launch_lanes<half_t, half_t>(a, r, p.lanes, stream);
    else if (a.table_type == kF32)
        launch_lanes<bf16_t, float>(a, r, p.lanes, stream);
    else
        launch_lanes<bf16_t, bf16_t>(a, r, p.lanes, stream);
    return hipGetLastError();
}

}  // namespace ccj

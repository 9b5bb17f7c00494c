// Gradient of an embedding lookup: the output gradient's rows, summed by id.
//
// The sum over the tokens of one id needs either atomic additions, whose order and so whose result
// changes from run to run, or the tokens in order of their ids. Here (id, token) pairs are sorted
// (stable, least significant digit first; an id outside the table sorts past its last row), and the
// rows are then read once each, in the order of the sorted pairs:
//
//   sum    the sorted tokens are cut into chunks of equal length, whatever the ids are, so that an
//          id that takes most of the tokens is shared out as evenly as ids that occur once. A group
//          of lanes adds a chunk's rows in 32 bits, run by run, and writes each run's sum; a run that
//          ends inside the next chunk is added up to its end, and that chunk begins after it. Only of
//          a run that covers whole chunks does each of them keep a partial sum. Further workgroups of
//          the same launch write zeros into the rows that no id points at.
//   fold   the same once more, with the partial sums of kFold chunks in the tokens' place: an id with
//          all of a million tokens leaves tens of thousands of them. Left out where few are possible.
//   join   the partial sums of each run are added up by a workgroup, in the order of the chunks.
//
// The work is bound by the bytes of grad_out and grad_table: pairs are 8 bytes a token, and the partial
// sums are 4 bytes a column of chunks that one id covers. 131,072 tokens of 2,048 bf16 columns (dropout,
// Zipf frequencies) into 50,000 rows of 32 bits: 224 us for 946 MB, of them 180 in `sum` (5.3 TB/s), 25 in
// the sort, 22 in fold and join. Few tokens, and tables of few rows, are done another way, further down.
#include <algorithm>

#include "grad_choice.h"
#include "layers_device.h"

namespace ccj {
namespace {

static_assert(kGradBlock == kCols, "the choice counts the kernels' column blocks");

// ---- sorted pairs ----

constexpr int kSortWaves = kSortThreads / 64;
constexpr int kMaxDigits = 1 << kMaxDigitBits;
constexpr int kClearWords = 4 * kSortThreads;   // of 16 bytes, cleared by a workgroup

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

// Counts of each digit value in every tile: counts[tile][digit]. The first pass's launch has further
// workgroups that clear `found`, a byte for every row of the table, and empties the list of runs.
template <typename Source>
__global__ __launch_bounds__(kSortThreads) void digit_counts(Source source, int64_t n, int64_t tile,
                                                             int shift, int digits, int tiles,
                                                             uint32_t *counts, words_t *found,
                                                             int64_t found_words,
                                                             uint32_t *list_count) {
    if (list_count && blockIdx.x == 0 && threadIdx.x == 0)
        *list_count = 0;
    if ((int)blockIdx.x >= tiles) {
        const int64_t first = (int64_t)((int)blockIdx.x - tiles) * kClearWords;
        const int64_t last = min(found_words, first + kClearWords);
        for (int64_t i = first + threadIdx.x; i < last; i += kSortThreads)
            found[i] = words_t{};
        return;
    }
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
                                                              Pair *out, uint8_t *found) {
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
        if (live) {
            out[first + rank] = p;
            if (found)
                found[p.key] = 1;
        }
    }
}

// ---- sums of runs ----

constexpr int64_t kStripBytes = 128 << 10, kMaxStrips = 1 << 21;

struct Runs {
    const Pair *pairs;
    const uint8_t *found;        // [rows]: an id points at the row
    float *partial;              // [chunks][2][width]: sums of the runs open at a chunk's start, end
    int64_t n, chunk, chunks;
    int32_t width;               // floats per partial row, a multiple of 8
    int32_t blocks;              // column blocks per row
    int32_t tiles;               // of 64 blocks or fewer each
    int64_t whole;               // tokens of the chunks that the partial sums come from
    bool listed;                 // the sums list their runs (no fold after them)
    uint32_t *list;              // [0]: how many; then the chunks in which runs start that the join adds up
    // By the one lane of a chunk that speaks for it. The order of the list changes no result.
    __device__ void append(int64_t c) const { list[1 + atomicAdd(list, 1u)] = (uint32_t)c; }
    // How many of the `chunk` pairs from i on have the key, by all lanes of a wavefront, L of them for
    // one i: the pairs are sorted, and the first does or none.
    template <int L>
    __device__ int leading(int64_t i, uint32_t key) const {
        const int lane = threadIdx.x & 63, in = lane % L;
        int count = 0;
        for (int64_t j = in; j - in < chunk; j += L) {
            const uint64_t same = __ballot(j < chunk && i + j < n && pairs[min(i + j, n - 1)].key == key);
            count += __popcll(L == 64 ? same : same >> (lane - in) & (((uint64_t)1 << L % 64) - 1));
        }
        return count;
    }
    // Whether a run that has the pair before i1 goes on through the whole chunk from i1 on.
    __device__ bool goes_on(int64_t i1, uint32_t key) const {
        return i1 < n && pairs[i1].key == key && pairs[min(n, i1 + whole) - 1].key == key;
    }
    __device__ int64_t chunk_of(int64_t group) const {
        return tiles == 1 ? group : (int64_t)((uint32_t)group / (uint32_t)tiles);
    }
};

constexpr int64_t kJoinGrid = 512;      // two workgroups per unit

// A group's pairs: through the scalar cache where the group is a wavefront.
template <int L>
__device__ __forceinline__ auto pairs_of(const Pair *p) {
    if constexpr (L == 64)
        return constant<Pair>(p);
    else
        return p;
}

template <typename T>
__device__ __forceinline__ const T *grad_row(const GradArgs &a, uint32_t token) {
    return (const T *)((const char *)a.grad + (int64_t)token * a.grad_stride);
}

// `empty`: no id points at the row.
template <typename T, bool TAIL>
__device__ __forceinline__ void write_row(const GradArgs &a, uint32_t key, int col, int exchange,
                                          const float (&sum)[kCols], bool empty = false) {
    T *p = (T *)((char *)a.table + (int64_t)key * a.table_stride) + col;
    const bool part = TAIL && col + kCols > a.cols;
    float y[kCols];
#pragma unroll
    for (int i = 0; i < kCols; ++i)
        y[i] = empty ? 0.0f : sum[i] * a.factor;       // zeros for any factor
    if (a.accumulate) {
        const Raw<T> old = part ? load_block(p, a.cols - col) : load_block(p);
#pragma unroll
        for (int i = 0; i < kCols; ++i)
            y[i] += (float)old[i];
    }
    if (part)
        store_block(p, y, a.cols - col);
    else if (TAIL)
        store_block(p, y);
    else
        stream_block(p, y, exchange);
}

// `strips` of the workgroups write zeros into `strip` rows each, where no id points at them; the others
// add up chunks, a group of L lanes per chunk and tile of L column blocks. The strips are spread
// evenly over the launch, their writes between the chunks' reads.
template <typename TG, typename TT, int L, bool DROP, bool TAIL>
__global__ __launch_bounds__(256) void sum_kernel(GradArgs a, Runs r, uint32_t strips, int strip) {
    const uint32_t strips_before = (uint32_t)((uint64_t)blockIdx.x * strips / gridDim.x);
    if ((uint32_t)((uint64_t)(blockIdx.x + 1) * strips / gridDim.x) > strips_before) {
        const int64_t first = (int64_t)strips_before * strip, last = min(first + strip, a.rows);
        const int lane = threadIdx.x & 63;
        for (int64_t row0 = first; row0 < last; row0 += 64) {
            const int count = (int)min((int64_t)64, last - row0);
            const uint64_t empty = __ballot(lane < count && !r.found[row0 + min(lane, count - 1)]);
            for (int row = threadIdx.x / L; row < count; row += 256 / L) {
                if (!(empty >> row & 1))
                    continue;
                TT *p = (TT *)((char *)a.table + (row0 + row) * a.table_stride);
                if (TAIL) {
                    for (int col = threadIdx.x % L; col < a.cols; col += L)
                        p[col] = (TT)0.0f;
                } else {
                    for (int i = threadIdx.x % L; i < a.cols * (int)sizeof(TT) / 16; i += L)
                        __builtin_nontemporal_store(words_t{}, (words_t *)p + i);
                }
            }
        }
        return;
    }
    // Chunk and column tile of the group, the wavefront's where it is one.
    const int64_t group = (int64_t)(blockIdx.x - strips_before) * (256 / L) +
                          (L == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / L)
                                   : threadIdx.x / L);
    const int64_t c = r.chunk_of(group);
    const int block = (int)(group - c * r.tiles) * L + (int)(threadIdx.x % L);
    const auto pairs = pairs_of<L>(r.pairs);
    const int64_t start = min(c, r.chunks - 1) * r.chunk, stop = min(r.n, start + r.chunk);
    const uint32_t low = pairs[start].key, high = pairs[stop - 1].key;
    const int of_low = r.leading<L>(start, low), of_high = stop < r.n ? r.leading<L>(stop, high) : 0;
    if (c >= r.chunks || block >= r.blocks)
        return;
    const bool began = start > 0 && pairs[start - 1].key == low;
    const ChunkEnds ends =
        chunk_ends(start, stop, r.n, r.chunk, began, of_low, of_high, high, a.rows);
    const int64_t i0 = ends.i0, i1 = ends.i1;
    const bool head = ends.head, tail = ends.tail;
    const int col = block * kCols;
    const int exchange = exchange_of(block, a.cols);
    uint32_t current = pairs[i0].key;
    bool first = true;
    float sum[kCols] = {};
    auto finish = [&](bool open) {
        if (current < (uint64_t)a.rows) {
            if (open)
                store_block(r.partial + (c * 2 + (first && head ? 0 : 1)) * r.width + col, sum);
            else
                write_row<TT, TAIL>(a, current, col, exchange, sum);
        }
    };
    auto add = [&](uint32_t key, uint32_t token, Raw<TG> x) {
        if (key != current) {
            finish(first && head);
            current = key;
            first = false;
#pragma unroll
            for (int k = 0; k < kCols; ++k)
                sum[k] = 0.0f;
        }
        load_rest<TAIL>(x, grad_row<TG>(a, token), col, a.cols, exchange);
        Bits bits;
        if (DROP)
            bits = draw_bits(a.mask, token, block);
#pragma unroll
        for (int k = 0; k < kCols; ++k) {
            const float v = (float)x[k];
            sum[k] += !DROP || bits.kept(k, a.mask.threshold) ? v : 0.0f;
        }
    };
    // kAhead rows are added while the next kAhead are on their way, then the rest. Ids outside the table
    // come last and end the loop: `current` is then the last id of the table.
    constexpr int kAhead = kSumAhead;
    uint32_t key[2][kAhead], token[2][kAhead];
    Raw<TG> x[2][kAhead];
    auto fetch = [&](int s, int64_t i) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            key[s][j] = pairs[min(i + j, i1 - 1)].key;
            token[s][j] = pairs[min(i + j, i1 - 1)].token;
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            x[s][j] = load_most<TAIL, true>(grad_row<TG>(a, token[s][j]), col, a.cols, exchange);
    };
    const int64_t even = pipelined(ends);
    if (i0 < even)
        fetch(0, i0);
    for (int64_t i = i0; i < even && key[0][0] < (uint64_t)a.rows; i += 2 * kAhead) {
        fetch(1, i + kAhead);
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            add(key[0][j], token[0][j], x[0][j]);
        if (i + 2 * kAhead < even)
            fetch(0, i + 2 * kAhead);
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            add(key[1][j], token[1][j], x[1][j]);
    }
    if (even < i1 && pairs[even].key < (uint64_t)a.rows) {
        fetch(0, even);
        if (even + kAhead < i1)
            fetch(1, even + kAhead);
#pragma unroll
        for (int j = 0; j < 2 * kAhead; ++j)
            if (even + j < i1)
                add(key[j / kAhead][j % kAhead], token[j / kAhead][j % kAhead],
                    x[j / kAhead][j % kAhead]);
    }
    finish((first && head) || tail);
    if (tail && !head && r.listed && block == 0 && current < (uint64_t)a.rows)
        r.append(c);
}

// The partial sums of kFold chunks, a wavefront for 64 column blocks of them. A lane looks at one
// of the 2 * kFold places for a partial sum; those that hold one, in order, are to this kernel what a chunk's
// sorted tokens are to the one above, and runs that leave its chunks go to `out`.
template <typename TT>
__global__ __launch_bounds__(64) void fold_kernel(GradArgs a, Runs r, int tiles, float *out) {
    static_assert(2 * kFold <= 64, "one place per lane");
    const int64_t f = blockIdx.x / tiles;
    const int lane = threadIdx.x;
    const int block = (int)(blockIdx.x - f * tiles) * 64 + lane;
    const int64_t c = f * kFold + lane / 2;
    bool held = false, goes_on = false;
    uint32_t key = 0;
    if (lane < 2 * kFold && c < r.chunks) {
        const int64_t i0 = c * r.chunk, i1 = min(r.n, i0 + r.chunk);
        const uint32_t low = r.pairs[i0].key, high = r.pairs[i1 - 1].key;
        const bool head = i0 > 0 && r.pairs[i0 - 1].key == low;
        const bool inside = head && low == high;       // a run that began earlier covers the chunk
        goes_on = r.goes_on(i1, high);
        key = lane & 1 ? high : low;
        held = lane & 1 ? goes_on && !inside : inside;
        held &= key < (uint64_t)a.rows;
    }
    uint64_t places = __ballot(held);
    if (!places)
        return;
    const int last_lane = (int)min(r.chunks - f * kFold, (int64_t)kFold) * 2 - 1;
    const bool last_open = __shfl((int)goes_on, last_lane) &&
                           __shfl((int)(key < (uint64_t)a.rows), last_lane);
    bool open = places & 1;                       // the run at hand began before these chunks
    const int col = block * kCols;
    const bool live = block < r.blocks;
    const int exchange = exchange_of(block, a.cols);
    const float *from = r.partial + f * 2 * kFold * r.width + (live ? col : 0);
    float sum[kCols] = {};
    constexpr int kAhead = 16;
    while (places) {
        Raw<float> x[kAhead];
        int place[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {        // the last one again where fewer are left
            place[j] = places ? __builtin_ctzll(places) : j ? place[j - 1] : 0;
            x[j] = load_block(from + (int64_t)place[j] * r.width);
            places &= places - 1;
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (j && place[j] == place[j - 1])
                break;
#pragma unroll
            for (int k = 0; k < kCols; ++k)
                sum[k] += x[j][k];
            const uint32_t here = __shfl(key, place[j]);
            const int next = j + 1 < kAhead && place[j + 1] != place[j] ? place[j + 1]
                             : places                                   ? __builtin_ctzll(places)
                                                                        : -1;
            const uint32_t there = __shfl(key, max(next, 0));
            if (next >= 0 && there == here)
                continue;
            const bool leaves = next < 0 && last_open;
            if (leaves && !open && block == 0)
                r.append(f);
            if (live) {
                if (open || leaves)
                    store_block(out + (f * 2 + (open ? 0 : 1)) * r.width + col, sum);
                else
                    write_row<TT, true>(a, here, col, exchange, sum);
            }
            open = false;
#pragma unroll
            for (int k = 0; k < kCols; ++k)
                sum[k] = 0.0f;
        }
    }
}

// The sums of T / L lane groups, added up in their order into the first group's; by the whole workgroup.
template <int L, int T>
__device__ __forceinline__ void add_groups(float (&part)[T][kCols + 1]) {
    __syncthreads();
    for (int i = threadIdx.x; i < L * kCols; i += T) {
        float sum = part[i / kCols][i % kCols];
#pragma unroll 8
        for (int g = 1; g < T / L; ++g)
            sum += part[g * L + i / kCols][i % kCols];
        part[i / kCols][i % kCols] = sum;
    }
    __syncthreads();
}

// The runs that go on through whole chunks: for each and every tile of L column blocks a workgroup adds
// up the partial sums. Lane groups take every (kJoinThreads / L)-th chunk of the run, and the first adds
// their sums in order.
template <typename TT, int L>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(GradArgs a, Runs r) {
    constexpr int kGroups = kJoinThreads / L;
    __shared__ float part[kJoinThreads][kCols + 1];
    const uint32_t total = r.list[0] * (uint32_t)r.tiles;
    for (uint32_t e = blockIdx.x; e < total; e += gridDim.x) {
        const uint32_t entry = e / (uint32_t)r.tiles;
        const int64_t c = r.list[1 + entry];
        const uint32_t key = r.pairs[min(r.n, (c + 1) * r.chunk) - 1].key;
        // The last chunk that holds a sum of the run: a probe per thread and round.
        int64_t end = c, past = r.chunks;              // `end` does, or is c; `past` does not
        while (past - end > 1) {
            const int64_t step = (past - end + kJoinThreads - 1) / kJoinThreads;
            const int64_t d = end + (threadIdx.x + 1) * step;
            const int hits = __syncthreads_count(d < past && r.goes_on(d * r.chunk, key));
            end += hits * step;
            past = min(past, end + step);
        }
        const int lane = threadIdx.x % L, group = threadIdx.x / L;
        const int block = (int)(e - entry * r.tiles) * L + lane;
        const int col = block * kCols;
        float sum[kCols] = {};
        constexpr int kAhead = 8;                      // sums on their way
        const float *from = r.partial + (block < r.blocks ? col : 0);
        for (int64_t d = c + group; d <= end; d += kAhead * kGroups) {
            Raw<float> x[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                // The run is open at its first chunk's end and at the later ones' start.
                const int64_t at = min(d + j * kGroups, end);
                x[j] = load_block(from + (at * 2 + (at == c ? 1 : 0)) * r.width);
            }
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
                if (d + j * kGroups <= end)
#pragma unroll
                    for (int k = 0; k < kCols; ++k)
                        sum[k] += x[j][k];
        }
#pragma unroll
        for (int k = 0; k < kCols; ++k)
            part[threadIdx.x][k] = sum[k];
        add_groups<L, kJoinThreads>(part);
        if (group == 0 && block < r.blocks) {
#pragma unroll
            for (int k = 0; k < kCols; ++k)
                sum[k] = part[lane][k];
            write_row<TT, true>(a, key, col, exchange_of(block, a.cols), sum);
        }
        __syncthreads();
    }
}

// ---- small calls and small tables: pairs in LDS ----

// A workgroup has a window of the tokens, `rows` rows of the table and one column tile. It reads the
// window's ids, puts its rows' tokens in order in LDS by the digit pass above, and adds them up as
// above: its lane groups share the tokens out evenly, and what runs leave at their edges meets in LDS.
//   A small call is one window and this launch.
//   A table of few rows has few sums per window, less than they are made of: they are added up over the
//   windows by a second launch, in place of the sort, the fold and the join of the whole call.
template <typename TG, typename TT, int L, bool DROP, bool TAIL, int T>
__global__ __launch_bounds__(T) void small_kernel(GradArgs a, Window v) {
    constexpr int kGroups = T / L, kEach = kSmallIds / kSortThreads, kWaves = T / 64;
    __shared__ uint32_t place[kWaves][kSmallRows];         // counts, then next places
    __shared__ uint32_t begin[kSmallRows + 1];
    __shared__ uint32_t list[T * kEach];                   // row << 12 | token, sorted
    __shared__ __attribute__((aligned(16))) float part[kGroups][2][L * kCols];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t tile = blockIdx.x % (uint32_t)v.tiles, rest = blockIdx.x / (uint32_t)v.tiles;
    const uint32_t window = rest % (uint32_t)v.count;
    const int64_t row0 = (int64_t)(rest / (uint32_t)v.count) * v.rows;
    const int64_t token0 = (int64_t)window * v.tokens;
    const int count = (int)min((int64_t)v.rows, a.rows - row0);
    const int n = (int)min((int64_t)v.tokens, a.n - token0);
    place[wave][lane] = 0;
    __syncthreads();
    // Each wavefront has a row of the tokens; row_of: of the range, or `count`.
    const int span = (n + T - 1) / T * 64, from = wave * span;
    const int to = min(n, from + span);
    auto row_of = [&](int i) {
        const int64_t at = token0 + i;
        const int64_t id = a.id_bytes == 8 ? static_cast<const int64_t *>(a.ids)[at]
                                           : static_cast<const int32_t *>(a.ids)[at];
        return id >= row0 && id < row0 + count ? (int)(id - row0) : count;
    };
    int row[kEach];
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const int i = from + j * 64 + lane;
        row[j] = j * 64 < span && i < to ? row_of(i) : count;
        if (row[j] < count)
            atomicAdd(&place[wave][row[j]], 1u);
    }
    __syncthreads();
    if (wave == 0) {
        uint32_t sum = 0;
        for (int w = 0; w < kWaves; ++w)
            sum += place[w][lane];
        uint32_t next = sum;                               // inclusive prefix over the rows
#pragma unroll
        for (int s = 1; s < 64; s <<= 1) {
            const uint32_t y = __shfl_up(next, s);
            if (lane >= s)
                next += y;
        }
        next -= sum;
        begin[lane] = next;
        if (lane == 63)
            begin[64] = next + sum;
        for (int w = 0; w < kWaves; ++w) {
            const uint32_t c = place[w][lane];
            place[w][lane] = next;
            next += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const bool live = row[j] < count;
        uint64_t peers = __ballot(live);
        if (!peers)
            continue;
#pragma unroll
        for (int b = 0; b < 6; ++b) {
            const uint64_t set = __ballot(row[j] >> b & 1);
            peers &= row[j] >> b & 1 ? set : ~set;
        }
        const uint32_t rank = __popcll(peers & (((uint64_t)1 << lane) - 1));
        const uint32_t first = live ? place[wave][row[j]] : 0;
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");    // as in digit_scatter
        __builtin_amdgcn_wave_barrier();
        if (live && rank == 0)
            place[wave][row[j]] = first + __popcll(peers);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (live)
            list[first + rank] = (uint32_t)row[j] << 12 | (uint32_t)(from + j * 64 + lane);
    }
    __syncthreads();
    const int total = (int)begin[64];
    const int in = threadIdx.x % L, group = threadIdx.x / L;
    const int block = (int)tile * L + in, col = block * kCols;
    const bool live = block < blocks_of(a.cols);
    const int exchange = live ? exchange_of(block, a.cols) : kAlone;
    auto write = [&](int r, const float (&sum)[kCols], bool empty) {
        if (!live)
            return;
        if (v.partial)
            store_block(v.partial + (window * a.rows + row0 + r) * v.width + col, sum);
        else
            write_row<TT, TAIL>(a, (uint32_t)(row0 + r), col, exchange, sum, empty);
    };
    // A window's row that no id points at has the sums -0, which no others are: those begin with +0.
    if (v.partial || !a.accumulate)
        for (int r = group; r < count; r += kGroups)
            if (begin[r] == begin[r + 1]) {
                float none[kCols];
#pragma unroll
                for (int k = 0; k < kCols; ++k)
                    none[k] = -0.0f;
                write(r, none, true);
            }
    // This group's tokens [i0, i1) of the list.
    const int chunk = (total + kGroups - 1) / kGroups;
    const int i0 = min(total, group * chunk), i1 = min(total, i0 + chunk);
    auto at_row = [&](int i) { return (int)(list[i] >> 12); };
    if (i0 < i1) {
        const bool head = (int)begin[at_row(i0)] < i0;
        int current = at_row(i0);
        bool first = true;
        float sum[kCols] = {};
        auto finish = [&](bool open) {
            if (open) {
#pragma unroll
                for (int k = 0; k < kCols; ++k)
                    part[group][first && head ? 0 : 1][in * kCols + k] = sum[k];
            } else {
                write(current, sum, false);
            }
        };
        constexpr int kAhead = 4;
        for (int i = i0; i < i1; i += kAhead) {
            Raw<TG> x[kAhead];
            uint32_t item[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                item[j] = list[min(i + j, i1 - 1)];
                x[j] = load_most<TAIL, true>(grad_row<TG>(a, (uint32_t)token0 + (item[j] & (kSmallIds - 1))),
                                             live ? col : 0, a.cols, exchange);
            }
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                if (i + j >= i1)
                    break;
                const uint32_t token = (uint32_t)token0 + (item[j] & (kSmallIds - 1));
                if ((int)(item[j] >> 12) != current) {
                    finish(first && head);
                    current = (int)(item[j] >> 12);
                    first = false;
#pragma unroll
                    for (int k = 0; k < kCols; ++k)
                        sum[k] = 0.0f;
                }
                load_rest<TAIL>(x[j], grad_row<TG>(a, token), live ? col : 0, a.cols, exchange);
                Bits bits;
                if (DROP)
                    bits = draw_bits(a.mask, token, block);
#pragma unroll
                for (int k = 0; k < kCols; ++k) {
                    const float v = (float)x[j][k];
                    sum[k] += !DROP || bits.kept(k, a.mask.threshold) ? v : 0.0f;
                }
            }
        }
        finish((first && head) || (int)begin[current + 1] > i1);
    }
    __syncthreads();
    // A run that starts in this group's tokens and goes on past them.
    if (i0 < i1) {
        const int r = at_row(i1 - 1);
        if ((int)begin[r] >= i0 && (int)begin[r + 1] > i1) {
            const int last = ((int)begin[r + 1] - 1) / chunk;
            float sum[kCols];
#pragma unroll
            for (int k = 0; k < kCols; ++k)
                sum[k] = part[group][1][in * kCols + k];
#pragma unroll 4
            for (int g = group + 1; g <= last; ++g)
#pragma unroll
                for (int k = 0; k < kCols; ++k)
                    sum[k] += part[g][0][in * kCols + k];
            write(r, sum, false);
        }
    }
}

// A row of a small table and one column tile: its sums over the windows, shared out among the lane
// groups and added up in order.
template <typename TT, int L>
__global__ __launch_bounds__(256) void windows_kernel(GradArgs a, Window v) {
    constexpr int kGroups = 256 / L;
    __shared__ float part[256][kCols + 1];
    const int row = blockIdx.x / v.tiles, lane = threadIdx.x % L, group = threadIdx.x / L;
    const int block = (int)(blockIdx.x - row * v.tiles) * L + lane, col = block * kCols;
    const bool live = block < blocks_of(a.cols);
    const int share = (v.count + kGroups - 1) / kGroups, last = min(v.count, (group + 1) * share);
    float sum[kCols];
#pragma unroll
    for (int k = 0; k < kCols; ++k)
        sum[k] = -0.0f;
    if (live)
#pragma unroll 8
        for (int w = group * share; w < last; ++w) {
            const Raw<float> x = load_block(v.partial + (w * a.rows + row) * v.width + col);
#pragma unroll
            for (int k = 0; k < kCols; ++k)
                sum[k] += x[k];
        }
#pragma unroll
    for (int k = 0; k < kCols; ++k)
        part[threadIdx.x][k] = sum[k];
    add_groups<L, 256>(part);
    if (group == 0 && live) {
#pragma unroll
        for (int k = 0; k < kCols; ++k)
            sum[k] = part[lane][k];
        const bool empty = __float_as_uint(sum[0]) == 0x80000000u;       // in every window
        if (!empty || !a.accumulate)
            write_row<TT, true>(a, row, col, exchange_of(block, a.cols), sum, empty);
    }
}

template <typename Source>
void launch_pass(Source source, const GradArgs &a, const GradPlan &p, int pass, Pair *out,
                 hipStream_t stream) {
    char *ws = static_cast<char *>(a.workspace);
    uint32_t *counts = (uint32_t *)(ws + p.counts);
    uint8_t *found = pass == 0 && !a.accumulate ? (uint8_t *)(ws + p.found) : nullptr;
    const int64_t words = found ? round16(a.rows + 1) / 16 : 0;
    const int64_t clears = (words + kClearWords - 1) / kClearWords;
    const int shift = pass * p.sort.digit_bits;
    if (p.sort.tiles + clears > 0)
        digit_counts<<<(unsigned)(p.sort.tiles + clears), kSortThreads, 0, stream>>>(
            source, a.n, p.sort.tile, shift, 1 << p.sort.digit_bits, p.sort.tiles, counts,
            (words_t *)found, words, pass == 0 ? (uint32_t *)(ws + p.list) : nullptr);
    if (p.sort.tiles > 0)
        digit_scatter<<<p.sort.tiles, kSortThreads, 0, stream>>>(
            source, a.n, p.sort.tile, shift, p.sort.digit_bits, counts, p.sort.tiles, out, found);
}

template <typename TG, typename TT, int L, bool DROP, bool TAIL>
void launch_small(const GradArgs &a, const Window &v, hipStream_t stream) {
    const unsigned groups = (unsigned)((a.rows + v.rows - 1) / v.rows * v.count * v.tiles);
    if (v.partial)
        small_kernel<TG, TT, L, DROP, TAIL, kWindowThreads>
            <<<groups, kWindowThreads, 0, stream>>>(a, v);
    else          // one kernel for all alignments: its time is not in the rows
        small_kernel<TG, TT, L, DROP, true, kSortThreads><<<groups, kSortThreads, 0, stream>>>(a, v);
}

template <typename TG, typename TT, int L, bool DROP, bool TAIL>
void launch_sum(const GradArgs &a, const Runs &r, const GradPlan &p, hipStream_t stream) {
    if (p.window.count) {
        Window v = p.window;
        v.partial = v.count > 1 ? static_cast<float *>(a.workspace) : nullptr;
        launch_small<TG, TT, L, DROP, TAIL>(a, v, stream);
        if (v.partial)
            windows_kernel<TT, L><<<(unsigned)(a.rows * v.tiles), 256, 0, stream>>>(a, v);
        return;
    }
    const int64_t sum_groups = (r.chunks * r.tiles + 256 / L - 1) / (256 / L);
    // Strips of rows of about 128 KiB, 64 rows at most, but more where the launch would have more
    // workgroups than it may (tables of over 2^27 rows).
    const int64_t row_bytes = (int64_t)a.cols * sizeof(TT);
    int strip = (int)std::max<int64_t>(1, std::min<int64_t>(64, kStripBytes / row_bytes));
    while (a.rows / strip > kMaxStrips)
        strip *= 2;
    const int64_t strips = a.accumulate ? 0 : (a.rows + strip - 1) / strip;
    if (sum_groups + strips > 0)
        sum_kernel<TG, TT, L, DROP, TAIL><<<(unsigned)(sum_groups + strips), 256, 0, stream>>>(
            a, r, (uint32_t)strips, strip);
    Runs j = r;
    if (p.folds) {
        j.partial = (float *)((char *)a.workspace + p.folded);
        j.chunk = r.chunk * kFold;
        j.chunks = p.folds;
        const int tiles = (r.blocks + 63) / 64;
        fold_kernel<TT><<<(unsigned)(p.folds * tiles), 64, 0, stream>>>(a, r, tiles, j.partial);
    }
    if (j.chunks > 1)
        join_kernel<TT, L><<<(unsigned)std::min<int64_t>(j.chunks * r.tiles, kJoinGrid),
                             kJoinThreads, 0, stream>>>(a, j);
}

template <typename TG, typename TT, int L>
void launch_drop(const GradArgs &a, const Runs &r, const GradPlan &p, hipStream_t stream) {
    const bool drop = a.mask.threshold != kThresholdOne;
    const bool tail = a.cols % kCols || !even_rows(a.grad, a.grad_stride) ||
                      !even_rows(a.table, a.table_stride);
    if (drop)
        tail ? launch_sum<TG, TT, L, true, true>(a, r, p, stream)
             : launch_sum<TG, TT, L, true, false>(a, r, p, stream);
    else
        tail ? launch_sum<TG, TT, L, false, true>(a, r, p, stream)
             : launch_sum<TG, TT, L, false, false>(a, r, p, stream);
}

template <typename TG, typename TT>
void launch_lanes(const GradArgs &a, const Runs &r, const GradPlan &p, hipStream_t stream) {
    if (p.lanes == 4)
        launch_drop<TG, TT, 4>(a, r, p, stream);
    else if (p.lanes == 16)
        launch_drop<TG, TT, 16>(a, r, p, stream);
    else
        launch_drop<TG, TT, 64>(a, r, p, stream);
}

}  // namespace

int64_t grad_workspace_bytes(int64_t n, int64_t rows, int32_t cols) {
    return grad_plan(n, rows, cols).bytes;
}

hipError_t launch_embedding_grad(const GradArgs &a, hipStream_t stream) {
    const GradPlan p = grad_plan(a.n, a.rows, a.cols);
    char *ws = static_cast<char *>(a.workspace);
    Pair *pairs[2] = {(Pair *)(ws + p.pairs0), (Pair *)(ws + p.pairs1)};
    for (int pass = 0; !p.window.count && pass < (a.n > 0 ? p.sort.passes : 1); ++pass) {
        Pair *out = pairs[pass & 1];
        if (pass)
            launch_pass(FromPairs{pairs[(pass - 1) & 1]}, a, p, pass, out, stream);
        else if (a.id_bytes == 4)
            launch_pass(FromIds<int32_t>{(const int32_t *)a.ids, a.rows}, a, p, 0, out, stream);
        else
            launch_pass(FromIds<int64_t>{(const int64_t *)a.ids, a.rows}, a, p, 0, out, stream);
    }
    const Runs r{pairs[(p.sort.passes - 1) & 1], (const uint8_t *)(ws + p.found),
                 (float *)(ws + p.partial), a.n, p.chunk, p.chunks, p.width, blocks_of(a.cols),
                 p.tiles, p.chunk, p.folds == 0, (uint32_t *)(ws + p.list)};
    if (a.grad_type == kF32)
        launch_lanes<float, float>(a, r, p, stream);
    else if (a.grad_type == kF16 && a.table_type == kF32)
        launch_lanes<half_t, float>(a, r, p, stream);
    else if (a.grad_type == kF16)
        launch_lanes<half_t, half_t>(a, r, p, stream);
    else if (a.table_type == kF32)
        launch_lanes<bf16_t, float>(a, r, p, stream);
    else
        launch_lanes<bf16_t, bf16_t>(a, r, p, stream);
    return hipGetLastError();
}

}  // namespace ccj

// Device helpers of the scoring model's input layer: blocks of 8 elements, dropout's bits, division
// by a launch's constant.
#pragma once

#include <stdint.h>

#include <hip/hip_runtime.h>

#include "layers_internal.h"

namespace ccj {
namespace {

typedef _Float16 half_t;
typedef __bf16 bf16_t;

typedef uint32_t words_t __attribute__((ext_vector_type(4), aligned(2)));   // aligned or not

constexpr int kCols = 8;         // columns of a block: one thread's unit of work, and as many as
                                 // one draw of dropout's generator serves

// What no part of a launch writes, so that a wavefront whose lanes all read one place of it can do so
// through the scalar cache.
template <typename T>
using Constant = const __attribute__((address_space(4))) T *;

template <typename T>
__device__ __forceinline__ Constant<T> constant(const void *p) {
    return (Constant<T>)(uintptr_t)p;
}

// Number of column blocks in a row.
inline __host__ __device__ int blocks_of(int cols) { return (cols + kCols - 1) / kCols; }

// Quotients of numbers below 2^31 by a divisor fixed at launch, 1 to 2^30: a multiplication and a
// shift. With s = ceil(log2 d) and m = ceil(2^(31 + s) / d) the error m * d - 2^(31 + s) is below
// d <= 2^s, so n * m / 2^(31 + s) has the quotient's integer part for every n < 2^31.
struct Divider {
    uint32_t m, s;
    explicit Divider(uint32_t d) {
        s = 0;
        while (((uint64_t)1 << s) < d)
            ++s;
        m = (uint32_t)((((uint64_t)1 << (31 + s)) + d - 1) / d);
        s += 31;
    }
    __device__ uint32_t operator()(uint32_t n) const { return (uint32_t)(((uint64_t)n * m) >> s); }
};

// Eight consecutive elements, from memory aligned to one element: the wide loads that come of it need
// no more on this architecture. Kept as words until they are used, so that several loads are in
// flight together.
template <typename T>
struct Raw {
    static constexpr int kWords = kCols * sizeof(T) / 16;
    words_t w[kWords];
    __device__ T operator[](int i) const {
        T v[16 / sizeof(T)];
        __builtin_memcpy(v, &w[i / (16 / sizeof(T))], 16);
        return v[i % (16 / sizeof(T))];
    }
};

// A block of 32-bit elements is two 16-byte pieces, so a wavefront's own blocks would be every second
// piece of memory: half cache lines, which past the caches move at 3 TB/s where whole ones reach 6.5.
// Lanes that hold consecutive blocks of one row therefore exchange pieces, and each access of four of
// them covers 64 bytes, of eight 128: the lane with number q of its 4 or 8 moves piece q of theirs,
// then piece q + 4 or q + 8.
enum : int { kAlone = 0, kFour = 4, kEight = 8 };

// How many lanes may exchange pieces, where lanes of consecutive numbers hold consecutive blocks and
// lane 0 a multiple of 8 of them: those whose blocks are all full.
__device__ __forceinline__ int exchange_of(uint32_t block, int cols) {
    return (int)((block | 7) + 1) * kCols <= cols   ? kEight
           : (int)((block | 3) + 1) * kCols <= cols ? kFour
                                                    : kAlone;
}

template <int CONTROL>
__device__ __forceinline__ words_t of_lanes(words_t x) {
    words_t y;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        y[i] = __builtin_amdgcn_mov_dpp((int)x[i], CONTROL, 0xf, 0xf, true);
    return y;
}

constexpr int quad_perm(int a, int b, int c, int d) { return a | b << 2 | c << 4 | d << 6; }
constexpr int kRowLeft4 = 0x104, kRowRight4 = 0x114;      // from the lane 4 further, 4 before

__device__ __forceinline__ words_t either(bool c, words_t x, words_t y) {
    words_t z;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        z[i] = c ? x[i] : y[i];
    return z;
}

// Of four lanes' blocks (a, b), the pieces q and q + 4; back again.
__device__ __forceinline__ void to_pieces4(words_t &a, words_t &b) {
    const bool odd = threadIdx.x & 1;
    const words_t lower = either(odd, of_lanes<quad_perm(0, 0, 1, 1)>(b),
                                 of_lanes<quad_perm(0, 0, 1, 1)>(a));
    b = either(odd, of_lanes<quad_perm(2, 2, 3, 3)>(b), of_lanes<quad_perm(2, 2, 3, 3)>(a));
    a = lower;
}

__device__ __forceinline__ void from_pieces4(words_t &a, words_t &b) {
    const bool upper = threadIdx.x & 2;
    const words_t first = either(upper, of_lanes<quad_perm(0, 2, 0, 2)>(b),
                                 of_lanes<quad_perm(0, 2, 0, 2)>(a));
    b = either(upper, of_lanes<quad_perm(1, 3, 1, 3)>(b), of_lanes<quad_perm(1, 3, 1, 3)>(a));
    a = first;
}

// Between the pieces q and q + 4 of the fours and q and q + 8 of their eight: its own inverse.
__device__ __forceinline__ void swap_fours(words_t &a, words_t &b) {
    const bool second = threadIdx.x & 4;
    const words_t c = either(second, of_lanes<kRowRight4>(b), a);
    b = either(second, b, of_lanes<kRowLeft4>(a));
    a = c;
}

template <typename T>
__device__ __forceinline__ Raw<T> load_block(const T *p) {
    Raw<T> r;
#pragma unroll
    for (int i = 0; i < Raw<T>::kWords; ++i)
        r.w[i] = ((const words_t *)p)[i];
    return r;
}

template <typename T>
__device__ __forceinline__ Raw<T> load_once(const T *p) {
    Raw<T> r;
#pragma unroll
    for (int i = 0; i < Raw<T>::kWords; ++i)
        r.w[i] = __builtin_nontemporal_load((const words_t *)p + i);
    return r;
}

// The load of a block whose lane exchanges pieces; settle() puts them in place.
template <bool ONCE, typename T>
__device__ __forceinline__ Raw<T> load_pieces(const T *p, int exchange) {
    Raw<T> r;
    const words_t *w = (const words_t *)p;
    if constexpr (Raw<T>::kWords == 2) {
        w -= threadIdx.x & (exchange ? exchange - 1 : 0);
        const words_t *second = w + (exchange ? exchange : 1);
        // Non-temporal: what is read once leaves the caches to what is read again, and comes at
        // 6.7 TB/s where other loads reach 5.9 (rows of 4 KiB in any order).
        r.w[0] = ONCE ? __builtin_nontemporal_load(w) : *w;
        r.w[1] = ONCE ? __builtin_nontemporal_load(second) : *second;
    } else {
        r.w[0] = ONCE ? __builtin_nontemporal_load(w) : *w;
    }
    return r;
}

template <typename T>
__device__ __forceinline__ void settle(Raw<T> &r, int exchange) {
    if constexpr (Raw<T>::kWords == 2) {
        words_t a = r.w[0], b = r.w[1];
        swap_fours(a, b);
        a = either(exchange == kEight, a, r.w[0]);
        b = either(exchange == kEight, b, r.w[1]);
        from_pieces4(a, b);
        r.w[0] = either(exchange != kAlone, a, r.w[0]);
        r.w[1] = either(exchange != kAlone, b, r.w[1]);
    }
}

// The first `count` elements of a row's last block, then zeros.
template <typename T>
__device__ __forceinline__ Raw<T> load_block(const T *p, int count) {
    T v[kCols];
#pragma unroll
    for (int i = 0; i < kCols; ++i)
        v[i] = i < count ? p[i] : (T)0.0f;
    Raw<T> r;
    __builtin_memcpy(&r, v, sizeof(r));
    return r;
}

template <typename T>
__device__ __forceinline__ Raw<T> packed(const float (&x)[kCols]) {
    typedef float floats __attribute__((ext_vector_type(kCols)));
    typedef T values __attribute__((ext_vector_type(kCols)));
    floats f;
#pragma unroll
    for (int i = 0; i < kCols; ++i)
        f[i] = x[i];
    const values v = __builtin_convertvector(f, values);     // in pairs
    Raw<T> r;
    __builtin_memcpy(&r, &v, sizeof(r));
    return r;
}

template <typename T>
__device__ __forceinline__ void store_block(T *p, const float (&x)[kCols]) {
    const Raw<T> r = packed<T>(x);
#pragma unroll
    for (int i = 0; i < Raw<T>::kWords; ++i)
        ((words_t *)p)[i] = r.w[i];
}

// The same as store_block past the caches' reach, for outputs that would push out of the caches what
// the kernel reads more than once. The lanes that exchange pieces are all here.
template <typename T>
__device__ __forceinline__ void stream_block(T *p, const float (&x)[kCols], int exchange) {
    const Raw<T> r = packed<T>(x);
    if constexpr (Raw<T>::kWords == 2) {
        words_t a = r.w[0], b = r.w[1];
        to_pieces4(a, b);
        words_t c = a, d = b;
        swap_fours(c, d);
        a = exchange == kEight ? c : exchange == kFour ? a : r.w[0];
        b = exchange == kEight ? d : exchange == kFour ? b : r.w[1];
        words_t *w = (words_t *)p - (threadIdx.x & (exchange ? exchange - 1 : 0));
        __builtin_nontemporal_store(a, w);
        __builtin_nontemporal_store(b, w + (exchange ? exchange : 1));
    } else {
        __builtin_nontemporal_store(r.w[0], (words_t *)p);
    }
}

template <typename T>
__device__ __forceinline__ void store_block(T *p, const float (&x)[kCols], int count) {
#pragma unroll
    for (int i = 0; i < kCols; ++i)
        if (i < count)
            p[i] = (T)x[i];
}

// A block of the row at p. TAIL: rows have a last block of fewer columns, or are not aligned to 16
// bytes (then accesses share cache lines, and what bypasses the caches moves them twice); its lanes read the block
// before it first (in rows of one block nothing), so that the loads of all lanes are in flight before
// the first of them is waited for.
template <bool TAIL, bool ONCE, typename T>
__device__ __forceinline__ Raw<T> load_most(const T *p, int col, int cols, int exchange) {
    if (TAIL && cols < kCols)
        return Raw<T>{};
    return load_pieces<ONCE && !TAIL>(p + (TAIL && col + kCols > cols ? col - kCols : col), exchange);
}

template <bool TAIL, typename T>
__device__ __forceinline__ void load_rest(Raw<T> &x, const T *p, int col, int cols, int exchange) {
    settle(x, exchange);
    if (TAIL && col + kCols > cols)
        x = load_block(p + col, cols - col);
}

// a ^ b ^ c in one instruction: of the truth table's inputs, 0x96 has the odd ones.
__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) {
    return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96);
}

// Philox4x32-10 (Salmon et al., SC 2011): ten rounds of two 32x32 -> 64 bit products. The four
// words are dropout's 16-bit numbers of eight columns.
struct Bits {
    uint32_t w[4];
    // Number i of the block lies below the threshold.
    __device__ bool kept(int i, int threshold) const {
        const uint32_t x = w[i >> 1];
        return (int)((i & 1) ? x >> 16 : x & 0xffffu) < threshold;
    }
};

__device__ __forceinline__ Bits draw_bits(const Mask &m, int64_t row, uint32_t block) {
    const uint64_t r = (uint64_t)(m.first_row + row);
    uint32_t c0 = (uint32_t)r, c1 = (uint32_t)(r >> 32), c2 = block, c3 = m.site;
    uint32_t k0 = m.key0, k1 = m.key1;
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
        c0 = xor3((uint32_t)(b >> 32), c1, k0);
        c2 = xor3((uint32_t)(a >> 32), c3, k1);
        c1 = (uint32_t)b;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return Bits{{c0, c1, c2, c3}};
}

}  // namespace
}  // namespace ccj

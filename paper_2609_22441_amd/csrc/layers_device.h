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

constexpr int kCols = 8;         // columns of a block: one thread's unit of work, and as many as
                                 // one draw of dropout's generator serves

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

// Eight consecutive elements in 32 bits, from memory aligned to one element (the wide loads that
// come of it need no more on this architecture) or, of a row's last block, the first `count`.
template <typename T>
struct Raw {
    T v[kCols];
};

template <typename T>
__device__ __forceinline__ Raw<T> load_block(const T *p) {
    Raw<T> r;
    __builtin_memcpy(&r, p, sizeof(r));
    return r;
}

template <typename T>
__device__ __forceinline__ Raw<T> load_block(const T *p, int count) {
    Raw<T> r;
#pragma unroll
    for (int i = 0; i < kCols; ++i)
        r.v[i] = i < count ? p[i] : (T)0.0f;
    return r;
}

template <typename T>
__device__ __forceinline__ void store_block(T *p, const float (&x)[kCols]) {
    Raw<T> r;
#pragma unroll
    for (int i = 0; i < kCols; ++i)
        r.v[i] = (T)x[i];
    __builtin_memcpy(p, &r, sizeof(r));
}

template <typename T>
__device__ __forceinline__ void store_block(T *p, const float (&x)[kCols], int count) {
#pragma unroll
    for (int i = 0; i < kCols; ++i)
        if (i < count)
            p[i] = (T)x[i];
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
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c1 = (uint32_t)b;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return Bits{{c0, c1, c2, c3}};
}

}  // namespace
}  // namespace ccj

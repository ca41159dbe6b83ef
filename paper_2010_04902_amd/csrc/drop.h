// Which values a dropout keeps (not part of the C-ABI): a counter-based generator, so that nothing is stored and every copy of a
// file drops the same values, wherever and in whatever order it is computed.
//
// Philox 4x32 of ten rounds (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011): the key is the
// seed, the counter (group of eight columns, row, low and high word of the call's offset).  Its four words are eight numbers of 16
// bits, low half first, one for each column: a value stays if its number is at least p 2^16, rounded to a whole number.  So p
// is taken to a multiple of 2^-16, and the scale is that of the p that is taken.  With 32 bits a value the generator
// would cost twice as much: its twenty products of 32 bits are a quarter of the rate of other instructions.
#ifndef BYZ_DROP_H
#define BYZ_DROP_H

#include <cmath>

#include "worker_internal.h"

namespace byz_worker {

struct Drop {
    uint32_t key0 = 0, key1 = 0;
    uint64_t offset = 0;
    const int64_t *offset_at = nullptr;  // added to the offset
    uint32_t first_row = 0;
    uint32_t threshold = 0;  // 0: everything stays, 65536: nothing does
    float scale = 1.0f;
};

inline bool drop_ok(float p, const int64_t *offset_at, int64_t first_row, int64_t rows, int64_t cols) {
    return p >= 0.0f && p <= 1.0f && aligned(offset_at, 8) && first_row >= 0 && rows >= 0 && rows <= ((int64_t)1 << 32) &&
           first_row <= ((int64_t)1 << 32) - rows && cols >= 0 && cols <= INT32_MAX;
}

inline Drop drop_of(float p, uint64_t seed, uint64_t offset, const int64_t *offset_at, int64_t first_row) {
    Drop d;
    d.key0 = (uint32_t)seed, d.key1 = (uint32_t)(seed >> 32);
    d.offset = offset, d.offset_at = offset_at, d.first_row = (uint32_t)first_row;
    d.threshold = (uint32_t)std::nearbyint((double)p * 65536.0);
    d.scale = d.threshold < 65536 ? (float)(65536.0 / (65536 - (int)d.threshold)) : 0.0f;
    return d;
}

__device__ __forceinline__ uint64_t drop_offset(const Drop &d) { return d.offset + (d.offset_at ? (uint64_t)*d.offset_at : 0); }

// The numbers of a row's eight columns from 8 `group` on.
struct Drop8 {
    uint32_t w[4];
    __device__ __forceinline__ Drop8(const Drop &d, uint64_t offset, uint32_t row, uint32_t group) {
        uint32_t c0 = group, c1 = d.first_row + row, c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
        uint32_t k0 = d.key0, k1 = d.key1;
#pragma unroll
        for (int i = 0; i < 10; i++) {
            const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
            c0 = (uint32_t)(b >> 32) ^ c1 ^ k0, c1 = (uint32_t)b;
            c2 = (uint32_t)(a >> 32) ^ c3 ^ k1, c3 = (uint32_t)a;
            k0 += 0x9E3779B9u, k1 += 0xBB67AE85u;
        }
        w[0] = c0, w[1] = c1, w[2] = c2, w[3] = c3;
    }
    __device__ __forceinline__ bool kept(int e, uint32_t threshold) const {
        return (e % 2 ? w[e / 2] >> 16 : w[e / 2] & 0xffffu) >= threshold;
    }
};

// The same for V of the columns from `col` on, a multiple of V.
template <int V>
struct DropV {
    uint32_t mask;  // bit e: the e-th stays
    __device__ __forceinline__ DropV(const Drop &d, uint64_t offset, uint32_t row, uint32_t col) {
        static_assert(V == 4 || V == 8, "");
        const Drop8 r(d, offset, row, col / 8);
        mask = 0;
        if constexpr (V == 8) {
#pragma unroll
            for (int e = 0; e < 8; e++) mask |= r.kept(e, d.threshold) ? 1u << e : 0u;
        } else {
            const bool high = col & 4;  // of the eight
            const uint32_t a = high ? r.w[2] : r.w[0], b = high ? r.w[3] : r.w[1];
            mask = ((a & 0xffffu) >= d.threshold ? 1u : 0u) | ((a >> 16) >= d.threshold ? 2u : 0u) |
                   ((b & 0xffffu) >= d.threshold ? 4u : 0u) | ((b >> 16) >= d.threshold ? 8u : 0u);
        }
    }
    __device__ __forceinline__ bool kept(int e) const { return mask >> e & 1; }
};

// A vector's values that lie in the row: `n` of V, the rest are `fill`.
template <typename T, int V>
__device__ __forceinline__ Words<T, V> get_some(const T *from, int n, float fill = 0.0f) {
    if (n >= V) return get_words<T, V>(from);
    float v[V];
#pragma unroll
    for (int e = 0; e < V; e++) v[e] = e < n ? (float)from[e] : fill;
    return Words<T, V>::of([&](int e) { return v[e]; });
}
template <typename T, int V>
__device__ __forceinline__ void put_some(T *to, int n, const Words<T, V> &v) {
    if (n >= V) return put_words(to, v);
#pragma unroll
    for (int e = 0; e < V; e++)
        if (e < n) to[e] = round_to<T>(v[e]);
}

}  // namespace byz_worker

#endif

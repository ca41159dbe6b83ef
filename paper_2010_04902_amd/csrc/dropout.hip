// Dropout whose mask is made where it is used (gfx950): y = x scale where a value stays, else 0.  Its gradient is the same call.
//
// Bound by memory: a value in, a value out; with 16-bit types the generator's ten rounds for eight values keep the vector units 0.69 of
// the time busy.  Groups of eight columns are numbered over rows and groups alike, so rows shorter than a wave leave no lanes idle; a
// thread does two.  Results go through the caches: stored past them 8192 x 16384 bf16 took 76 us alone, but 190 with an operation
// behind it that reads the result, for 90 and 179.
//
// 8192 x 16384 bf16 90 to 96 us (5.9 TB/s), fp32 191 to 237; 70000 x 1517 bf16, rows at odd addresses, 97 (4.4 TB/s); 30 x 512 3.1.
#include <algorithm>

#include "drop.h"

using namespace byz_worker;

namespace {

struct Args {
    const void *x;
    int64_t rows, cols, x_ld;
    void *y;
    int64_t y_ld;
    Drop drop;
    uint32_t groups;  // of a row
    double per_group;  // 1 / groups
    uint32_t magic;    // x / groups for x < 2^30: (x magic) >> shift
    int shift;
};

__device__ __forceinline__ uint32_t over_groups(const Args &a, uint32_t x) { return (uint32_t)((uint64_t)x * a.magic >> a.shift); }

constexpr int kThreads = 256, kEach = 2;  // groups a thread

// Row and group of a block's first: the quotient in fp64 is one off at most.
struct First {
    int64_t row, rest;
    __device__ __forceinline__ First(const Args &a, int64_t number) {
        row = (int64_t)((double)number * a.per_group), rest = number - row * a.groups;
        if (rest < 0) row--, rest += a.groups;
        if (rest >= a.groups) row++, rest -= a.groups;
    }
};

// 16-bit types: a group is a vector.
template <typename T>
__global__ __launch_bounds__(kThreads) void dropout_kernel(Args a) {
    const uint64_t offset = drop_offset(a.drop);
    const int64_t total = a.rows * (int64_t)a.groups;
    for (int64_t number = (int64_t)blockIdx.x * (kThreads * kEach); number < total; number += (int64_t)gridDim.x * (kThreads * kEach)) {
        const First first(a, number);
#pragma unroll
        for (int u = 0; u < kEach; u++) {
            const uint32_t local = (uint32_t)first.rest + u * kThreads + threadIdx.x;  // below 2^28 + 2^9
            const uint32_t down = over_groups(a, local), group = local - down * a.groups;
            const int64_t row = first.row + down;
            if (row >= a.rows) break;
            const T *from = (const T *)a.x + row * a.x_ld + (int64_t)group * 8;
            const int n = (int)std::min<int64_t>(a.cols - (int64_t)group * 8, 8);
            const Words<T, 8> v = get_some<T, 8>(from, n);
            const Drop8 r(a.drop, offset, (uint32_t)row, group);
            put_some<T, 8>((T *)a.y + row * a.y_ld + (int64_t)group * 8, n,
                           Words<T, 8>::of([&](int e) { return r.kept(e, a.drop.threshold) ? v[e] * a.drop.scale : 0.0f; }));
        }
    }
}

// fp32: a group is two vectors, of two neighbouring lanes, so that a wave's accesses are 1 KB without gaps.  A lane makes the numbers of
// one of two groups that are 32 apart, and the lanes of a pair exchange the halves they do not need.  (With both vectors of a
// group in one lane 8192 x 16384 took 315 us, half the rate of bf16.)
__global__ __launch_bounds__(kThreads) void dropout_pairs_kernel(Args a) {
    constexpr int V = 4;
    const uint64_t offset = drop_offset(a.drop);
    const int64_t total = a.rows * (int64_t)a.groups;
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const bool odd = lane & 1;
    for (int64_t number = (int64_t)blockIdx.x * (kThreads * kEach); number < total; number += (int64_t)gridDim.x * (kThreads * kEach)) {
        const First first(a, number);
#pragma unroll
        for (int u = 0; u < kEach; u++) {
            int64_t row[2], col[2];
            int n[2];
            Words<float, V> v[2];
#pragma unroll
            for (int k = 0; k < 2; k++) {
                const uint32_t local = (uint32_t)first.rest + (wave * kEach + u) * 64 + k * 32 + lane / 2;
                const uint32_t down = over_groups(a, local);
                row[k] = first.row + down, col[k] = (int64_t)(local - down * a.groups) * 8 + (odd ? V : 0);
                n[k] = row[k] < a.rows ? (int)std::max<int64_t>(0, std::min<int64_t>(a.cols - col[k], V)) : 0;
                if (n[k] > 0) v[k] = get_some<float, V>((const float *)a.x + row[k] * a.x_ld + col[k], n[k]);
            }
            const Drop8 r(a.drop, offset, (uint32_t)(odd ? row[1] : row[0]), (uint32_t)((odd ? col[1] : col[0]) / 8));
            const uint32_t given[2] = {odd ? r.w[0] : r.w[2], odd ? r.w[1] : r.w[3]};
            uint32_t taken[2];
#pragma unroll
            for (int i = 0; i < 2; i++) taken[i] = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)given[i], 0xB1, 0xf, 0xf, true);
#pragma unroll
            for (int k = 0; k < 2; k++) {
                const bool own = odd == (k == 1);
                const uint32_t w[2] = {own ? (odd ? r.w[2] : r.w[0]) : taken[0], own ? (odd ? r.w[3] : r.w[1]) : taken[1]};
                if (n[k] > 0)
                    put_some<float, V>((float *)a.y + row[k] * a.y_ld + col[k], n[k], Words<float, V>::of([&](int e) {
                                           return (e % 2 ? w[e / 2] >> 16 : w[e / 2] & 0xffffu) >= a.drop.threshold ? v[k][e] * a.drop.scale : 0.0f;
                                       }));
            }
        }
    }
}

int launch(Args a, int dtype, hipStream_t s) {
    const int64_t blocks = (a.rows * (int64_t)a.groups + kThreads * kEach - 1) / (kThreads * kEach);
    const unsigned grid = (unsigned)std::min<int64_t>(blocks, 1 << 20);
    int log = 0;
    while ((1u << log) < a.groups) log++;
    a.per_group = 1.0 / a.groups, a.shift = 30 + log;
    a.magic = (uint32_t)((((uint64_t)1 << a.shift) + a.groups - 1) / a.groups);
    if (dtype == BYZ_F32)
        dropout_pairs_kernel<<<grid, kThreads, 0, s>>>(a);
    else if (dtype == BYZ_BF16)
        dropout_kernel<bf16><<<grid, kThreads, 0, s>>>(a);
    else
        dropout_kernel<f16><<<grid, kThreads, 0, s>>>(a);
    BYZ_HIP(hipGetLastError());
    return BYZ_OK;
}

}  // namespace

extern "C" int byz_dropout(const void *x, int64_t rows, int64_t cols, int64_t x_ld, int dtype, float p, uint64_t seed,
                           uint64_t offset, const int64_t *offset_at, int64_t first_row, void *y, int64_t y_ld, void *stream) {
    if (!dtype_known(dtype) || !drop_ok(p, offset_at, first_row, rows, cols)) return BYZ_EINVAL;
    if (rows == 0 || cols == 0) return BYZ_OK;
    const size_t e = dtype_size(dtype);
    if (!x || !y || !aligned(x, e) || !aligned(y, e) || x_ld < cols || y_ld < cols || !extent_ok(rows, x_ld, cols) ||
        !extent_ok(rows, y_ld, cols))
        return BYZ_EINVAL;
    Args a{};
    a.x = x, a.rows = rows, a.cols = cols, a.x_ld = x_ld, a.y = y, a.y_ld = y_ld;
    a.drop = drop_of(p, seed, offset, offset_at, first_row), a.groups = (uint32_t)((cols + 7) / 8);
    return launch(a, dtype, (hipStream_t)stream);
}

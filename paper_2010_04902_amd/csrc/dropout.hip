// Dropout whose mask is made where it is used (gfx950): y = x scale where a value stays, else 0.  Its gradient is the same call.
//
// Bound by memory: a value in, a value out.  The generator's ten rounds for eight values take about half of the
// instruction slots that reading and writing eight bf16 values leave.  A thread does groups of eight columns, numbered over
// rows and groups alike, so rows shorter than a wave leave no lanes idle.
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
};

constexpr int kThreads = 256, kEach = 2;  // groups a thread

template <typename T>
__global__ __launch_bounds__(kThreads) void dropout_kernel(Args a) {
    const uint64_t offset = drop_offset(a.drop);
    const int64_t total = a.rows * (int64_t)a.groups;
    for (int64_t first = (int64_t)blockIdx.x * (kThreads * kEach); first < total; first += (int64_t)gridDim.x * (kThreads * kEach)) {
        // row and group of the block's first: the quotient in fp64 is one off at most
        int64_t row0 = (int64_t)((double)first * a.per_group), rest = first - row0 * a.groups;
        if (rest < 0) row0--, rest += a.groups;
        if (rest >= a.groups) row0++, rest -= a.groups;
#pragma unroll
        for (int u = 0; u < kEach; u++) {
            const int64_t number = first + u * kThreads + threadIdx.x;
            if (number >= total) break;
            const uint32_t local = (uint32_t)rest + u * kThreads + threadIdx.x;  // below 2^28 + 2^9
            const uint32_t down = local / a.groups, group = local - down * a.groups;
            const int64_t row = row0 + down;
            const T *from = (const T *)a.x + row * a.x_ld + (int64_t)group * 8;
            T *to = (T *)a.y + row * a.y_ld + (int64_t)group * 8;
            const Drop8 r(a.drop, offset, (uint32_t)row, group);
            constexpr int V = sizeof(T) == 2 ? 8 : 4;
#pragma unroll
            for (int h = 0; h < 8; h += V) {
                const int n = (int)std::min<int64_t>(a.cols - (int64_t)group * 8 - h, V);
                if (n <= 0) break;
                const Words<T, V> v = get_some<T, V>(from + h, n);
                put_some<T, V>(to + h, n, Words<T, V>::of([&](int e) { return r.kept(h + e, a.drop.threshold) ? v[e] * a.drop.scale : 0.0f; }));
            }
        }
    }
}

template <typename T>
int launch(const Args &a, hipStream_t s) {
    const int64_t blocks = (a.rows * (int64_t)a.groups + kThreads * kEach - 1) / (kThreads * kEach);
    dropout_kernel<T><<<(unsigned)std::min<int64_t>(blocks, 1 << 20), kThreads, 0, s>>>(a);
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
    const uint32_t groups = (uint32_t)((cols + 7) / 8);
    const Args a{x, rows, cols, x_ld, y, y_ld, drop_of(p, seed, offset, offset_at, first_row), groups, 1.0 / groups};
    const hipStream_t s = (hipStream_t)stream;
    return dtype == BYZ_F32 ? launch<float>(a, s) : dtype == BYZ_BF16 ? launch<bf16>(a, s) : launch<f16>(a, s);
}

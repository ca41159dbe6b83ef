// A block's output joins the residual: norm, dropout, gate and scale on the way in, and the norm in front of the next block
// (gfx950).
//
//     u = norm(h) w1 + b1,  t = x + s g drop(u),  y = norm(t) w2 + b2
// The gradients make t again from x and h instead of reading it rounded, so both passes see the same sums.  With
// a = dy w2, means over a row, and the mean of a alone for the layer norm only,
//     dt = dout + rstd2 (a - mean a - tn mean(a tn)),  du = s g drop(dt),  dx = dt
//     dh = rstd1 (b - mean b - hn mean(b hn)),  b = du w1
//     dw2 = sum dy tn,  db2 = sum dy,  dw1 = sum du hn,  db1 = sum du,  dg = sum s drop(u) dt
//
// Bound by memory where rows are many: four tensors forward, six backward, each once.  Rows of 8 to 8192 columns (16384 forward) are held
// in registers, eight columns a thread, which is one call of the generator: a row is part of a wave, a wave, or up to 1024 threads.
// Backward a thread also sums its columns over the rows of its block; the blocks' sums are joined by finish_kernel.  Narrower and wider
// rows, and gates of a few rows each on more than 4096 columns, take kernels that read a row up to three times (once up to 16384 columns of
// 16 bits, root mean squares) and the columns' sums by a second reading.  Short calls are bound by one row's chain (2 us, two reductions); code
// counts there: with partial vectors unrolled a backward kernel of 15 KB took 13 us for one row; of half that length it takes 11 for two.
//
// 8192 x 4096 bf16, both norms RMS, gate and dropout: forward 48 to 53 us (5.6 TB/s, vector units busy 0.61), backward 91 (4.7 TB/s with the blocks'
// sums, busy 0.57) and 6 for the join; with layer norms and biases 67 and 106 together.  1920 x 512 4.8, 10 and 5.
#include <algorithm>

#include "drop.h"

using namespace byz_worker;

namespace {

constexpr int64_t kMaxGrid = 1 << 20;
constexpr int kCus = 256;  // compute units

struct Args {
    const void *x, *h;
    int64_t x_ld, h_ld, rows, cols;
    int post, pre;
    float eps, scale;
    const float *w1, *b1, *gate, *w2, *b2;
    int64_t gate_rows;
    Drop drop;
    void *out, *y;
    int64_t out_ld, y_ld;
    float *stats;
};

// Which of gate's rows row has; there are 2^32 rows at most.
__device__ __forceinline__ int64_t group_of(const Args &a, int64_t row) {
    return row < a.gate_rows ? 0 : (int64_t)((uint32_t)row / (uint32_t)a.gate_rows);
}

struct Back {
    const void *dout, *dy;
    int64_t dout_ld, dy_ld;
    const float *stats;
    void *dx, *dh;
    int64_t dx_ld, dh_ld;
    float *rest;      // of each row: mean a, mean a tn, mean b, mean b hn
    float *partials;  // [chunk][kind][column]
    float *d_gate;
    uint32_t kinds;     // bit k: kind k is wanted
    uint32_t chunks, per_group;  // per_group: of a group of gate's rows; 0: a chunk has whole groups
    int64_t groups;
};
enum { kW2, kB2, kW1, kB1, kGate, kKinds };

// Sums over the NT threads of a row in a fixed order; every thread gets them.  Two buffers, so that one barrier is enough.
template <int NT>
struct Joiner {
    static constexpr int waves = NT / 64;
    float2 *lds;  // 2 * waves
    int turn = 0;
    __device__ explicit Joiner(float2 *l) : lds(l) {}
    __device__ __forceinline__ float2 sum(float a, float b) {
        auto add = [](float2 p, const float2 &q) { return make_float2(p.x + q.x, p.y + q.y); };
        float2 v = wave_reduce(make_float2(a, b), add);
        if constexpr (waves > 1) {
            float2 *at = lds + turn * waves;
            turn ^= 1;
            if (threadIdx.x % 64 == 0) at[threadIdx.x / 64] = v;
            __syncthreads();
            v = make_float2(0.0f, 0.0f);
#pragma unroll
            for (int w = 0; w < waves; w++) v = add(v, at[w]);
        }
        return v;
    }
};

// V columns of a vector of parameters; 0 beyond the row's end.
template <int V>
__device__ __forceinline__ void parameters(const float *p, int64_t col, int n, float none, float (&v)[V]) {
    if (p && n >= V) {
        const auto w = get_words<float, V>(p + col);
#pragma unroll
        for (int e = 0; e < V; e++) v[e] = w[e];
    } else {
#pragma unroll
        for (int e = 0; e < V; e++) v[e] = e >= n ? 0.0f : p ? p[col + e] : none;
    }
}

struct Stats {
    float mean1 = 0.0f, rstd1 = 1.0f, mean2 = 0.0f, rstd2 = 1.0f;
};

// V columns of a row: what the block gives, dropped, and the sum.
template <typename T, int V>
struct Piece {
    float hn[V], v[V], sg[V], t[V];  // normalised h; drop(u); scale * gate; the sum
    uint32_t kept;
    __device__ __forceinline__ Piece(const Args &a, const Stats &s, uint64_t offset, int64_t row, int64_t col, int n) {
        const auto x = get_some<T, V>((const T *)a.x + row * a.x_ld + col, n);
        if (!a.h) {
#pragma unroll
            for (int e = 0; e < V; e++) hn[e] = v[e] = sg[e] = 0.0f, t[e] = x[e];
            kept = 0;
            return;
        }
        const auto h = get_some<T, V>((const T *)a.h + row * a.h_ld + col, n);
        float w1[V], b1[V];
        parameters<V>(a.w1, col, n, 1.0f, w1);
        parameters<V>(a.b1, col, n, 0.0f, b1);
        parameters<V>(a.gate ? a.gate + group_of(a, row) * a.cols : nullptr, col, n, 1.0f, sg);
        kept = a.drop.threshold ? DropV<V>(a.drop, offset, (uint32_t)row, (uint32_t)col).mask : ~0u;
#pragma unroll
        for (int e = 0; e < V; e++) {
            // without a norm, whose sums it would be in, what is dropped may be no number: it is in no product below
            hn[e] = a.post == BYZ_NORM_NONE && !(kept >> e & 1) ? 0.0f : (h[e] - s.mean1) * s.rstd1;
            v[e] = kept >> e & 1 ? fmaf(hn[e], w1[e], b1[e]) * a.drop.scale : 0.0f;
            sg[e] *= a.scale;
            t[e] = e < n ? fmaf(sg[e], v[e], x[e]) : 0.0f;
        }
    }
};

// The gradient of the sum and of u at V columns.
template <typename T, int V>
struct Gradients {
    float dy[V], tn[V], dt[V], du[V];
    __device__ __forceinline__ Gradients(const Args &a, const Back &b, const Stats &s, const Piece<T, V> &p, float mean_a, float mean_atn,
                                         int64_t row, int64_t col, int n) {
        float dout[V], w2[V];
#pragma unroll
        for (int e = 0; e < V; e++) dout[e] = dy[e] = 0.0f;
        if (b.dout) {
            const auto w = get_some<T, V>((const T *)b.dout + row * b.dout_ld + col, n);
#pragma unroll
            for (int e = 0; e < V; e++) dout[e] = w[e];
        }
        if (b.dy) {
            const auto w = get_some<T, V>((const T *)b.dy + row * b.dy_ld + col, n);
#pragma unroll
            for (int e = 0; e < V; e++) dy[e] = w[e];
        }
        parameters<V>(a.w2, col, n, 1.0f, w2);
#pragma unroll
        for (int e = 0; e < V; e++) {
            tn[e] = (p.t[e] - s.mean2) * s.rstd2;
            dt[e] = b.dy ? dout[e] + s.rstd2 * (dy[e] * w2[e] - mean_a - tn[e] * mean_atn) : dout[e];
            du[e] = p.kept >> e & 1 ? p.sg[e] * a.drop.scale * dt[e] : 0.0f;
        }
    }
};

template <typename T, int NT>
__global__ __launch_bounds__(NT) void forward_kernel(Args a) {
    constexpr int V = 16 / sizeof(T);
    __shared__ float2 lds[2 * NT / 64];
    Joiner<NT> join(lds);
    const uint64_t offset = drop_offset(a.drop);
    const float inv = 1.0f / (float)a.cols;
    auto over = [&](auto f) {
        for (int64_t col = (int64_t)threadIdx.x * V; col < a.cols; col += NT * V) f(col, (int)std::min<int64_t>(V, a.cols - col));
    };
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        Stats s;
        auto moments = [&](int kind, float &mean, float &rstd, auto value) {
            if (kind == BYZ_NORM_NONE) return;
            float sum = 0.0f;
            if (kind == BYZ_NORM_LAYER) {
                over([&](int64_t col, int n) { value(col, n, [&](int e, float v) { sum += v; }); });
                mean = join.sum(sum, 0.0f).x * inv;
                sum = 0.0f;
            }
            over([&](int64_t col, int n) {
                value(col, n, [&](int e, float v) { sum += e < n ? (v - mean) * (v - mean) : 0.0f; });
            });
            rstd = 1.0f / sqrtf(join.sum(sum, 0.0f).x * inv + a.eps);
        };
        if (a.h)
            moments(a.post, s.mean1, s.rstd1, [&](int64_t col, int n, auto f) {
                const auto h = get_some<T, V>((const T *)a.h + row * a.h_ld + col, n);
#pragma unroll
                for (int e = 0; e < V; e++) f(e, h[e]);
            });
        moments(a.pre, s.mean2, s.rstd2, [&](int64_t col, int n, auto f) {
            const Piece<T, V> p(a, s, offset, row, col, n);
#pragma unroll
            for (int e = 0; e < V; e++) f(e, p.t[e]);
        });
        over([&](int64_t col, int n) {
            const Piece<T, V> p(a, s, offset, row, col, n);
            if (a.out && a.h) put_some<T, V>((T *)a.out + row * a.out_ld + col, n, Words<T, V>::of([&](int e) { return p.t[e]; }));
            if (a.pre == BYZ_NORM_NONE) return;
            float w2[V], b2[V];
            parameters<V>(a.w2, col, n, 1.0f, w2);
            parameters<V>(a.b2, col, n, 0.0f, b2);
            put_some<T, V>((T *)a.y + row * a.y_ld + col, n,
                           Words<T, V>::of([&](int e) { return fmaf((p.t[e] - s.mean2) * s.rstd2, w2[e], b2[e]); }));
        });
        if (a.stats && threadIdx.x == 0) {
            float *at = a.stats + row * 4;
            at[0] = s.mean1, at[1] = s.rstd1, at[2] = s.mean2, at[3] = s.rstd2;
        }
    }
}

__device__ __forceinline__ Stats stats_of(const float *stats, int64_t row) {
    Stats s;
    s.mean1 = stats[row * 4], s.rstd1 = stats[row * 4 + 1], s.mean2 = stats[row * 4 + 2], s.rstd2 = stats[row * 4 + 3];
    return s;
}

// dx and dh, and the means of each row that the columns' kernel needs.
template <typename T, int NT>
__global__ __launch_bounds__(NT) void rows_kernel(Args a, Back b) {
    constexpr int V = 16 / sizeof(T);
    __shared__ float2 lds[2 * NT / 64];
    Joiner<NT> join(lds);
    const uint64_t offset = drop_offset(a.drop);
    const float inv = 1.0f / (float)a.cols;
    const float inv_a = a.pre == BYZ_NORM_LAYER ? inv : 0.0f, inv_b = a.post == BYZ_NORM_LAYER ? inv : 0.0f;
    const float inv_atn = a.pre != BYZ_NORM_NONE ? inv : 0.0f, inv_bhn = a.post != BYZ_NORM_NONE ? inv : 0.0f;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const Stats s = stats_of(b.stats, row);
        float mean_a = 0.0f, mean_atn = 0.0f, mean_b = 0.0f, mean_bhn = 0.0f;
        auto over = [&](auto f) {
            for (int64_t col = (int64_t)threadIdx.x * V; col < a.cols; col += NT * V) {
                const int n = (int)std::min<int64_t>(V, a.cols - col);
                const Piece<T, V> p(a, s, offset, row, col, n);
                f(p, Gradients<T, V>(a, b, s, p, mean_a, mean_atn, row, col, n), col, n);
            }
        };
        if (a.pre != BYZ_NORM_NONE && b.dy) {
            float p1 = 0.0f, p2 = 0.0f;
            over([&](const Piece<T, V> &, const Gradients<T, V> &g, int64_t col, int n) {
                float w2[V];
                parameters<V>(a.w2, col, n, 1.0f, w2);
#pragma unroll
                for (int e = 0; e < V; e++) p1 += g.dy[e] * w2[e], p2 += g.dy[e] * w2[e] * g.tn[e];
            });
            const float2 r = join.sum(p1, p2);
            mean_a = r.x * inv_a, mean_atn = r.y * inv_atn;
        }
        if (a.h && a.post != BYZ_NORM_NONE) {
            float p3 = 0.0f, p4 = 0.0f;
            over([&](const Piece<T, V> &p, const Gradients<T, V> &g, int64_t col, int n) {
                float w1[V];
                parameters<V>(a.w1, col, n, 1.0f, w1);
#pragma unroll
                for (int e = 0; e < V; e++) p3 += g.du[e] * w1[e], p4 += g.du[e] * w1[e] * p.hn[e];
            });
            const float2 r = join.sum(p3, p4);
            mean_b = r.x * inv_b, mean_bhn = r.y * inv_bhn;
        }
        over([&](const Piece<T, V> &p, const Gradients<T, V> &g, int64_t col, int n) {
            put_some<T, V>((T *)b.dx + row * b.dx_ld + col, n, Words<T, V>::of([&](int e) { return g.dt[e]; }));
            if (!a.h) return;
            float w1[V];
            parameters<V>(a.w1, col, n, 1.0f, w1);
            put_some<T, V>((T *)b.dh + row * b.dh_ld + col, n,
                           Words<T, V>::of([&](int e) {
                               const float v = g.du[e] * w1[e];
                               return a.post == BYZ_NORM_NONE ? v : s.rstd1 * (v - mean_b - p.hn[e] * mean_bhn);
                           }));
        });
        if (threadIdx.x == 0) {
            float *at = b.rest + row * 4;
            at[0] = mean_a, at[1] = mean_atn, at[2] = mean_b, at[3] = mean_bhn;
        }
    }
}

// Sums over a chunk's rows, four waves with a row each in turn and 64 V columns a wave.  A group of gate's rows is dealt out to
// per_group chunks, row by row, so that the chunks are at neighbouring rows at any time (with runs of neighbouring rows for each they would
// be a power of two apart, in a few of the memory's channels); or a chunk has whole groups, which a wave takes whole: their
// d_gate is written here.
template <typename T>
__global__ __launch_bounds__(256) void columns_kernel(Args a, Back b) {
    constexpr int V = 16 / sizeof(T), W = 4;
    __shared__ float lds[W][64 * V];
    const uint64_t offset = drop_offset(a.drop);
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t col = ((int64_t)blockIdx.x * 64 + lane) * V;
    const int n = (int)std::max<int64_t>(0, std::min<int64_t>(V, a.cols - col));
    const int64_t chunk = blockIdx.y, group_rows = a.gate ? a.gate_rows : a.rows;
    float acc[kKinds][V] = {};
    auto add = [&](int64_t row) {
        if (n == 0) return;
        const Stats s = stats_of(b.stats, row);
        const Piece<T, V> p(a, s, offset, row, col, n);
        const Gradients<T, V> g(a, b, s, p, b.rest[row * 4], b.rest[row * 4 + 1], row, col, n);
#pragma unroll
        for (int e = 0; e < V; e++) {
            acc[kW2][e] += g.dy[e] * g.tn[e], acc[kB2][e] += g.dy[e];
            acc[kW1][e] += g.du[e] * p.hn[e], acc[kB1][e] += g.du[e];
            acc[kGate][e] += a.scale * p.v[e] * g.dt[e];
        }
    };
    if (b.per_group) {
        const uint32_t group = blockIdx.y / b.per_group;
        const int64_t end = std::min((group + 1) * group_rows, a.rows);
        for (int64_t row = group * group_rows + blockIdx.y % b.per_group * W + wave; row < end; row += b.per_group * W) add(row);
    } else {
        for (int64_t group = chunk * W + wave; group < b.groups; group += b.chunks * W) {
            const int64_t end = std::min((group + 1) * group_rows, a.rows);
            for (int64_t row = group * group_rows; row < end; row++) add(row);
#pragma unroll
            for (int e = 0; e < V; e++) {
                if (b.d_gate && e < n) b.d_gate[group * a.cols + col + e] = acc[kGate][e];
                acc[kGate][e] = 0.0f;
            }
        }
    }
    int at = 0;
#pragma unroll
    for (int k = 0; k < kKinds; k++) {
        if (!(b.kinds >> k & 1)) continue;
        __syncthreads();
#pragma unroll
        for (int e = 0; e < V; e++) lds[wave][lane * V + e] = acc[k][e];
        __syncthreads();
        for (int i = threadIdx.x; i < 64 * V; i += 256) {
            const int64_t c = (int64_t)blockIdx.x * 64 * V + i;
            if (c < a.cols)
                b.partials[(chunk * __builtin_popcount(b.kinds) + at) * a.cols + c] = (lds[0][i] + lds[1][i]) + (lds[2][i] + lds[3][i]);
        }
        at++;
    }
}

// ------------------------------------------------------------------ rows in registers

// Sums over the TPR threads of a row: part of a wave, a wave, or several, of which a block may have more than one such row.
template <int TPR, int SLOTS>
struct RowJoiner {
    static constexpr int waves = TPR / 64, places = waves > 8 ? 16 : waves > 4 ? 8 : waves > 2 ? 4 : 2;
    static constexpr int size = waves > 1 ? 2 * places * SLOTS : 1;
    float2 *lds;
    int turn = 0;
    // starts with a barrier where rows have several waves: they may have fewer than there are places
    __device__ explicit RowJoiner(float2 *l) : lds(l) {
        if constexpr (waves > 1) {
            if (threadIdx.x < size) lds[threadIdx.x] = make_float2(0.0f, 0.0f);
            lds += SLOTS > 1 ? (int)threadIdx.x / TPR * (2 * places) : 0;
            __syncthreads();
        }
    }
    // over 2^LANES lanes that lie together; every one gets the same bits
    template <int LANES>
    static __device__ __forceinline__ float2 lanes(float2 v) {
        auto step = [&](auto k) {
            if constexpr (k.value < LANES) {
                float2 p, q;
                wave_pair<k.value>(v, p, q);
                v = make_float2(p.x + q.x, p.y + q.y);
            }
        };
        wave_steps(1, step);
        return v;
    }
    __device__ __forceinline__ float2 sum(float a, float b) {
        constexpr int own = TPR >= 64 ? 6 : TPR == 32 ? 5 : TPR == 16 ? 4 : 2;
        float2 v = make_float2(a, b);
        if constexpr (TPR == 8) {  // the eight lanes' mirror image; their halves then have the same four sums
            v.x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v.x), 0x141, 0xf, 0xf, true));
            v.y += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v.y), 0x141, 0xf, 0xf, true));
        }
        v = lanes<own>(v);
        if constexpr (waves > 1) {
            float2 *at = lds + turn * places;
            turn ^= 1;
            if (threadIdx.x % 64 == 0) at[threadIdx.x % TPR / 64] = v;
            __syncthreads();
            v = lanes<places == 16 ? 4 : places == 8 ? 3 : places == 4 ? 2 : 1>(at[threadIdx.x % places]);
        }
        return v;
    }
};

constexpr int kCols = 8;  // columns of a thread: one call of the generator

// Threads of a block that has rows of TPR threads: forward, and backward, where a block's rows share what it writes of its sums
// (3950 x 1024 bf16, layer norm, with one row a block: 31.7 us).
template <int TPR>
constexpr int block_of() {
    return TPR <= 64 ? 256 : TPR;
}
template <int TPR>
constexpr int back_block_of() {
    return TPR <= 64 ? 256 : TPR == 192 ? 384 : TPR <= 256 ? 512 : TPR;
}
// The threads it is launched with: where it has one row, the waves that this needs (3674 x 5240 fp16, forward, with all 1024: 58 us
// for 33).
template <int TPR, int NT>
int threads_of(int64_t cols) {
    return NT > TPR ? NT : (int)((cols + 64 * kCols - 1) / (64 * kCols)) * 64;
}

// Which of a block's rows a thread is at: a number that the compiler knows to be a wave's where it is.
template <int TPR, int NT>
__device__ __forceinline__ int slot_of() {
    if constexpr (NT == TPR) return 0;
    const int slot = threadIdx.x / TPR;
    return TPR >= 64 ? __builtin_amdgcn_readfirstlane(slot) : slot;
}

// A vector's values from the `skip`-th on.  The few are stored one by one in a loop: unrolled, with a branch for each, a kernel's
// code would be half as long again, and a short call is bound by reading its code.
template <typename T, int V>
__device__ __forceinline__ void put_from(T *to, int skip, const Words<T, V> &v) {
    if (skip == 0) return put_words(to, v);
    Words<T, V> w = v;
#pragma unroll 1
    for (int e = 0; e < V; e++) {
        if (e >= skip) to[e] = __builtin_bit_cast(Pack<T, 4 / sizeof(T)>, (uint32_t)w.w[0]).v[0];
#pragma unroll
        for (int i = 0; i < w.N; i++) {
            const uint32_t next = i + 1 < w.N ? (uint32_t)w.w[i + 1] : 0;
            w.w[i] = sizeof(T) == 4 ? next : (uint32_t)__builtin_amdgcn_alignbit(next, w.w[i], 16);
        }
    }
}

// A thread's eight columns.  The vector of a row's last thread ends with the row, so its first `skip` columns are those of the
// thread before it; threads beyond have nothing but such columns.  They are read, but in no sum, and not written.
template <int TPR>
struct Columns {
    int first, skip, number;  // number: of the generator's group
    __device__ __forceinline__ explicit Columns(int64_t cols, int vector = 0) {  // the thread's vector of that number
        const int own = vector * TPR + threadIdx.x % TPR;
        first = std::min(own * kCols, (int)cols - kCols);
        skip = std::min(own * kCols - first, kCols);
        number = std::min(own, ((int)cols - 1) / kCols);
    }
    // The address is a row's, which a wave shares, and 32 bits of a thread's own, made afresh: six tensors' whole addresses kept
    // over the rows would take twelve registers.
    template <typename T>
    __device__ __forceinline__ T *at(const void *base, int64_t row, int64_t ld) const {
        return (T *)((char *)((T *)base + row * ld) + (uint32_t)afresh(first) * (uint32_t)sizeof(T));
    }
    template <typename T>
    __device__ __forceinline__ Words<T, kCols> get(const void *base, int64_t row, int64_t ld) const {
        return get_words<T, kCols>(at<T>(base, row, ld));
    }
    // zeros for the columns that are skipped
    template <typename T>
    __device__ __forceinline__ void only_own(Words<T, kCols> &w) const {
        if (skip == 0) return;
        const Words<T, kCols> v = w;
        w = Words<T, kCols>::of([&](int e) { return e >= skip ? v[e] : 0.0f; });
    }
    template <typename T>
    __device__ __forceinline__ void put(void *base, int64_t row, int64_t ld, const Words<T, kCols> &w) const {
        put_from(at<T>(base, row, ld), skip, w);
    }
    __device__ __forceinline__ void parameters_of(const float *p, float none, float (&v)[kCols]) const {
        if (p) {
            const auto w = get_words<float, kCols>(p + first);
#pragma unroll
            for (int e = 0; e < kCols; e++) v[e] = w[e];
        } else {
#pragma unroll
            for (int e = 0; e < kCols; e++) v[e] = none;
        }
    }
    // 1 where a column is the thread's own and stays
    __device__ __forceinline__ void kept(const Args &a, uint64_t offset, int64_t row, float (&keep)[kCols]) const {
        if (a.drop.threshold) {
            const Drop8 r(a.drop, offset, (uint32_t)row, (uint32_t)number);
#pragma unroll
            for (int e = 0; e < kCols; e++) keep[e] = r.kept(e, a.drop.threshold) ? 1.0f : 0.0f;
        } else {
#pragma unroll
            for (int e = 0; e < kCols; e++) keep[e] = 1.0f;
        }
#pragma unroll 1
        for (int i = 0; i < skip; i++) {  // the group's columns are the vector's last ones
#pragma unroll
            for (int e = kCols - 1; e > 0; e--) keep[e] = keep[e - 1];
            keep[0] = 0.0f;
        }
    }
};

// What is dropped is multiplied by 0 below.  Without a norm of h, whose sums it would be in, a value that is not finite is
// not to reach anything from there: it is 0 from the start.
template <typename T>
__device__ __forceinline__ void drop_first(const Args &a, Words<T, kCols> &h, const float (&keep)[kCols]) {
    if (a.post != BYZ_NORM_NONE || !a.drop.threshold) return;
    const Words<T, kCols> v = h;
    h = Words<T, kCols>::of([&](int e) { return keep[e] != 0.0f ? v[e] : 0.0f; });
}

// What a block's normalised output is multiplied by on its way into the sum, and the bias on that way: scale, gate, weight and
// dropout's scale are one factor, for a group of gate's rows.
template <int TPR, bool GENERAL>
struct Way {
    float w[kCols], b[kCols];
    __device__ __forceinline__ Way() {}
    __device__ __forceinline__ Way(const Args &a, const Columns<TPR> &mine, int64_t group) {
        float g[kCols];
        mine.parameters_of(a.gate ? a.gate + group * a.cols : nullptr, 1.0f, g);
        mine.parameters_of(a.w1, 1.0f, w);
        if constexpr (GENERAL) mine.parameters_of(a.b1, 0.0f, b);
#pragma unroll
        for (int e = 0; e < kCols; e++) {
            g[e] *= a.scale * a.drop.scale, w[e] *= g[e];
            if constexpr (GENERAL) b[e] *= g[e];
        }
    }
    __device__ __forceinline__ float of(int e, float normal) const { return GENERAL ? fmaf(normal, w[e], b[e]) : normal * w[e]; }
};

// R times eight columns of a row to each of TPR threads.  GENERAL: means and biases; without, there are none.
template <typename T, int TPR, int R, bool GENERAL>
__global__ __launch_bounds__(block_of<TPR>(), 4) void forward_rows_kernel(Args a) {
    constexpr int V = kCols, NT = block_of<TPR>(), SLOTS = NT / TPR;
    __shared__ float2 lds[RowJoiner<TPR, SLOTS>::size];
    RowJoiner<TPR, SLOTS> join(lds);
    auto mine = [&](int r) __attribute__((always_inline)) { return Columns<TPR>(a.cols, r); };
    const uint64_t offset = drop_offset(a.drop);
    const float inv = 1.0f / (float)a.cols;
    float w2[R][V], b2[R][V];
    Way<TPR, GENERAL> way[R];
    constexpr bool HELD = R == 1 || !GENERAL;  // the second norm's parameters fit into the registers too
    auto second = [&](int r) __attribute__((always_inline)) {
        mine(r).parameters_of(a.w2, 1.0f, w2[r]);
        if constexpr (GENERAL) mine(r).parameters_of(a.b2, 0.0f, b2[r]);
    };
    if constexpr (HELD) {
#pragma unroll
        for (int r = 0; r < R; r++) second(r);
    }
    int64_t group_end = 0;
    for (int64_t row = (int64_t)blockIdx.x * SLOTS + slot_of<TPR, NT>(); row < a.rows; row += (int64_t)gridDim.x * SLOTS) {
        Words<T, V> x[R], h[R] = {};
#pragma unroll
        for (int r = 0; r < R; r++) {
            x[r] = mine(r).template get<T>(a.x, row, a.x_ld);
            if (a.h) h[r] = mine(r).template get<T>(a.h, row, a.h_ld);
            mine(r).only_own(x[r]), mine(r).only_own(h[r]);
        }
        if (row >= group_end) {
            const int64_t group = group_of(a, row);
#pragma unroll
            for (int r = 0; r < R; r++) way[r] = Way<TPR, GENERAL>(a, mine(r), group);
            group_end = (group + 1) * a.gate_rows;
        }
        Stats s;
        float t[R][V];
        // the mean of rows of the layer norm first, then that of the squares about it
        auto moments = [&](int kind, float &mean, float &rstd, auto value) __attribute__((always_inline)) {
            float sum = 0.0f;
            if (GENERAL && kind == BYZ_NORM_LAYER) {
#pragma unroll
                for (int r = 0; r < R; r++)
#pragma unroll
                    for (int e = 0; e < V; e++) sum += value(r, e);
                mean = join.sum(sum, 0.0f).x * inv;
                sum = 0.0f;
#pragma unroll
                for (int r = 0; r < R; r++)
#pragma unroll
                    for (int e = 0; e < V; e++) {
                        const float d = value(r, e) - mean;
                        sum += e >= mine(r).skip ? d * d : 0.0f;
                    }
            } else {
#pragma unroll
                for (int r = 0; r < R; r++)
#pragma unroll
                    for (int e = 0; e < V; e++) sum = fmaf(value(r, e), value(r, e), sum);
            }
            rstd = 1.0f / sqrtf(join.sum(sum, 0.0f).x * inv + a.eps);
        };
        if (a.h) {
            float keep[R][V];
#pragma unroll
            for (int r = 0; r < R; r++) {
                mine(r).kept(a, offset, row, keep[r]);
                drop_first(a, h[r], keep[r]);
            }
            if (a.post != BYZ_NORM_NONE) moments(a.post, s.mean1, s.rstd1, [&](int r, int e) { return h[r][e]; });
#pragma unroll
            for (int r = 0; r < R; r++) {
#pragma unroll
                for (int e = 0; e < V; e++)
                    t[r][e] = fmaf(way[r].of(e, GENERAL ? (h[r][e] - s.mean1) * s.rstd1 : h[r][e] * s.rstd1), keep[r][e], x[r][e]);
                mine(r).template put<T>(a.out, row, a.out_ld, Words<T, V>::of([&](int e) { return t[r][e]; }));
            }
        } else {
#pragma unroll
            for (int r = 0; r < R; r++)
#pragma unroll
                for (int e = 0; e < V; e++) t[r][e] = x[r][e];
        }
        if (a.pre != BYZ_NORM_NONE) {
            moments(a.pre, s.mean2, s.rstd2, [&](int r, int e) { return t[r][e]; });
#pragma unroll
            for (int r = 0; r < R; r++) {
                if constexpr (!HELD) second(r);
                mine(r).template put<T>(a.y, row, a.y_ld, Words<T, V>::of([&](int e) {
                                            return GENERAL ? fmaf((t[r][e] - s.mean2) * s.rstd2, w2[r][e], b2[r][e]) : t[r][e] * s.rstd2 * w2[r][e];
                                        }));
            }
        }
        if (a.stats && threadIdx.x % TPR == 0) {
            float *at = a.stats + row * 4;
            at[0] = s.mean1, at[1] = s.rstd1, at[2] = s.mean2, at[3] = s.rstd2;
        }
    }
}

// Waves of a SIMD that the registers of backward_rows_kernel are to leave room for: four where that costs few spills or none.  us at
// four and at two: 8192 x 4096 bf16 with layer norms 106 and 127.
template <typename T>
constexpr int back_waves(int tpr, bool general, bool part) {
    return tpr == 1024 || (sizeof(T) == 2 && (part || !general)) || (part && !general) ? 4 : 2;
}

// dx and dh of a chunk's rows, and the chunk's sums of the columns: a thread has eight columns of every row of its slot, whose
// sums stay in its registers.  Chunks are those of columns_kernel.  Over a group of gate's rows
//     A = sum drop(dt) hn,  B = sum drop(dt)   give   dw1 = s g A,  db1 = s g B,  dg = s (w1 A + b1 B).
template <typename T, int TPR, bool GENERAL, bool PART>
__global__ __launch_bounds__(back_block_of<TPR>(), back_waves<T>(TPR, GENERAL, PART)) void backward_rows_kernel(Args a, Back b) {
    constexpr int V = kCols, NT = back_block_of<TPR>(), SLOTS = NT / TPR;
    constexpr bool PACE = SLOTS > 1 && TPR > 64;  // barriers, at which all slots of the block meet
    __shared__ float2 lds[RowJoiner<TPR, SLOTS>::size];
    extern __shared__ float room[];
    RowJoiner<TPR, SLOTS> join(lds);
    const Columns<TPR> mine(a.cols);
    const uint64_t offset = drop_offset(a.drop);
    const float inv = 1.0f / (float)a.cols;
    const float inv_a = a.pre == BYZ_NORM_LAYER ? inv : 0.0f, inv_b = a.post == BYZ_NORM_LAYER ? inv : 0.0f;
    const int slot = slot_of<TPR, NT>();
    float sum_w2[V] = {}, sum_b2[V] = {}, sum_a[V] = {}, sum_b[V] = {}, bias[V];
    // A thread's own weights in LDS, read where they are used: in registers they would take sixteen.
    enum { kWay, kPre };
    auto store = [&](int which, const float (&v)[V]) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < V; e++) room[((which * 2 + e / 4) * NT + threadIdx.x) * 4 + e % 4] = v[e];
    };
    auto fetch = [&](int which, float (&v)[V]) __attribute__((always_inline)) {
        const int at = afresh((int)threadIdx.x);
#pragma unroll
        for (int q = 0; q < 2; q++) {
            const float4 w = *(const float4 *)&room[((which * 2 + q) * NT + at) * 4];
            v[q * 4] = w.x, v[q * 4 + 1] = w.y, v[q * 4 + 2] = w.z, v[q * 4 + 3] = w.w;
        }
    };
    {
        float w2[V];
        mine.parameters_of(a.w2, 1.0f, w2);
        store(kPre, w2);
    }
    struct Loaded {
        Words<T, V> x, h, dout, dy;
        Stats s;
    };
    // What is absent is read from x and set to zero in use: with loads that may not be made, waiting for one is waiting for all.
    const void *const h_at = a.h ? a.h : a.x, *const dy_at = b.dy ? b.dy : a.x, *const dout_at = b.dout ? b.dout : a.x;
    const int64_t h_ld = a.h ? a.h_ld : a.x_ld, dy_ld = b.dy ? b.dy_ld : a.x_ld, dout_ld = b.dout ? b.dout_ld : a.x_ld;
    auto load = [&](int64_t row) __attribute__((always_inline)) {
        Loaded l;
        l.s = stats_of(b.stats, row);
        l.h = mine.template get<T>(h_at, row, h_ld);
        l.x = mine.template get<T>(a.x, row, a.x_ld);
        l.dy = mine.template get<T>(dy_at, row, dy_ld);
        l.dout = mine.template get<T>(dout_at, row, dout_ld);
        return l;
    };
    // The row that l has; the next one is loaded meanwhile.  Of a row that is not the slot's (its waves only keep pace with those of
    // others) nothing is in a sum or written.
    auto work = [&](Loaded &l, int64_t row, int64_t next, bool active) __attribute__((always_inline)) {
        const Words<T, V> x = l.x;
        Words<T, V> h = l.h, dout = l.dout, dy = l.dy;
        const Stats s = l.s;
        l = load(next);
        float keep[V], tn[V], w2[V], way[V];
        fetch(kWay, way), fetch(kPre, w2);
        mine.kept(a, offset, row, keep);
        if (!b.dy || (PACE && !active)) dy = {};
        if (!b.dout) dout = {};
        if (!a.h) h = {};
        mine.only_own(dy);
        if (PACE && !active)
#pragma unroll
            for (int e = 0; e < V; e++) keep[e] = 0.0f;
        drop_first(a, h, keep);
        auto hn = [&](int e) { return GENERAL ? (h[e] - s.mean1) * s.rstd1 : h[e] * s.rstd1; };
        float p1 = 0.0f, p2 = 0.0f;
#pragma unroll
        for (int e = 0; e < V; e++) {
            const float u = GENERAL ? fmaf(hn(e), way[e], bias[e]) : hn(e) * way[e];
            const float t = a.h ? fmaf(u, keep[e], x[e]) : x[e];
            tn[e] = GENERAL ? (t - s.mean2) * s.rstd2 : t * s.rstd2;
            const float g = dy[e] * w2[e];
            if constexpr (GENERAL) p1 += g;
            p2 = fmaf(g, tn[e], p2);
        }
        h.keep(), dout.keep(), dy.keep();  // unpacked again below, which takes fewer registers
        float mean_a = 0.0f, mean_atn = 0.0f;
        if (b.dy) {
            const float2 r = join.sum(p1, p2);
            mean_a = r.x * inv_a * -s.rstd2, mean_atn = r.y * inv * -s.rstd2;
        }
        fetch(kPre, w2);
        float dt[V], p3 = 0.0f, p4 = 0.0f;
#pragma unroll
        for (int e = 0; e < V; e++) {
            dt[e] = dout[e];
            if (b.dy) {
                dt[e] = fmaf(s.rstd2, dy[e] * w2[e], GENERAL ? dt[e] + mean_a : dt[e]);
                dt[e] = fmaf(tn[e], mean_atn, dt[e]);
            }
            sum_w2[e] = fmaf(dy[e], tn[e], sum_w2[e]);
            if constexpr (GENERAL) sum_b2[e] += dy[e];
        }
        if (!PACE || active) mine.template put<T>(b.dx, row, b.dx_ld, Words<T, V>::of([&](int e) { return dt[e]; }));
        fetch(kWay, way);
#pragma unroll
        for (int e = 0; e < V; e++) {
            const float normal = hn(e), dv = keep[e] * dt[e];
            sum_a[e] = fmaf(dv, normal, sum_a[e]);
            if constexpr (GENERAL) sum_b[e] += dv;
            dt[e] = dv * way[e];
            if constexpr (GENERAL) p3 += dt[e];
            p4 = fmaf(dt[e], normal, p4);
        }
        if (!a.h) return;
        if (a.post != BYZ_NORM_NONE) {
            h.keep();
            const float2 r = join.sum(p3, p4);
            const float mean_b = r.x * inv_b * -s.rstd1, mean_bhn = r.y * inv * -s.rstd1;
#pragma unroll
            for (int e = 0; e < V; e++) dt[e] = fmaf(hn(e), mean_bhn, GENERAL ? fmaf(s.rstd1, dt[e], mean_b) : s.rstd1 * dt[e]);
        }
        if (!PACE || active) mine.template put<T>(b.dh, row, b.dh_ld, Words<T, V>::of([&](int e) { return dt[e]; }));
    };
    // some of a group's rows (PART), or whole groups for each slot
    const int64_t chunk = blockIdx.x, group_rows = a.gate_rows;
    int64_t group = PART ? blockIdx.x / b.per_group : chunk * SLOTS + slot;
    float gate_sum[V], w1_sum[V], b1_sum[V];
    float *const own = room + (2 * NT + threadIdx.x) * V;  // sums over the groups: of b1 NT * V behind those of w1
    if constexpr (!PART) {
#pragma unroll
        for (int e = 0; e < V; e++) own[e] = own[NT * V + e] = 0.0f;
    }
    // with PACE every slot of a block goes through as many rows
    for (int64_t base = PART ? group : chunk * SLOTS; base < (PART ? base + 1 : b.groups); base += (int64_t)gridDim.x * SLOTS) {
        if constexpr (!PART) group = base + slot;
        const bool there = group < b.groups;
        if (!there) {
            if constexpr (!PACE) break;
            group = b.groups - 1;
        }
        {
            const Way<TPR, GENERAL> way(a, mine, group);
            store(kWay, way.w);
            if constexpr (GENERAL)
#pragma unroll
                for (int e = 0; e < V; e++) bias[e] = way.b[e];
        }
        const int64_t end = std::min(a.rows, (group + 1) * group_rows), step = PART ? (int64_t)b.per_group * SLOTS : 1;
        const int64_t start = group * group_rows + (PART ? blockIdx.x % b.per_group * SLOTS : 0);
        const int64_t most = PART ? end : start + group_rows;  // where the slot with most rows ends
        int64_t row = start + (PART ? slot : 0);
        if (PACE ? start < most : row < end) {
            Loaded l = load(std::min(row, end - 1));
            for (int64_t at = PACE ? start : row; at < (PACE ? most : end); at += step, row += step)
                work(l, PACE ? std::min(row, end - 1) : row, std::min(row + step, end - 1), !PACE || (there && row < end));
        }
        // the sums of a group's rows make those of its vectors
        float g[V], w1[V], b1[V];
        mine.parameters_of(a.gate ? a.gate + group * a.cols : nullptr, 1.0f, g);
        mine.parameters_of(a.w1, 1.0f, w1);
        if constexpr (GENERAL) mine.parameters_of(a.b1, 0.0f, b1);
        const float factor = a.scale * a.drop.scale;
#pragma unroll
        for (int e = 0; e < V; e++) {
            gate_sum[e] = factor * (GENERAL ? fmaf(w1[e], sum_a[e], b1[e] * sum_b[e]) : w1[e] * sum_a[e]);
            w1_sum[e] = factor * g[e] * sum_a[e], b1_sum[e] = factor * g[e] * sum_b[e];
        }
        if constexpr (PART) break;
        if (b.d_gate && there) mine.template put<float>(b.d_gate, group, a.cols, Words<float, V>::of([&](int e) { return gate_sum[e]; }));
#pragma unroll
        for (int e = 0; e < V; e++) own[e] += w1_sum[e], own[NT * V + e] += b1_sum[e], sum_a[e] = sum_b[e] = 0.0f;
    }
    if constexpr (!PART) {
#pragma unroll
        for (int e = 0; e < V; e++) w1_sum[e] = own[e], b1_sum[e] = own[NT * V + e];
    }
    // What the chunk has for each kind, joined over the slots and written by neighbouring threads.  The weights' place is free.
    int at = 0;
    auto write = [&](int kind, const float (&v)[V]) __attribute__((always_inline)) {
        if (!(b.kinds >> kind & 1)) return;
        float *const to = b.partials + (chunk * __builtin_popcount(b.kinds) + at++) * a.cols;
        __syncthreads();
        const auto w = Words<float, V>::of([&](int e) { return v[e]; });
        __builtin_memcpy(room + threadIdx.x * V, &w, sizeof(w));
        __syncthreads();
        for (int i = threadIdx.x; i < (int)a.cols; i += blockDim.x) {
            const int first = i / V * V, place = first + i - std::min(first, (int)a.cols - V);
            float sum = 0.0f;
#pragma unroll
            for (int l = 0; l < SLOTS; l++) sum += room[l * (TPR * V) + place];
            to[i] = sum;
        }
    };
    write(kW2, sum_w2);
    if constexpr (GENERAL) write(kB2, sum_b2);
    write(kW1, w1_sum);
    if constexpr (GENERAL) write(kB1, b1_sum);
    if constexpr (PART) write(kGate, gate_sum);
}

// dx, dh and the means of rows of 8193 to 16384 columns of 16 bits, root mean squares only and without additions: sixteen columns a
// thread, in registers from the one read that rows_kernel does three times.  Their sums would not fit beside them and are
// columns_kernel's.  Of the other norms and of fp32 the four tensors in registers spill: rows_kernel's.  us of a whole backward pass, so and with
// rows_kernel: 2048 x 16384 bf16 200 and 260; with layer norms 284 and 255, 3000 x 9001 of them 344 and 257, 1024 x 16384 fp32 240 and 215.
template <typename T>
__global__ __launch_bounds__(1024, 4) void wide_rows_kernel(Args a, Back b) {
    constexpr int V = kCols, R = 2, TPR = 1024;
    __shared__ float2 lds[RowJoiner<TPR, 1>::size];
    RowJoiner<TPR, 1> join(lds);
    auto mine = [&](int r) __attribute__((always_inline)) { return Columns<TPR>(a.cols, r); };
    const uint64_t offset = drop_offset(a.drop);
    const float inv = 1.0f / (float)a.cols;
    float w2[R][V];
    Way<TPR, false> way[R];
#pragma unroll
    for (int r = 0; r < R; r++) mine(r).parameters_of(a.w2, 1.0f, w2[r]);
    int64_t group_end = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        Words<T, V> x[R], h[R] = {}, dout[R] = {}, dy[R] = {};
#pragma unroll
        for (int r = 0; r < R; r++) {
            x[r] = mine(r).template get<T>(a.x, row, a.x_ld);
            if (a.h) h[r] = mine(r).template get<T>(a.h, row, a.h_ld);
            if (b.dy) dy[r] = mine(r).template get<T>(b.dy, row, b.dy_ld);
            if (b.dout) dout[r] = mine(r).template get<T>(b.dout, row, b.dout_ld);
        }
        const Stats s = stats_of(b.stats, row);
        if (row >= group_end) {
            const int64_t group = group_of(a, row);
#pragma unroll
            for (int r = 0; r < R; r++) way[r] = Way<TPR, false>(a, mine(r), group);
            group_end = (group + 1) * a.gate_rows;
        }
        uint32_t mask[R];
        auto hn = [&](int r, int e) { return h[r][e] * s.rstd1; };
        auto kept = [&](int r, int e) { return mask[r] >> e & 1 ? 1.0f : 0.0f; };
        auto tn = [&](int r, int e) {
            const float t = a.h ? fmaf(way[r].of(e, hn(r, e)), kept(r, e), x[r][e]) : x[r][e];
            return t * s.rstd2;
        };
        auto unpack_again = [&](int r) __attribute__((always_inline)) { x[r].keep(), h[r].keep(), dout[r].keep(), dy[r].keep(); };
        float p2 = 0.0f;
#pragma unroll
        for (int r = 0; r < R; r++) {
            float keep[V];
            mine(r).kept(a, offset, row, keep);
            mine(r).only_own(dy[r]);
            drop_first(a, h[r], keep);
            mask[r] = 0;
#pragma unroll
            for (int e = 0; e < V; e++) mask[r] |= keep[e] != 0.0f ? 1u << e : 0u;
#pragma unroll
            for (int e = 0; e < V; e++) p2 = fmaf(dy[r][e] * w2[r][e], tn(r, e), p2);
            unpack_again(r);
            __builtin_amdgcn_sched_barrier(0);
        }
        float mean_atn = 0.0f;
        if (b.dy) mean_atn = join.sum(0.0f, p2).y * inv;
        float dt[R][V], p4 = 0.0f;
#pragma unroll
        for (int r = 0; r < R; r++) {
#pragma unroll
            for (int e = 0; e < V; e++) {
                dt[r][e] = dout[r][e];
                if (b.dy) {
                    dt[r][e] = fmaf(s.rstd2, dy[r][e] * w2[r][e], dt[r][e]);
                    dt[r][e] = fmaf(tn(r, e), -s.rstd2 * mean_atn, dt[r][e]);
                }
            }
            mine(r).template put<T>(b.dx, row, b.dx_ld, Words<T, V>::of([&](int e) { return dt[r][e]; }));
#pragma unroll
            for (int e = 0; e < V; e++) {
                dt[r][e] *= kept(r, e) * way[r].w[e];
                p4 = fmaf(dt[r][e], hn(r, e), p4);
            }
            h[r].keep();
            __builtin_amdgcn_sched_barrier(0);
        }
        float mean_bhn = 0.0f;
        if (a.h) {
            if (a.post != BYZ_NORM_NONE) mean_bhn = join.sum(0.0f, p4).y * inv;
#pragma unroll
            for (int r = 0; r < R; r++) {
                if (a.post != BYZ_NORM_NONE) {
#pragma unroll
                    for (int e = 0; e < V; e++) dt[r][e] = fmaf(hn(r, e), -s.rstd1 * mean_bhn, s.rstd1 * dt[r][e]);
                }
                mine(r).template put<T>(b.dh, row, b.dh_ld, Words<T, V>::of([&](int e) { return dt[r][e]; }));
            }
        }
        if (threadIdx.x == 0) {
            float *at = b.rest + row * 4;
            at[0] = 0.0f, at[1] = mean_atn, at[2] = 0.0f, at[3] = mean_bhn;
        }
    }
}

struct Outputs {
    float *of[kKinds];
};

// Sums of the chunks' partials: a block 64 columns of one kind (and one group of gate's rows), its sixteen waves every sixteenth
// chunk.
__global__ __launch_bounds__(1024) void finish_kernel(const float *partials, Outputs out, uint32_t kinds, int64_t cols, int64_t chunks,
                                                      int64_t per_group, int64_t groups) {
    constexpr int W = 16;
    __shared__ float lds[W][64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, count = __builtin_popcount(kinds);
    const int64_t col = (int64_t)blockIdx.x * 64 + lane;
    int kind = 0, left = blockIdx.y;
    for (int k = 0; k < kKinds; k++)
        if (kinds >> k & 1) {
            if (left == 0) kind = k;
            left--;
        }
    const bool gate = kind == kGate;
    for (int64_t group = blockIdx.z; group < (gate ? groups : 1); group += gridDim.z) {
        const int64_t from = gate ? group * per_group : 0, to = gate ? from + per_group : chunks;
        float sum = 0.0f;
        if (col < cols) {
            const float *at = partials + ((from + wave) * count + blockIdx.y) * cols + col;
            const int64_t step = W * count * cols;
#pragma unroll 8
            for (int64_t c = from + wave; c < to; c += W, at += step) sum += *at;
        }
        __syncthreads();
        lds[wave][lane] = sum;
        __syncthreads();
        if (wave == 0 && col < cols) {
            sum = 0.0f;
#pragma unroll
            for (int w = 0; w < W; w++) sum += lds[w][lane];
            float *to_ = out.of[0];
#pragma unroll
            for (int k = 1; k < kKinds; k++) to_ = kind == k ? out.of[k] : to_;
            to_[(gate ? group * cols : 0) + col] = sum;
        }
    }
}

constexpr int64_t kRowsInRegisters = 1024 * kCols;  // columns a block's threads hold
constexpr int64_t kGroupsInLds = 512 * kCols;        // columns whose sums over short groups of gate's rows are kept in LDS
bool in_registers(int64_t cols) { return cols >= kCols && cols <= kRowsInRegisters; }

// fn(threads of a row as a constant)
template <typename F>
int with_threads(int64_t cols, F fn) {
    const int64_t threads = (cols + kCols - 1) / kCols;
    if (threads <= 8) return fn(std::integral_constant<int, 8>{});
    if (threads <= 16) return fn(std::integral_constant<int, 16>{});
    if (threads <= 32) return fn(std::integral_constant<int, 32>{});
    if (threads <= 64) return fn(std::integral_constant<int, 64>{});
    if (threads <= 128) return fn(std::integral_constant<int, 128>{});
    if (threads <= 192) return fn(std::integral_constant<int, 192>{});
    if (threads <= 256) return fn(std::integral_constant<int, 256>{});
    if (threads <= 512) return fn(std::integral_constant<int, 512>{});
    return fn(std::integral_constant<int, 1024>{});
}

// How the rows are cut for the sums of columns: chunks for sixteen waves a compute unit, but of two rows a slot at least, each
// within a group of gate's rows, or of whole groups where these are short.  columns_kernel's blocks, of 512 columns of 16 bits each, are some
// eight a compute unit: with 512 chunks whatever the width, backward of 2048 x 16384 bf16 took 68 us more, 1024 x 40000 78 more.
constexpr int64_t kLeast = 2;  // us at 2, 4, 8: backward of 333 x 1000 fp32 18, 23, 33, of 3950 x 604 bf16 30, 29, 36
struct Cut {
    int64_t per_group, groups, chunks;
    Cut(int64_t rows, int64_t cols, int64_t gate_rows) {
        int64_t blocks = std::max<int64_t>(8, 8 * kCus / ((cols + 511) / 512)), least = 4;
        if (in_registers(cols))
            with_threads(cols, [&](auto tpr) -> int {
                constexpr int TPR = tpr.value, NT = back_block_of<TPR>();
                blocks = kCus * (1024 / threads_of<TPR, NT>(cols)), least = kLeast * (NT / TPR);
                return 0;
            });
        const int64_t want = std::max(least, (rows + blocks - 1) / blocks);
        groups = (rows + gate_rows - 1) / gate_rows;
        if (gate_rows >= want) {
            per_group = (gate_rows + want - 1) / want, chunks = groups * per_group;
        } else {
            const int64_t each = (want + gate_rows - 1) / gate_rows;  // groups of a chunk
            per_group = 0, chunks = (groups + each - 1) / each;
        }
    }
};

bool sizes_ok(int64_t rows, int64_t cols, int dtype, int64_t gate_rows) {
    int64_t values;
    return rows >= 0 && cols >= 1 && cols <= INT32_MAX && dtype_known(dtype) && gate_rows >= 1 &&
           !__builtin_mul_overflow(rows, cols, &values) && values <= (INT64_MAX >> 8);
}

size_t rest_bytes(int64_t rows) { return (size_t)rows * 16; }

size_t workspace(int64_t rows, int64_t cols, int64_t gate_rows) {
    return rows == 0 ? 0 : rest_bytes(rows) + (size_t)Cut(rows, cols, std::min(gate_rows, rows)).chunks * kKinds * (size_t)cols * 4;
}

template <typename T>
int launch_forward(const Args &a, hipStream_t s) {
    const bool general = a.b1 || a.b2 || a.post == BYZ_NORM_LAYER || a.pre == BYZ_NORM_LAYER;
    if (a.cols > kRowsInRegisters && a.cols <= 2 * kRowsInRegisters) {
        const unsigned blocks = (unsigned)std::min<int64_t>(a.rows, kCus * 2);
        (general ? &forward_rows_kernel<T, 1024, 2, true> : &forward_rows_kernel<T, 1024, 2, false>)<<<blocks, 1024, 0, s>>>(a);
        BYZ_HIP(hipGetLastError());
        return BYZ_OK;
    }
    if (in_registers(a.cols)) {
        return with_threads(a.cols, [&](auto tpr) -> int {
            constexpr int TPR = tpr.value, NT = block_of<TPR>(), slots = NT / TPR;
            const int threads = threads_of<TPR, NT>(a.cols);
            const int64_t blocks = std::min((a.rows + slots - 1) / slots, (int64_t)kCus * (2048 / threads));
            (general ? &forward_rows_kernel<T, TPR, 1, true> : &forward_rows_kernel<T, TPR, 1, false>)<<<(unsigned)blocks, threads, 0, s>>>(a);
            BYZ_HIP(hipGetLastError());
            return BYZ_OK;
        });
    }
    if (a.cols > kRowsInRegisters && a.rows < kCus)
        forward_kernel<T, 1024><<<(unsigned)std::min(a.rows, kMaxGrid), 1024, 0, s>>>(a);
    else
        forward_kernel<T, 256><<<(unsigned)std::min(a.rows, kMaxGrid), 256, 0, s>>>(a);
    BYZ_HIP(hipGetLastError());
    return BYZ_OK;
}

template <typename T>
int launch_backward(const Args &a, Back b, const Cut &cut, const Outputs &out, hipStream_t s) {
    constexpr int V = 16 / sizeof(T);
    const bool general = a.b1 || (b.kinds & (1u << kB1 | 1u << kB2)) || a.post == BYZ_NORM_LAYER || a.pre == BYZ_NORM_LAYER;
    if (in_registers(a.cols) && (cut.per_group || a.cols <= kGroupsInLds)) {
        const int rc = with_threads(a.cols, [&](auto tpr) -> int {
            constexpr int TPR = tpr.value, NT = back_block_of<TPR>(), each = NT * kCols * (int)sizeof(float);
            if (cut.per_group) {
                (general ? &backward_rows_kernel<T, TPR, true, true> : &backward_rows_kernel<T, TPR, false, true>)
                    <<<(unsigned)cut.chunks, threads_of<TPR, NT>(a.cols), 2 * each, s>>>(a, b);
            } else if constexpr (TPR <= 512) {
                (general ? &backward_rows_kernel<T, TPR, true, false> : &backward_rows_kernel<T, TPR, false, false>)
                    <<<(unsigned)cut.chunks, threads_of<TPR, NT>(a.cols), 4 * each, s>>>(a, b);
            }
            BYZ_HIP(hipGetLastError());
            return BYZ_OK;
        });
        if (rc != BYZ_OK) return rc;
    } else {
        const bool wide = sizeof(T) == 2 && !general && a.cols > kRowsInRegisters && a.cols <= 2 * kRowsInRegisters;
        if (wide) {
            if constexpr (sizeof(T) == 2) wide_rows_kernel<T><<<(unsigned)std::min<int64_t>(a.rows, kCus * 2), 1024, 0, s>>>(a, b);
        } else if (a.cols > kGroupsInLds && a.rows < kCus) {
            rows_kernel<T, 1024><<<(unsigned)std::min(a.rows, kMaxGrid), 1024, 0, s>>>(a, b);
        } else {
            rows_kernel<T, 256><<<(unsigned)std::min(a.rows, kMaxGrid), 256, 0, s>>>(a, b);
        }
        BYZ_HIP(hipGetLastError());
        if (!b.kinds && !b.d_gate) return BYZ_OK;
        columns_kernel<T><<<dim3((unsigned)((a.cols + 64 * V - 1) / (64 * V)), (unsigned)cut.chunks), 256, 0, s>>>(a, b);
        BYZ_HIP(hipGetLastError());
    }
    if (!b.kinds) return BYZ_OK;
    const unsigned depth = b.kinds >> kGate & 1 ? (unsigned)std::min<int64_t>(cut.groups, 1024) : 1;
    finish_kernel<<<dim3((unsigned)((a.cols + 63) / 64), (unsigned)__builtin_popcount(b.kinds), depth), 1024, 0, s>>>(
        b.partials, out, b.kinds, a.cols, cut.chunks, cut.per_group, cut.groups);
    BYZ_HIP(hipGetLastError());
    return BYZ_OK;
}

__global__ void zero_kernel(float *p, int64_t n) {
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (int64_t)gridDim.x * blockDim.x) p[i] = 0.0f;
}

bool norm_known(int n) { return n >= BYZ_NORM_NONE && n <= BYZ_NORM_LAYER; }
bool real(float v) { return v > -INFINITY && v < INFINITY; }

// A matrix that may not be there.
bool matrix_ok(const void *p, int64_t ld, int64_t rows, int64_t cols, int dtype) {
    return !p || (aligned(p, dtype_size(dtype)) && ld >= cols && extent_ok(rows, ld, cols));
}
bool floats_ok(const float *p) { return aligned(p, 4); }

int check(const Args &a, const byz_residual_form *f, int dtype) {
    if (!f || !sizes_ok(a.rows, a.cols, dtype, a.gate_rows) || !norm_known(f->post) || !norm_known(f->pre) || !(f->eps >= 0.0f) ||
        !real(f->eps) || !real(f->scale) || !drop_ok(f->p, f->offset_at, f->first_row, a.rows, a.cols))
        return BYZ_EINVAL;
    if (a.rows > 0 && !a.h && (f->post != BYZ_NORM_NONE || a.w1 || a.b1 || a.gate || f->pre == BYZ_NORM_NONE)) return BYZ_EINVAL;
    if (f->pre == BYZ_NORM_NONE && (a.w2 || a.b2)) return BYZ_EINVAL;
    if (!floats_ok(a.w1) || !floats_ok(a.b1) || !floats_ok(a.gate) || !floats_ok(a.w2) || !floats_ok(a.b2)) return BYZ_EINVAL;
    if (a.rows == 0) return BYZ_OK;
    if (!a.x || !matrix_ok(a.x, a.x_ld, a.rows, a.cols, dtype) || !matrix_ok(a.h, a.h_ld, a.rows, a.cols, dtype)) return BYZ_EINVAL;
    return BYZ_OK;
}

Args args_of(const void *x, int64_t x_ld, const void *h, int64_t h_ld, int64_t rows, int64_t cols, const byz_residual_form *f,
             const float *w1, const float *b1, const float *gate, int64_t gate_rows, const float *w2, const float *b2) {
    Args a{};
    a.x = x, a.h = h, a.x_ld = x_ld, a.h_ld = h_ld, a.rows = rows, a.cols = cols;
    a.w1 = w1, a.b1 = b1, a.gate = gate, a.w2 = w2, a.b2 = b2;
    a.gate_rows = gate ? std::min(gate_rows, std::max<int64_t>(rows, 1)) : std::max<int64_t>(rows, 1);
    if (gate && gate_rows < 1) a.gate_rows = gate_rows;  // refused
    if (!f) return a;
    a.post = f->post, a.pre = f->pre, a.eps = f->eps, a.scale = f->scale;
    return a;
}

}  // namespace

extern "C" int byz_residual_norm(const void *x, int64_t x_ld, const void *h, int64_t h_ld, int64_t rows, int64_t cols, int dtype,
                                 const byz_residual_form *form, const float *post_weight, const float *post_bias, const float *gate,
                                 int64_t gate_rows, const float *pre_weight, const float *pre_bias, void *out, int64_t out_ld,
                                 void *y, int64_t y_ld, float *stats, void *stream) {
    Args a = args_of(x, x_ld, h, h_ld, rows, cols, form, post_weight, post_bias, gate, gate_rows, pre_weight, pre_bias);
    const int rc = check(a, form, dtype);
    if (rc != BYZ_OK || rows == 0) return rc;
    if ((h && !out) || (form->pre != BYZ_NORM_NONE && !y) || !floats_ok(stats) || !matrix_ok(h ? out : nullptr, out_ld, rows, cols, dtype) ||
        !matrix_ok(form->pre != BYZ_NORM_NONE ? y : nullptr, y_ld, rows, cols, dtype))
        return BYZ_EINVAL;
    a.drop = drop_of(form->p, form->seed, form->offset, form->offset_at, form->first_row);
    a.out = out, a.out_ld = out_ld, a.y = y, a.y_ld = y_ld, a.stats = stats;
    const hipStream_t s = (hipStream_t)stream;
    return dtype == BYZ_F32 ? launch_forward<float>(a, s) : dtype == BYZ_BF16 ? launch_forward<bf16>(a, s) : launch_forward<f16>(a, s);
}

extern "C" size_t byz_residual_norm_backward_workspace_bytes(int64_t rows, int64_t cols, int dtype, int64_t gate_rows) {
    return sizes_ok(rows, cols, dtype, gate_rows) ? workspace(rows, cols, gate_rows) : 0;
}

extern "C" int byz_residual_norm_backward(const void *dout, int64_t dout_ld, const void *dy, int64_t dy_ld, const void *x,
                                          int64_t x_ld, const void *h, int64_t h_ld, const float *stats, int64_t rows, int64_t cols,
                                          int dtype, const byz_residual_form *form, const float *post_weight,
                                          const float *post_bias, const float *gate, int64_t gate_rows, const float *pre_weight,
                                          void *dx, int64_t dx_ld, void *dh, int64_t dh_ld, float *d_post_weight,
                                          float *d_post_bias, float *d_gate, float *d_pre_weight, float *d_pre_bias,
                                          void *workspace_, size_t workspace_bytes, void *stream) {
    Args a = args_of(x, x_ld, h, h_ld, rows, cols, form, post_weight, post_bias, gate, gate_rows, pre_weight, nullptr);
    const int rc = check(a, form, dtype);
    if (rc != BYZ_OK) return rc;
    if (!floats_ok(d_post_weight) || !floats_ok(d_post_bias) || !floats_ok(d_gate) || !floats_ok(d_pre_weight) || !floats_ok(d_pre_bias) ||
        (rows > 0 && !h && (d_post_weight || d_post_bias || d_gate)) || (d_gate && !gate) ||
        (form->pre == BYZ_NORM_NONE && (d_pre_weight || d_pre_bias || dy)))
        return BYZ_EINVAL;
    const hipStream_t s = (hipStream_t)stream;
    const Outputs out{{d_pre_weight, d_pre_bias, d_post_weight, d_post_bias, d_gate}};
    if (rows == 0) {
        for (int k = 0; k < kKinds; k++)
            if (out.of[k]) {
                zero_kernel<<<(unsigned)((cols + 255) / 256), 256, 0, s>>>(out.of[k], cols);
                BYZ_HIP(hipGetLastError());
            }
        return BYZ_OK;
    }
    if (!dx || (h && !dh) || !stats || !floats_ok(stats) || (!dout && !dy) || !matrix_ok(dout, dout_ld, rows, cols, dtype) ||
        !matrix_ok(dy, dy_ld, rows, cols, dtype) || !matrix_ok(dx, dx_ld, rows, cols, dtype) ||
        !matrix_ok(h ? dh : nullptr, dh_ld, rows, cols, dtype))
        return BYZ_EINVAL;
    if (!workspace_ || !aligned(workspace_, 16) || workspace_bytes < workspace(rows, cols, a.gate_rows)) return BYZ_ENOMEM;
    a.drop = drop_of(form->p, form->seed, form->offset, form->offset_at, form->first_row);
    const Cut cut(rows, cols, a.gate_rows);
    Back b{};
    b.dout = dout, b.dout_ld = dout_ld, b.dy = dy, b.dy_ld = dy_ld, b.stats = stats;
    b.dx = dx, b.dx_ld = dx_ld, b.dh = dh, b.dh_ld = dh_ld;
    b.rest = (float *)workspace_, b.partials = b.rest + rows * 4;
    b.d_gate = cut.per_group ? nullptr : d_gate;
    for (int k = 0; k < kKinds; k++)
        if (out.of[k] && (k != kGate || cut.per_group)) b.kinds |= 1u << k;
    b.chunks = (uint32_t)cut.chunks, b.per_group = (uint32_t)cut.per_group, b.groups = cut.groups;
    return dtype == BYZ_F32 ? launch_backward<float>(a, b, cut, out, s)
           : dtype == BYZ_BF16 ? launch_backward<bf16>(a, b, cut, out, s) : launch_backward<f16>(a, b, cut, out, s);
}

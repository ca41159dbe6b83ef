// Group norm with an activation on channels-last features, forward and backward (gfx950).
//
// A sample is a p x c matrix, a group a strip of c / groups of its columns.  A block takes a slice:
// some whole groups (or a part of one wide group), all positions or a chunk of them.  Thread t holds the
// same V channels at positions t / tx, t / tx + ty, ...
//
//   forward    a thread's own mean and squared distances from it, joined pairwise (count, mean, distances) over
//              threads, waves and chunks in a fixed order, so there is no difference of large sums.  The means are fp64:
//              their pairwise differences then lose nothing where a group's mean is many times its deviation.
//              Then act((x - mean) rstd gamma + beta).
//   backward   with the activation's slope recomputed, dz = dy act'(z): per channel the sums A of dz and
//              B of dz xhat are all that is needed,
//                  dbeta = sum A,  dgamma = sum B  (over the samples, in order),
//                  S1 = sum gamma A / m,  S2 = sum gamma B / m  (over a group's channels),
//                  dx = rstd (gamma dz - S1 - xhat S2).
//
// Bound by memory: 2 values moved per value forward, 3 backward, a dozen operations each.  Where a slice
// of a sample fits the registers of one block ("whole") everything is read once.  Larger samples are cut into
// chunks: a first kernel writes their statistics, a second joins them in chunk order, a third reads the chunks again and
// stores past the caches, which then still hold inputs for the next pass (backward sums behind the forward pass 46.6 / 38.4 us,
// gradients 54.9 / 48.8, without / with that).  A slice is 64 bytes of a row wide at least, which is 200 KB on 64 x 56 x 56 x 256
// bf16: registers for that, 16 vectors a thread, spill and were slower (64 us for 58 in three kernels); narrower slices that would
// fit, 100 KB, have not been tried.
// No atomics.
//
// us, traced: 64 x 112 x 112 x 64 fp16 forward: statistics 21.2 (103 MB, 4.9 TB/s), join 4.7, pass 36.1 (206 MB, 5.7 TB/s).
// 64 x 56 x 56 x 256 bf16: forward 20.4 + 4.8 + 33.3; backward sums 37.2 (206 MB, 5.5 TB/s), totals 5.0, pass 48.4 (309 MB, 6.4 TB/s),
// parameters 4.8.  30 x 32 x 32 x 64 bf16: 10.6 forward, 12.0 backward (12.1 and 16.0 with joins through LDS), 3.3
// parameters: a block's chain of loads, joins and stores.  Slices of 64 x 28 x 28 x 512 bf16 fit: 33.7 forward (floor 16), 63
// backward (24), as loads, joins and stores of a block follow one another with little else on the compute unit.
#include <algorithm>
#include <type_traits>

#include "worker_internal.h"

using namespace byz_worker;

namespace {

constexpr int kForwardThreads = 1024;  // most threads of a whole slice and most 16-byte vectors that a thread holds of a
constexpr int kForwardR = 8;           // tensor: 128 registers a thread of 1024, 256 a thread of 512, which the two
constexpr int kBackwardThreads = 512;  // tensors of the backward pass need
constexpr int kBackwardR = 8;
constexpr int kMaxLanes = 256;         // most vectors of a slice's row
constexpr int kDepth = 32;             // positions of a thread in a chunk at most: what its sums about its first
                                       // value can lose is 2^-24 times this
constexpr int64_t kMaxGrid = 1 << 20;  // blocks of a launch; more tiles are taken in turn
// Blocks go to the eight dies in turn; neighbouring tiles (slices of the same rows share cache lines, chunks a group's
// statistics) are numbered so that they meet on one die and its L2.

struct Plan {
    int64_t n, p, c;
    uint32_t groups, gc;          // groups of gc channels
    uint32_t slices, chunks, tiles;
    uint32_t per_xcd;             // tiles of a block number modulo 8
    int vec, cs, tx, ty, threads, r, unit;  // unit: neighbouring channels of a vector that are in one group
    int head;                     // groups of a slice
    uint32_t parts;               // blocks that share a group's channels (1: a slice has whole groups)
    int64_t chunk;
};

int64_t gcd(int64_t a, int64_t b) { return b ? gcd(b, a % b) : a; }

// Neighbouring elements that are loaded in one piece, at any address of an element: a plan goes by sizes and type alone, or the
// order of the sums would change with the place of a tensor.
int widest_vec(int elem, int64_t c) {
    for (int vec : {16 / elem, 4 / elem})
        if (c % vec == 0) return vec;
    return 1;
}

// Positions of a chunk of a large sample: as many as leave `blocks` of them.  Blocks that sum end in joins, which cost less
// over long chunks; those that only pass over the data again are better short.  us on 64 x 56 x 56 x 256 bf16, 512 / 2048 blocks and
// more: sums of the backward pass 46.5 / 51.6, forward's 21.1 / 25.1; gradients 63.2 / 55.6.
constexpr int64_t kSumBlocks = 700, kPassBlocks = 2048;
int64_t chunk_of(const Plan &q, int64_t slices, int64_t blocks) {
    int depth = kDepth;
    while (depth > 8 && q.n * slices * ((q.p + (int64_t)q.ty * depth - 1) / ((int64_t)q.ty * depth)) < blocks) depth /= 2;
    return (int64_t)q.ty * depth;
}

// False: more tiles than can be counted.
bool make_plan(Plan &q, int64_t n, int64_t p, int64_t c, int64_t groups, int elem, bool forward) {
    const int max_r = forward ? kForwardR : kBackwardR;
    int max_threads, vec = widest_vec(elem, c);
    q = Plan{};
    const int64_t gc = c / groups;
    int64_t slices, step;
    q.n = n, q.p = p, q.c = c, q.groups = (uint32_t)groups, q.gc = (uint32_t)gc;
    // a slice of whole groups whose rows start at multiples of vec, or a part of one group; narrower
    // vectors where neither is possible
    for (;; vec = vec > 4 / elem ? (4 / elem > 1 ? 4 / elem : 1) : 1) {
        step = gc / gcd(gc, vec) * vec;
        // four units a thread or eight: the statistics of 1024 threads would not fit 64 KB of LDS
        max_threads = !forward ? kBackwardThreads : kForwardThreads / (int)std::max<int64_t>(1, vec / gcd(gc, vec) / 2);
        if (step / vec <= kMaxLanes) {
            // 128 bytes of a row, a cache line, where the channels reach
            int64_t cs = step;
            while (cs * elem < 128 && cs + step <= c) cs += step;
            // narrower, down to 64 bytes, for a slice that fits a block, or to 32 for a block on every compute unit
            auto narrow = [&](int64_t w) { return (w / 2 + step - 1) / step * step; };
            while (cs > step && narrow(cs) < cs &&
                   ((narrow(cs) * elem >= 64 && p * (cs / vec) > (int64_t)max_threads * max_r) ||
                    (narrow(cs) * elem >= 32 && n * ((c + cs - 1) / cs) < 256)))
                cs = narrow(cs);
            if (p * (cs / vec) > (int64_t)max_threads * max_r)  // chunks after all: back to whole lines
                while (cs * elem < 128 && cs + step <= c) cs += step;
            q.cs = (int)cs, q.parts = 1;
            slices = (c + cs - 1) / cs;
            break;
        }
        if (gc % vec == 0) {
            const int64_t lanes = gc / vec, parts = (lanes + kMaxLanes - 1) / kMaxLanes;
            q.cs = (int)((lanes + parts - 1) / parts) * vec;
            q.parts = (uint32_t)((gc + q.cs - 1) / q.cs);
            slices = groups * q.parts;
            break;
        }
    }
    q.vec = vec;
    q.unit = (int)gcd(gc, vec);
    q.head = q.parts > 1 ? 1 : (int)(q.cs / gc);
    q.tx = q.cs / vec;
    const int64_t vectors = p * q.tx;
    int64_t chunks = 1;
    if (q.parts == 1 && vectors <= (int64_t)max_threads * max_r) {
        // four vectors a thread where that gives enough threads
        int64_t threads = (vectors + 3) / 4;
        threads = threads < 64 ? 64 : threads > max_threads ? max_threads : (threads + 63) / 64 * 64;
        if (threads < q.tx) threads = (q.tx + 63) / 64 * 64;
        q.threads = (int)threads;
        q.ty = q.threads / q.tx;
        const int64_t r = (p + q.ty - 1) / q.ty;
        if (r <= max_r) {
            q.r = r <= 1 ? 1 : r <= 2 ? 2 : r <= 4 ? 4 : 8;
            q.chunk = p;
        }
    }
    if (!q.r) {
        q.threads = 256;
        q.ty = q.threads / q.tx;
        q.chunk = chunk_of(q, slices, kSumBlocks);
        chunks = (p + q.chunk - 1) / q.chunk;
    }
    int64_t tiles;
    if (__builtin_mul_overflow(n, slices, &tiles) || __builtin_mul_overflow(tiles, chunks, &tiles) || tiles > (q.r ? INT32_MAX : INT32_MAX / 4) ||
        n * groups > INT32_MAX)
        return false;
    q.slices = (uint32_t)slices, q.chunks = (uint32_t)chunks, q.tiles = (uint32_t)tiles;
    q.per_xcd = (q.tiles + 7) / 8;
    return true;
}

bool whole(const Plan &q) { return q.r > 0; }

// The call for the kernel that passes over a large sample again.  Its chunks are shorter by 32 / 8 at most: a tile's number still fits.
template <typename A>
A pass_again(A a) {
    Plan &q = a.q;
    q.chunk = chunk_of(q, q.slices, kPassBlocks);
    q.chunks = (uint32_t)((q.p + q.chunk - 1) / q.chunk);
    q.tiles = (uint32_t)q.n * q.slices * q.chunks;
    q.per_xcd = (q.tiles + 7) / 8;
    return a;
}

// Mean, count, squared distances from it.
struct Stat {
    double m;
    float n, d;
};

struct Args {
    Plan q;
    const void *x, *dy;
    void *out;  // y or dx
    int64_t xs, xp, ds, dp, os, op;
    const float *gamma, *beta;
    float *mean, *rstd;
    float eps;
    int act;
    Stat *stat;     // forward: of [sample][group][chunk][part]
    float2 *part;   // backward: (A, B) of [sample][chunk][channel]
    float2 *total;  // backward: (A, B) of [sample][channel]
    float2 *sums;   // backward: (S1, S2) of [sample][group]
    float *dgamma, *dbeta;
};

// What a block works on.
struct Tile {
    int64_t i, p0, c0;          // sample, first position, first channel
    uint32_t chunk, part, g0;   // g0: first group
    int np, nc;                 // positions, channels
    int tx, ty;                 // this thread's vector and first position
    bool mine;                  // the thread has channels
    __device__ Tile(const Plan &q, uint32_t t, int V) {
        const uint32_t rest = t / q.slices, slice = t - rest * q.slices, sample = rest / q.chunks;
        i = sample;
        chunk = rest - sample * q.chunks;
        p0 = chunk * q.chunk;
        np = (int)(q.p - p0 < q.chunk ? q.p - p0 : q.chunk);
        int64_t end;
        if (q.parts > 1) {
            g0 = slice / q.parts, part = slice - g0 * q.parts;
            c0 = (int64_t)g0 * q.gc + (int64_t)part * q.cs;
            end = (int64_t)(g0 + 1) * q.gc;
        } else {
            c0 = (int64_t)slice * q.cs, end = q.c;
            g0 = (uint32_t)c0 / q.gc, part = 0;
        }
        nc = (int)(end - c0 < q.cs ? end - c0 : q.cs);
        ty = threadIdx.x / q.tx;
        tx = threadIdx.x - ty * q.tx;
        mine = ty < q.ty && tx * V < nc;
        if (ty >= q.ty) ty = q.ty;  // threads beyond the last whole row of them
    }
    __device__ int groups(const Plan &q) const { return q.parts > 1 ? 1 : nc / (int)q.gc; }
    __device__ int width(const Plan &q) const { return q.parts > 1 ? nc : (int)q.gc; }  // of a group, here
    // groups of this thread's channels, counted from g0
    template <int V>
    __device__ void groups_of(const Plan &q, int (&g)[V]) const {
        const int w = width(q), first = mine ? tx * V : 0;
        int at = first / w, rem = first - at * w;
#pragma unroll
        for (int v = 0; v < V; v++) {
            g[v] = at;
            if (++rem == w) rem = 0, at++;
        }
    }
    template <typename T>
    __device__ const T *in(const void *base, int64_t sample, int64_t pixel, int V) const {
        return (const T *)base + i * sample + (p0 + ty) * pixel + c0 + tx * V;
    }
    template <typename T>
    __device__ T *out(const Args &a, int V) const {
        return (T *)a.out + i * a.os + (p0 + ty) * a.op + c0 + tx * V;
    }
};

__device__ __forceinline__ Stat join(Stat a, Stat b) {
    // written so that a set with a count of 0 changes nothing
    const float n = a.n + b.n, f = n > 0.0f ? b.n * __builtin_amdgcn_rcpf(n) : 0.0f;
    const double e = b.n > 0.0f ? b.m - a.m : 0.0;
    const float e1 = (float)e;
    return Stat{a.n > 0.0f ? a.m + e * (double)f : b.m, n, a.d + b.d + (a.n > 0.0f ? e1 * e1 * (a.n * f) : 0.0f)};
}

// Joins the statistics of lanes that are `first` and more apart; each gets the same bits.
__device__ __forceinline__ Stat join_wave(Stat s, int first) {
    wave_steps(first, [&](auto step) {
        Stat lower, upper;
        wave_pair<step.value>(s, lower, upper);
        if (step.value < 4 && (threadIdx.x & (1 << step.value))) {
            const Stat own = lower;
            lower = upper, upper = own;
        }
        s = join(lower, upper);
    });
    return s;
}

constexpr int kStatRows = 16;
constexpr int kSerial = 16;  // entries of a group that one thread joins

// Joins the threads' statistics (n values each of V channels, mean m, distances d) into the groups', one thread calls
// done(g, statistics) for each.  Ends with a barrier.  `entry`: LDS for one Stat a thread and unit, or a wave's column and unit.
template <int V, typename F>
__device__ void group_stats(const Plan &q, const Tile &t, float n, double (&m)[V], float (&d)[V], Stat *entry, F done) {
    // channels of a unit first: equal counts
    float count = n;
#pragma unroll
    for (int w = 1; w < V; w *= 2)
        if (q.unit > w) {
#pragma unroll
            for (int v = 0; v < V; v += 2 * w) {
                const float e = (float)(m[v + w] - m[v]);
                m[v] = 0.5 * (m[v] + m[v + w]);
                d[v] += d[v + w] + e * e * (0.5f * count);
            }
            count *= 2.0f;
        }
    const int units = q.cs / q.unit;  // of a row of threads
    int rows = q.ty, row = t.ty;
    bool writes = t.mine;
    const bool joined = q.tx < 64 && (q.tx & (q.tx - 1)) == 0;  // a wave holds whole rows
    if (joined) {
        rows = q.threads / 64, row = threadIdx.x / 64;
        writes = (int)(threadIdx.x % 64) < q.tx && t.tx * V < t.nc;
    }
    const bool even = t.np % q.ty == 0 && t.nc == q.cs;  // all threads have equal counts
#pragma unroll
    for (int v = 0; v < V; v++)
        if (v % q.unit == 0) {
            Stat s{m[v], t.mine ? count : 0.0f, d[v]};
            if (joined && even) {
                wave_steps(q.tx, [&](auto step) {
                    // the pair's lanes get the same bits: their sum, and the square of their difference
                    double ma, mb;
                    float da, db;
                    wave_pair<step.value>(s.m, ma, mb);
                    wave_pair<step.value>(s.d, da, db);
                    const float e = (float)(mb - ma);
                    s.m = 0.5 * (ma + mb);
                    s.d = (da + db) + e * e * (0.5f * s.n);
                    s.n *= 2.0f;
                });
            } else if (joined) {
                s = join_wave(s, q.tx);
            }
            if (writes) entry[row * units + (t.tx * V + v) / q.unit] = s;
        }
    __syncthreads();
    const int ng = t.groups(q), per = t.width(q) / q.unit;
    if (rows * per <= kSerial) {  // a thread a group
        for (int g = threadIdx.x; g < ng; g += q.threads) {
            Stat s = entry[g * per];
            for (int y = 0; y < rows; y++)
                for (int e = y == 0; e < per; e++) s = join(s, entry[y * units + g * per + e]);
            done(g, s);
        }
    } else {  // a wave a group
        const int lane = threadIdx.x % 64;
        for (int g = threadIdx.x / 64; g < ng; g += q.threads / 64) {
            Stat s{0.0, 0.0f, 0.0f};
            for (int e = lane; e < rows * per; e += 64) s = join(s, entry[e / per * units + g * per + e % per]);
            s = join_wave(s, 1);
            if (lane == 0) done(g, s);
        }
    }
    __syncthreads();
}

// Sums K values a thread has for each of its V channels over the threads of a channel, in a fixed order;
// chan[k * cs + channel] gets them.  Ends with a barrier.
template <int K, int V>
__device__ void channel_sums(const Plan &q, const Tile &t, float (&acc)[K][V], float *lds, float *chan) {
    const int cs = q.cs;
    int rows = q.ty, row = t.ty;
    bool writes = t.ty < q.ty;
    if (q.tx < 64 && (q.tx & (q.tx - 1)) == 0) {  // a wave holds whole rows: join them in registers first
        wave_steps(q.tx, [&](auto step) {
#pragma unroll
            for (int k = 0; k < K; k++)
#pragma unroll
                for (int v = 0; v < V; v++) {
                    float a, b;
                    wave_pair<step.value>(acc[k][v], a, b);
                    acc[k][v] = a + b;
                }
        });
        rows = q.threads / 64;
        row = threadIdx.x / 64;
        writes = (int)(threadIdx.x % 64) < q.tx;
    }
    if (writes)
#pragma unroll
        for (int k = 0; k < K; k++)
#pragma unroll
            for (int v = 0; v < V; v++) lds[(row * K + k) * cs + t.tx * V + v] = acc[k][v];
    __syncthreads();
    if (rows > kStatRows) {  // many rows: up to 16 threads a channel, in place
        int segs = q.threads / (K * cs);
        segs = segs < 1 ? 1 : segs > 16 ? 16 : segs;
        if (segs > 1) {
            const int seg = threadIdx.x / (K * cs), at = threadIdx.x % (K * cs);
            float s = 0.0f;
            if (seg < segs)
                for (int y = seg; y < rows; y += segs) s += lds[y * K * cs + at];
            __syncthreads();
            if (seg < segs) lds[seg * K * cs + at] = s;
            __syncthreads();
            rows = segs;
        }
    }
    for (int at = threadIdx.x; at < K * cs; at += q.threads) {
        float s = 0.0f;
        for (int y = 0; y < rows; y++) s += lds[y * K * cs + at];
        chan[at] = s;
    }
    __syncthreads();
}

// Sums chan (times gamma where given) over each group's channels: a wave a group, lanes strided, then a
// butterfly.  grp[k * stride + group].  Ends with a barrier.
template <int K>
__device__ void group_sums(const Plan &q, const Tile &t, const float *chan, int cs, const float *gamma, float *grp,
                           int stride) {
    const int ng = t.groups(q), gw = t.width(q), lane = threadIdx.x % 64;
    for (int g = threadIdx.x / 64; g < ng; g += q.threads / 64) {
        float s[K] = {};
        for (int j = lane; j < gw; j += 64) {
            const float w = gamma ? gamma[t.c0 + g * gw + j] : 1.0f;
#pragma unroll
            for (int k = 0; k < K; k++) s[k] += w * chan[k * cs + g * gw + j];
        }
#pragma unroll
        for (int k = 0; k < K; k++) s[k] = wave_reduce(s[k], [](float a, float b) { return a + b; });
        if (lane == 0)
#pragma unroll
            for (int k = 0; k < K; k++) grp[k * stride + g] = s[k];
    }
    __syncthreads();
}

// This thread's positions of the tile, U at a time with their loads ahead: fn(position's number, vectors).
template <typename T, int V, int U, int N, typename F>
__device__ __forceinline__ void each_position(const Plan &q, const Tile &t, const T *const (&at)[N], const int64_t (&pixel)[N], F fn) {
    if (!t.mine) return;
    for (int r = 0; t.ty + r * q.ty < t.np; r += U) {
        Words<T, V> v[U][N];
        const bool all = t.ty + (r + U - 1) * q.ty < t.np;
#pragma unroll
        for (int u = 0; u < U; u++)
            if (all || t.ty + (r + u) * q.ty < t.np)
#pragma unroll
                for (int j = 0; j < N; j++) v[u][j] = get_words<T, V>(at[j] + (int64_t)(r + u) * q.ty * pixel[j]);
#pragma unroll
        for (int u = 0; u < U; u++)
            if (all || t.ty + (r + u) * q.ty < t.np) {
                fn(r + u, v[u]);
                __builtin_amdgcn_sched_barrier(0);  // one vector's values in registers at a time, not U
            }
    }
}

// The affine part of y of a thread's channels: (x - m) s + b.
template <int V>
struct Affine {
    float m[V], s[V], b[V];
    template <typename Mean, typename Rstd>
    __device__ Affine(const Args &a, const Tile &t, Mean mean, Rstd rstd) {
        int g[V];
        t.groups_of<V>(a.q, g);
#pragma unroll
        for (int v = 0; v < V; v++) {
            const int64_t c = t.c0 + (t.mine ? t.tx * V + v : 0);
            m[v] = mean(g[v]);
            s[v] = rstd(g[v]) * (a.gamma ? a.gamma[c] : 1.0f);
            b[v] = a.beta ? a.beta[c] : 0.0f;
        }
    }
    __device__ __forceinline__ float z(float x, int v) const { return (x - m[v]) * s[v] + b[v]; }
};

template <int ACT, typename T, int V>
__device__ __forceinline__ Words<T, V> normalised(const Affine<V> &f, const Words<T, V> &x) {
    return Words<T, V>::of([&](int v) { return act_value<ACT>(f.z(x[v], v)); });
}

// Forward, a whole slice in registers.
template <typename T, int V, int R>
__global__ __launch_bounds__(kForwardThreads) void norm_whole_kernel(Args a) {
    extern __shared__ float lds[];
    const Plan &q = a.q;
    for (uint32_t b = blockIdx.x; b < 8 * q.per_xcd; b += gridDim.x) {
        const uint32_t tile = b % 8 * q.per_xcd + b / 8;
        if (tile >= q.tiles) continue;
        const Tile t(q, tile, V);
        float2 *grp = (float2 *)lds;  // means and rstd, in the room of as many Stats
        Words<T, V> x[R];
        const T *at = t.in<T>(a.x, a.xs, a.xp, V);
        int count = 0;
#pragma unroll
        for (int r = 0; r < R; r++)
            if (t.mine && t.ty + r * q.ty < t.np) x[r] = get_words<T, V>(at + (int64_t)r * q.ty * a.xp), count++;
        // counted from the thread's first value, x[0]
        float m[V] = {}, d[V] = {};
#pragma unroll
        for (int r = 1; r < R; r++)
            if (r < count)
#pragma unroll
                for (int v = 0; v < V; v++) m[v] += x[r][v] - x[0][v];
        const float inv = count ? __builtin_amdgcn_rcpf((float)count) : 0.0f;
#pragma unroll
        for (int v = 0; v < V; v++) m[v] *= inv;
#pragma unroll
        for (int r = 0; r < R; r++) x[r].keep();
#pragma unroll
        for (int r = 0; r < R; r++)
            if (r < count)
#pragma unroll
                for (int v = 0; v < V; v++) {
                    const float e = (x[r][v] - x[0][v]) - m[v];
                    d[v] += e * e;
                }
        double centre[V] = {};
        if (count)
#pragma unroll
            for (int v = 0; v < V; v++) centre[v] = (double)x[0][v] + (double)m[v];
#pragma unroll
        for (int r = 0; r < R; r++) x[r].keep();
        const float m1 = 1.0f / ((float)q.p * (float)q.gc);
        group_stats<V>(q, t, (float)count, centre, d, (Stat *)lds + q.head, [&](int g, const Stat &s) {
            const float mean = (float)s.m, rstd = 1.0f / sqrtf(s.d * m1 + a.eps);
            grp[g] = make_float2(mean, rstd);
            a.mean[t.i * q.groups + t.g0 + g] = mean;
            a.rstd[t.i * q.groups + t.g0 + g] = rstd;
        });
        auto mean = [&](int g) { return grp[g].x; };
        auto rstd = [&](int g) { return grp[g].y; };
        if (t.mine) {
            const Affine<V> f(a, t, mean, rstd);
            T *to = t.out<T>(a, V);
            with_act(a.act, [&](auto act) {
#pragma unroll
                for (int r = 0; r < R; r++)
                    if (r < count) {
                        put_words(to + (int64_t)r * q.ty * a.op, normalised<act.value>(f, x[r]));
                        __builtin_amdgcn_sched_barrier(0);
                    }
            });
        }
        __syncthreads();
    }
}

// Forward, first kernel of a large sample: the chunk's statistics.  A thread sums about its first value.
template <typename T, int V>
__global__ __launch_bounds__(256) void norm_stats_kernel(Args a) {
    extern __shared__ float lds[];
    const Plan &q = a.q;
    for (uint32_t b = blockIdx.x; b < 8 * q.per_xcd; b += gridDim.x) {
        const uint32_t tile = b % 8 * q.per_xcd + b / 8;
        if (tile >= q.tiles) continue;
        const Tile t(q, tile, V);
        float pivot[V] = {}, s[V] = {}, d[V] = {};
        int count = 0;
        const T *const at[1] = {t.in<T>(a.x, a.xs, a.xp, V)};
        const int64_t pixel[1] = {a.xp};
        each_position<T, V, 4, 1>(q, t, at, pixel, [&](int r, const Words<T, V>(&x)[1]) {
            if (r == 0)
#pragma unroll
                for (int v = 0; v < V; v++) pivot[v] = x[0][v];
#pragma unroll
            for (int v = 0; v < V; v++) {
                const float e = x[0][v] - pivot[v];
                s[v] += e, d[v] += e * e;
            }
            count++;
        });
        const float inv = count ? __builtin_amdgcn_rcpf((float)count) : 0.0f;
        double centre[V];
#pragma unroll
        for (int v = 0; v < V; v++) {
            // NaN and infinities go on as NaN; what rounding leaves below 0 does not
            const float e = d[v] - s[v] * s[v] * inv;
            d[v] = e < 0.0f ? 0.0f : e;
            centre[v] = (double)pivot[v] + (double)(s[v] * inv);
        }
        group_stats<V>(q, t, (float)count, centre, d, (Stat *)lds, [&](int g, const Stat &s) {
            a.stat[((t.i * q.groups + t.g0 + g) * q.chunks + t.chunk) * q.parts + t.part] = s;
        });
    }
}

// Second kernel of a large sample: joins the chunks' statistics, a wave a group.
__global__ __launch_bounds__(256) void norm_join_kernel(Args a) {
    const Plan &q = a.q;
    const int lane = threadIdx.x % 64;
    const uint32_t all = (uint32_t)q.n * q.groups, entries = q.chunks * q.parts;
    for (uint32_t group = blockIdx.x * 4 + threadIdx.x / 64; group < all; group += gridDim.x * 4) {
        Stat s{0.0, 0.0f, 0.0f};
        for (uint32_t e = lane; e < entries; e += 64) s = join(s, a.stat[(int64_t)group * entries + e]);
        s = join_wave(s, 1);
        if (lane == 0) {
            a.mean[group] = (float)s.m;
            a.rstd[group] = 1.0f / sqrtf(s.d / ((float)q.p * (float)q.gc) + a.eps);
        }
    }
}

// Third kernel of a large sample: normalises a chunk.
template <typename T, int V>
__global__ __launch_bounds__(256) void norm_apply_kernel(Args a) {
    const Plan &q = a.q;
    for (uint32_t b = blockIdx.x; b < 8 * q.per_xcd; b += gridDim.x) {
        const uint32_t tile = b % 8 * q.per_xcd + b / 8;
        if (tile >= q.tiles) continue;
        const Tile t(q, tile, V);
        if (!t.mine) continue;
        const float *mean = a.mean + t.i * q.groups + t.g0, *rstd = a.rstd + t.i * q.groups + t.g0;
        const Affine<V> f(a, t, [&](int g) { return mean[g]; }, [&](int g) { return rstd[g]; });
        T *to = t.out<T>(a, V);
        const T *const at[1] = {t.in<T>(a.x, a.xs, a.xp, V)};
        const int64_t pixel[1] = {a.xp};
        with_act(a.act, [&](auto act) {
            each_position<T, V, 4, 1>(q, t, at, pixel, [&](int r, const Words<T, V>(&x)[1]) {
                put_past_caches(to + (int64_t)r * q.ty * a.op, normalised<act.value>(f, x[0]));
            });
        });
    }
}

// dz of a value, for the sums and for dx
template <int ACT, int V>
__device__ __forceinline__ float slope_of(const Affine<V> &f, float x, float dy, int v) {
    return dy * act_slope<ACT>((x - f.m[v]) * f.s[v] + f.b[v]);
}

// A and B of this thread's values; B without rstd, which channel_total() multiplies
template <int ACT, typename T, int V>
__device__ __forceinline__ void add_values(const Affine<V> &f, const Words<T, V> &x, const Words<T, V> &dy, float (&acc)[2][V]) {
#pragma unroll
    for (int v = 0; v < V; v++) {
        const float e = x[v] - f.m[v];
        const float dz = slope_of<ACT>(f, x[v], dy[v], v);
        acc[0][v] += dz;
        acc[1][v] += dz * e;
    }
}

// dx = s dz + (x - m) k1 + k0 with s = rstd gamma, k1 = -rstd^2 S2, k0 = -rstd S1
template <int ACT, typename T, int V>
__device__ __forceinline__ Words<T, V> gradient(const Affine<V> &f, const float (&k1)[V], const float (&k0)[V], const Words<T, V> &x,
                                               const Words<T, V> &dy) {
    return Words<T, V>::of([&](int v) {
        const float e = x[v] - f.m[v];
        return slope_of<ACT>(f, x[v], dy[v], v) * f.s[v] + (e * k1[v] + k0[v]);
    });
}

// Backward, a whole slice in registers: the channels' A and B, and dx.  Up to four vectors a thread in 128 registers, so that two
// blocks share a compute unit: 64 x 14 x 14 x 1024 takes 33 (bf16) and 35 us (fp16, 7 values in memory) so, 42 with more.
template <typename T, int V, int R>
__global__ __launch_bounds__(kBackwardThreads, R <= 4 ? 4 : 2) void norm_backward_whole_kernel(Args a) {
    extern __shared__ float lds[];
    const Plan &q = a.q;
    const int cs = q.cs;
    for (uint32_t b = blockIdx.x; b < 8 * q.per_xcd; b += gridDim.x) {
        const uint32_t tile = b % 8 * q.per_xcd + b / 8;
        if (tile >= q.tiles) continue;
        const Tile t(q, tile, V);
        float *chan = lds, *grp = chan + 2 * cs, *rows = grp + 2 * cs;
        const float *mean = a.mean + t.i * q.groups + t.g0, *rstd = a.rstd + t.i * q.groups + t.g0;
        Words<T, V> x[R], dy[R];
        const T *xat = t.in<T>(a.x, a.xs, a.xp, V), *dat = t.in<T>(a.dy, a.ds, a.dp, V);
        int count = 0;
#pragma unroll
        for (int r = 0; r < R; r++)
            if (t.mine && t.ty + r * q.ty < t.np) {
                x[r] = get_words<T, V>(xat + (int64_t)r * q.ty * a.xp);
                dy[r] = get_words<T, V>(dat + (int64_t)r * q.ty * a.dp);
                count++;
            }
        const Affine<V> f(a, t, [&](int g) { return mean[g]; }, [&](int g) { return rstd[g]; });
        float acc[2][V] = {};
        with_act(a.act, [&](auto act) {
#pragma unroll
            for (int r = 0; r < R; r++)
                if (r < count) {
                    add_values<act.value>(f, x[r], dy[r], acc);
                    __builtin_amdgcn_sched_barrier(0);
                }
        });
#pragma unroll
        for (int r = 0; r < R; r++) x[r].keep(), dy[r].keep();
        channel_sums<2, V>(q, t, acc, rows, chan);
        for (int j = threadIdx.x; j < t.nc; j += q.threads) {
            chan[cs + j] *= rstd[j / (int)q.gc];
            a.total[t.i * q.c + t.c0 + j] = make_float2(chan[j], chan[cs + j]);
        }
        __syncthreads();
        group_sums<2>(q, t, chan, cs, a.gamma, grp, cs);
        if (t.mine) {
            const float inv = 1.0f / ((float)q.p * (float)q.gc);
            float k0[V], k1[V];
            int g[V];
            t.groups_of<V>(q, g);
#pragma unroll
            for (int v = 0; v < V; v++) {
                const float rs = rstd[g[v]];
                k0[v] = -rs * (grp[g[v]] * inv), k1[v] = -rs * (rs * (grp[cs + g[v]] * inv));
            }
            T *to = t.out<T>(a, V);
            with_act(a.act, [&](auto act) {
#pragma unroll
                for (int r = 0; r < R; r++)
                    if (r < count) {
                        put_words(to + (int64_t)r * q.ty * a.op, gradient<act.value>(f, k1, k0, x[r], dy[r]));
                        __builtin_amdgcn_sched_barrier(0);
                    }
            });
        }
        __syncthreads();
    }
}

// Backward, first kernel of a large sample: the channels' A and B of a chunk.
template <typename T, int V>
__global__ __launch_bounds__(256) void norm_backward_sums_kernel(Args a) {
    extern __shared__ float lds[];
    const Plan &q = a.q;
    const int cs = q.cs;
    for (uint32_t b = blockIdx.x; b < 8 * q.per_xcd; b += gridDim.x) {
        const uint32_t tile = b % 8 * q.per_xcd + b / 8;
        if (tile >= q.tiles) continue;
        const Tile t(q, tile, V);
        float *chan = lds, *rows = chan + 2 * cs;
        const float *mean = a.mean + t.i * q.groups + t.g0, *rstd = a.rstd + t.i * q.groups + t.g0;
        const Affine<V> f(a, t, [&](int g) { return mean[g]; }, [&](int g) { return rstd[g]; });
        float acc[2][V] = {};
        const T *const at[2] = {t.in<T>(a.x, a.xs, a.xp, V), t.in<T>(a.dy, a.ds, a.dp, V)};
        const int64_t pixel[2] = {a.xp, a.dp};
        with_act(a.act, [&](auto act) {
            each_position<T, V, 2, 2>(q, t, at, pixel, [&](int r, const Words<T, V>(&v)[2]) { add_values<act.value>(f, v[0], v[1], acc); });
        });
        channel_sums<2, V>(q, t, acc, rows, chan);
        const int w = t.width(q);
        for (int j = threadIdx.x; j < t.nc; j += q.threads)
            a.part[(t.i * q.chunks + t.chunk) * q.c + t.c0 + j] = make_float2(chan[j], chan[cs + j] * rstd[j / w]);
        __syncthreads();
    }
}

// Large samples: adds the chunks' A and B per channel, and S1 and S2 per group.  A block a group and sample.
__global__ __launch_bounds__(256) void norm_backward_totals_kernel(Args a) {
    __shared__ float sums[2][4];
    __shared__ float2 row[256];
    const Plan &q = a.q;
    const uint32_t all = (uint32_t)q.n * q.groups;
    for (uint32_t ig = blockIdx.x; ig < all; ig += gridDim.x) {
        const uint32_t i = ig / q.groups, g = ig - i * q.groups;
        // lanes of a channel: as many as fit, each takes chunks in turn
        const int gc = q.gc < 256 ? (int)q.gc : 256, lanes = min(256 / gc, 16);
        const int lane = threadIdx.x / gc, j = threadIdx.x - lane * gc;
        float s1 = 0.0f, s2 = 0.0f;
        for (uint32_t j0 = 0; j0 < q.gc; j0 += gc) {
            const int64_t c = (int64_t)g * q.gc + j0 + j;
            float A = 0.0f, B = 0.0f;
            if (j0 + j < q.gc && lane < lanes)
                for (uint32_t k = lane; k < q.chunks; k += lanes) {
                    const float2 v = a.part[((int64_t)i * q.chunks + k) * q.c + c];
                    A += v.x, B += v.y;
                }
            row[threadIdx.x] = make_float2(A, B);
            __syncthreads();
            if (j0 + j < q.gc && lane == 0) {
                for (int l = 1; l < lanes; l++) A += row[l * gc + j].x, B += row[l * gc + j].y;
                a.total[i * q.c + c] = make_float2(A, B);
                const float w = a.gamma ? a.gamma[c] : 1.0f;
                s1 += w * A, s2 += w * B;
            }
            __syncthreads();
        }
        s1 = wave_reduce(s1, [](float a, float b) { return a + b; }), s2 = wave_reduce(s2, [](float a, float b) { return a + b; });
        if (threadIdx.x % 64 == 0) sums[0][threadIdx.x / 64] = s1, sums[1][threadIdx.x / 64] = s2;
        __syncthreads();
        if (threadIdx.x == 0) {
            const float inv = 1.0f / ((float)q.p * (float)q.gc);
            a.sums[ig] = make_float2((sums[0][0] + sums[0][1] + sums[0][2] + sums[0][3]) * inv,
                                     (sums[1][0] + sums[1][1] + sums[1][2] + sums[1][3]) * inv);
        }
        __syncthreads();
    }
}

template <typename T, int V>
__global__ __launch_bounds__(256) void norm_backward_apply_kernel(Args a) {
    const Plan &q = a.q;
    for (uint32_t b = blockIdx.x; b < 8 * q.per_xcd; b += gridDim.x) {
        const uint32_t tile = b % 8 * q.per_xcd + b / 8;
        if (tile >= q.tiles) continue;
        const Tile t(q, tile, V);
        if (!t.mine) continue;
        const float *mean = a.mean + t.i * q.groups + t.g0, *rstd = a.rstd + t.i * q.groups + t.g0;
        const float2 *sums = a.sums + t.i * q.groups + t.g0;
        const Affine<V> f(a, t, [&](int g) { return mean[g]; }, [&](int g) { return rstd[g]; });
        float k0[V], k1[V];
        int g[V];
        t.groups_of<V>(q, g);
#pragma unroll
        for (int v = 0; v < V; v++) {
            const float rs = rstd[g[v]];
            const float2 s = sums[g[v]];
            k0[v] = -rs * s.x, k1[v] = -rs * (rs * s.y);
        }
        T *to = t.out<T>(a, V);
        const T *const at[2] = {t.in<T>(a.x, a.xs, a.xp, V), t.in<T>(a.dy, a.ds, a.dp, V)};
        const int64_t pixel[2] = {a.xp, a.dp};
        with_act(a.act, [&](auto act) {
            each_position<T, V, 2, 2>(q, t, at, pixel, [&](int r, const Words<T, V>(&v)[2]) {
                put_past_caches(to + (int64_t)r * q.ty * a.op, gradient<act.value>(f, k1, k0, v[0], v[1]));
            });
        });
    }
}

// dgamma and dbeta: the samples' B and A added in a fixed order.  32 channels a block, 32 rows at a time.
__global__ __launch_bounds__(1024) void norm_parameters_kernel(const float2 *total, int64_t n, int64_t c, float *dgamma,
                                                               float *dbeta) {
    __shared__ float2 row[32][33];
    const int lane = threadIdx.x % 32, y = threadIdx.x / 32;
    const int64_t j = (int64_t)blockIdx.x * 32 + lane;
    float A = 0.0f, B = 0.0f;
    if (j < c)
        for (int64_t i = y; i < n; i += 32) {
            const float2 v = total[i * c + j];
            A += v.x, B += v.y;
        }
    row[y][lane] = make_float2(A, B);
    __syncthreads();
    if (y == 0 && j < c) {
        for (int k = 1; k < 32; k++) A += row[k][lane].x, B += row[k][lane].y;
        dbeta[j] = A, dgamma[j] = B;
    }
}

__global__ void norm_empty_kernel(float *mean, float *rstd, int64_t count, float eps) {
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < count; i += (int64_t)gridDim.x * blockDim.x)
        mean[i] = 0.0f, rstd[i] = 1.0f / sqrtf(eps);
}

unsigned grid_of(int64_t tiles) { return (unsigned)(tiles < kMaxGrid ? tiles : kMaxGrid); }

// rows of threads that leave an entry in LDS
size_t lds_rows(const Plan &q) { return q.tx < 64 && (q.tx & (q.tx - 1)) == 0 ? q.threads / 64 : q.ty; }

size_t stat_bytes(const Plan &q) { return sizeof(Stat) * (q.head + lds_rows(q) * (q.cs / q.unit)); }

size_t sum_bytes(const Plan &q, int head) { return sizeof(float) * q.cs * (head + 2 * lds_rows(q)); }

template <typename T, int V>
int launch_forward(const Args &a, hipStream_t s) {
    const unsigned grid = grid_of((int64_t)8 * a.q.per_xcd);
    const int threads = a.q.threads;
    const size_t lds = stat_bytes(a.q);
    switch (a.q.r) {
        case 1: norm_whole_kernel<T, V, 1><<<grid, threads, lds, s>>>(a); break;
        case 2: norm_whole_kernel<T, V, 2><<<grid, threads, lds, s>>>(a); break;
        case 4: norm_whole_kernel<T, V, 4><<<grid, threads, lds, s>>>(a); break;
        case 8: norm_whole_kernel<T, V, 8><<<grid, threads, lds, s>>>(a); break;
        default: {
            norm_stats_kernel<T, V><<<grid, threads, lds, s>>>(a);
            BYZ_HIP(hipGetLastError());
            norm_join_kernel<<<grid_of((a.q.n * a.q.groups + 3) / 4), 256, 0, s>>>(a);
            BYZ_HIP(hipGetLastError());
            const Args again = pass_again(a);
            norm_apply_kernel<T, V><<<grid_of((int64_t)8 * again.q.per_xcd), threads, 0, s>>>(again);
        }
    }
    BYZ_HIP(hipGetLastError());
    return BYZ_OK;
}

template <typename T, int V>
int launch_backward(const Args &a, hipStream_t s) {
    const unsigned grid = grid_of((int64_t)8 * a.q.per_xcd);
    const int threads = a.q.threads;
    switch (a.q.r) {
        case 1: norm_backward_whole_kernel<T, V, 1><<<grid, threads, sum_bytes(a.q, 4), s>>>(a); break;
        case 2: norm_backward_whole_kernel<T, V, 2><<<grid, threads, sum_bytes(a.q, 4), s>>>(a); break;
        case 4: norm_backward_whole_kernel<T, V, 4><<<grid, threads, sum_bytes(a.q, 4), s>>>(a); break;
        case 8: norm_backward_whole_kernel<T, V, 8><<<grid, threads, sum_bytes(a.q, 4), s>>>(a); break;
        default: {
            norm_backward_sums_kernel<T, V><<<grid, threads, sum_bytes(a.q, 2), s>>>(a);
            BYZ_HIP(hipGetLastError());
            norm_backward_totals_kernel<<<grid_of(a.q.n * a.q.groups), 256, 0, s>>>(a);
            BYZ_HIP(hipGetLastError());
            const Args again = pass_again(a);
            norm_backward_apply_kernel<T, V><<<grid_of((int64_t)8 * again.q.per_xcd), threads, 0, s>>>(again);
        }
    }
    BYZ_HIP(hipGetLastError());
    if (a.dgamma) {
        norm_parameters_kernel<<<(unsigned)((a.q.c + 31) / 32), 1024, 0, s>>>(a.total, a.q.n, a.q.c, a.dgamma, a.dbeta);
        BYZ_HIP(hipGetLastError());
    }
    return BYZ_OK;
}

template <typename T, bool FORWARD>
int launch_vec(const Args &a, hipStream_t s) {
    constexpr int wide = 16 / sizeof(T), narrow = 4 / sizeof(T);
    if (a.q.vec == wide) return FORWARD ? launch_forward<T, wide>(a, s) : launch_backward<T, wide>(a, s);
    if constexpr (narrow > 1)
        if (a.q.vec == narrow) return FORWARD ? launch_forward<T, narrow>(a, s) : launch_backward<T, narrow>(a, s);
    return FORWARD ? launch_forward<T, 1>(a, s) : launch_backward<T, 1>(a, s);
}

template <bool FORWARD>
int launch(const Args &a, int dtype, hipStream_t s) {
    if (dtype == BYZ_F32) return launch_vec<float, FORWARD>(a, s);
    if (dtype == BYZ_BF16) return launch_vec<bf16, FORWARD>(a, s);
    return launch_vec<f16, FORWARD>(a, s);
}

size_t round_up(size_t bytes) { return (bytes + 255) / 256 * 256; }

bool sizes_ok(int64_t n, int64_t p, int64_t c, int groups, int dtype) {
    int64_t all;
    return n >= 0 && p >= 0 && c >= 1 && groups >= 1 && c % groups == 0 && dtype_known(dtype) && c <= (1 << 24) &&
           !__builtin_mul_overflow(n, p, &all) && !__builtin_mul_overflow(all, c, &all) && all <= (INT64_MAX >> 8);
}

size_t forward_bytes(const Plan &q) { return whole(q) ? 0 : round_up(sizeof(Stat) * q.n * q.groups * q.chunks * q.parts); }

struct BackwardLayout {
    size_t total, sums, part, bytes;
    explicit BackwardLayout(const Plan &q) {
        total = 0;
        sums = round_up(sizeof(float2) * q.n * q.c);
        part = sums + (whole(q) ? 0 : round_up(sizeof(float2) * q.n * q.groups));
        bytes = part + (whole(q) ? 0 : round_up(sizeof(float2) * q.n * q.chunks * q.c));
    }
};

}  // namespace

extern "C" size_t byz_group_norm_workspace_bytes(int64_t n, int64_t p, int64_t c, int groups, int dtype) {
    if (!sizes_ok(n, p, c, groups, dtype) || n == 0 || p == 0) return 0;
    Plan q;
    return make_plan(q, n, p, c, groups, (int)dtype_size(dtype), true) ? forward_bytes(q) : 0;
}

extern "C" int byz_group_norm(const void *x, int64_t x_sample, int64_t x_pixel, int64_t n, int64_t p, int64_t c,
                              int groups, int dtype, const float *gamma, const float *beta, float eps, int act,
                              void *y, int64_t y_sample, int64_t y_pixel, float *mean, float *rstd, void *workspace,
                              size_t workspace_bytes, void *stream) {
    if (!sizes_ok(n, p, c, groups, dtype) || !act_known(act) || !(eps >= 0.0f) || !(eps < INFINITY)) return BYZ_EINVAL;
    const hipStream_t s = (hipStream_t)stream;
    if (n == 0) return BYZ_OK;
    if (!mean || !rstd) return BYZ_EINVAL;
    if (p == 0) {
        norm_empty_kernel<<<(unsigned)std::min<int64_t>((n * groups + 255) / 256, 4096), 256, 0, s>>>(mean, rstd, n * groups, eps);
        BYZ_HIP(hipGetLastError());
        return BYZ_OK;
    }
    const int elem = (int)dtype_size(dtype);
    if (!x || !y || !aligned(x, elem) || !aligned(y, elem)) return BYZ_EINVAL;
    for (int64_t pixel : {x_pixel, y_pixel})
        if (pixel < c || !extent_ok(p, pixel, c)) return BYZ_EINVAL;
    if (!extent_ok(n, x_sample, (p - 1) * x_pixel + c) || !extent_ok(n, y_sample, (p - 1) * y_pixel + c)) return BYZ_EINVAL;
    if (n > 1 && y_sample < (p - 1) * y_pixel + c) return BYZ_EINVAL;  // samples of the output may not overlap
    Args a{};
    if (!make_plan(a.q, n, p, c, groups, elem, true)) return BYZ_EUNSUPPORTED;
    if (forward_bytes(a.q) > workspace_bytes || (forward_bytes(a.q) && (!workspace || !aligned(workspace, 16)))) return BYZ_ENOMEM;
    a.x = x, a.xs = x_sample, a.xp = x_pixel;
    a.out = y, a.os = y_sample, a.op = y_pixel;
    a.gamma = gamma, a.beta = beta, a.mean = mean, a.rstd = rstd, a.eps = eps, a.act = act;
    a.stat = (Stat *)workspace;
    return launch<true>(a, dtype, s);
}

extern "C" size_t byz_group_norm_backward_workspace_bytes(int64_t n, int64_t p, int64_t c, int groups, int dtype) {
    if (!sizes_ok(n, p, c, groups, dtype) || n == 0 || p == 0) return 0;
    Plan q;
    return make_plan(q, n, p, c, groups, (int)dtype_size(dtype), false) ? BackwardLayout(q).bytes : 0;
}

extern "C" int byz_group_norm_backward(const void *dy, int64_t dy_sample, int64_t dy_pixel, const void *x,
                                       int64_t x_sample, int64_t x_pixel, int64_t n, int64_t p, int64_t c, int groups,
                                       int dtype, const float *gamma, const float *beta, const float *mean,
                                       const float *rstd, int act, void *dx, int64_t dx_sample, int64_t dx_pixel,
                                       float *dgamma, float *dbeta, void *workspace, size_t workspace_bytes,
                                       void *stream) {
    if (!sizes_ok(n, p, c, groups, dtype) || !act_known(act) || !dgamma != !dbeta) return BYZ_EINVAL;
    const hipStream_t s = (hipStream_t)stream;
    const int elem = (int)dtype_size(dtype);
    Args a{};
    if (n == 0 || p == 0) {
        if (dgamma) {
            norm_parameters_kernel<<<(unsigned)((c + 31) / 32), 1024, 0, s>>>(nullptr, 0, c, dgamma, dbeta);
            BYZ_HIP(hipGetLastError());
        }
        return BYZ_OK;
    }
    if (!dy || !x || !dx || !mean || !rstd || !aligned(dy, elem) || !aligned(x, elem) || !aligned(dx, elem)) return BYZ_EINVAL;
    for (int64_t pixel : {dy_pixel, x_pixel, dx_pixel})
        if (pixel < c || !extent_ok(p, pixel, c)) return BYZ_EINVAL;
    if (!extent_ok(n, dy_sample, (p - 1) * dy_pixel + c) || !extent_ok(n, x_sample, (p - 1) * x_pixel + c) ||
        !extent_ok(n, dx_sample, (p - 1) * dx_pixel + c))
        return BYZ_EINVAL;
    if (n > 1 && dx_sample < (p - 1) * dx_pixel + c) return BYZ_EINVAL;
    if (!make_plan(a.q, n, p, c, groups, elem, false)) return BYZ_EUNSUPPORTED;
    const BackwardLayout lay(a.q);
    if (!workspace || lay.bytes > workspace_bytes || !aligned(workspace, 16)) return BYZ_ENOMEM;
    a.x = x, a.xs = x_sample, a.xp = x_pixel;
    a.dy = dy, a.ds = dy_sample, a.dp = dy_pixel;
    a.out = dx, a.os = dx_sample, a.op = dx_pixel;
    a.gamma = gamma, a.beta = beta, a.mean = const_cast<float *>(mean), a.rstd = const_cast<float *>(rstd), a.act = act;
    a.total = (float2 *)((char *)workspace + lay.total);
    a.sums = (float2 *)((char *)workspace + lay.sums);
    a.part = (float2 *)((char *)workspace + lay.part);
    a.dgamma = dgamma, a.dbeta = dbeta;
    return launch<false>(a, dtype, s);
}

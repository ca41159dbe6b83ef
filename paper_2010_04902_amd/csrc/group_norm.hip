// Group norm with an activation on channels-last features, forward and backward (gfx950).
//
// A sample is a p x c matrix, a group a strip of c / groups of its columns.  A block takes a slice:
// some whole groups (or a part of one wide group), all positions or a chunk of them.  Thread t holds the
// same V channels at positions t / tx, t / tx + ty, ...: its values stay in registers as they were loaded.
//
//   forward    mean of the tile, then the sum of squared distances from it (both from registers, so no
//              difference of large sums), then act(xhat gamma + beta).
//   backward   with xhat and the activation's slope recomputed, dz = dy act'(z): per channel the
//              sums A of dz and B of dz xhat are all that is needed,
//                  dbeta = sum A,  dgamma = sum B  (over the samples, in order),
//                  S1 = sum gamma A / m,  S2 = sum gamma B / m  (over a group's channels),
//                  dx = rstd (gamma dz - S1 - xhat S2).
//
// Bound by memory: 2 values moved per value forward, 3 backward, a dozen operations each.  Where a slice
// of a sample fits the registers of one block ("whole") everything is read once.  Larger samples are cut into
// chunks: their statistics are written by a first kernel, joined by the second in chunk order (pairwise
// update of mean and squared distances), which reads the chunk again.  No atomics.
#include <type_traits>

#include "worker_internal.h"

using namespace byz_worker;

namespace {

constexpr int kMaxThreads = 1024;
constexpr int kMaxLanes = 256;         // most vectors of a slice's row
constexpr int64_t kMaxGrid = 1 << 20;  // blocks of a launch; more tiles are taken in turn

struct Plan {
    int64_t n, p, c, groups, gc;  // gc: channels of a group
    int vec, cs, tx, ty, threads, r;
    int parts;                    // blocks that share a group's channels (1: a slice has whole groups)
    int64_t slices, chunk, chunks, tiles;
};

struct View {
    const void *at;
    int64_t sample, pixel;
};

int64_t gcd(int64_t a, int64_t b) { return b ? gcd(b, a % b) : a; }

// Largest number of neighbouring elements that all views load in one piece.
int widest_vec(int elem, int64_t c, std::initializer_list<View> views) {
    for (int vec : {16 / elem, 4 / elem, 1}) {
        if (vec < 1 || c % vec) continue;
        bool ok = true;
        for (const View &v : views)
            ok = ok && aligned(v.at, (size_t)vec * elem) && v.sample % vec == 0 && v.pixel % vec == 0;
        if (ok) return vec;
    }
    return 1;
}

// `regs`: 16-byte vectors that a thread holds of each tensor at most.
Plan make_plan(int64_t n, int64_t p, int64_t c, int64_t groups, int elem, int vec, int max_r) {
    Plan q{};
    q.n = n, q.p = p, q.c = c, q.groups = groups, q.gc = c / groups;
    // a slice of whole groups whose rows start at multiples of vec, or a part of one group; narrower
    // vectors where neither is possible
    for (;; vec = vec > 4 / elem ? (4 / elem > 1 ? 4 / elem : 1) : 1) {
        const int64_t step = q.gc / gcd(q.gc, vec) * vec;
        if (step / vec <= kMaxLanes) {
            int64_t cs = step;
            while (cs * elem < 128 && cs + step <= c) cs += step;
            q.cs = (int)cs, q.parts = 1;
            q.slices = (c + cs - 1) / cs;
            break;
        }
        if (q.gc % vec == 0) {
            const int64_t lanes = q.gc / vec, parts = (lanes + kMaxLanes - 1) / kMaxLanes;
            q.cs = (int)((lanes + parts - 1) / parts) * vec;
            q.parts = (int)((q.gc + q.cs - 1) / q.cs);
            q.slices = groups * q.parts;
            break;
        }
    }
    q.vec = vec;
    q.tx = q.cs / vec;
    // four vectors a thread where that gives enough threads, max_r of them at most
    const int64_t vectors = p * q.tx;
    int64_t threads = (vectors + 3) / 4;
    threads = threads < 64 ? 64 : threads > kMaxThreads ? kMaxThreads : (threads + 63) / 64 * 64;
    if (threads < q.tx) threads = (q.tx + 63) / 64 * 64;
    q.threads = (int)threads;
    q.ty = q.threads / q.tx;
    int64_t r = (p + q.ty - 1) / q.ty;
    if (r > max_r || q.parts > 1) {
        q.threads = q.tx > 128 ? 512 : 256;
        q.ty = q.threads / q.tx;
        r = max_r < 8 ? max_r : 8;
        if (r > (p + q.ty - 1) / q.ty) r = (p + q.ty - 1) / q.ty;
    }
    q.r = r <= 1 ? 1 : r <= 2 ? 2 : r <= 4 ? 4 : r <= 8 ? 8 : 16;
    q.chunk = (int64_t)q.ty * q.r;
    q.chunks = (p + q.chunk - 1) / q.chunk;
    q.tiles = n * q.chunks * q.slices;
    return q;
}

bool whole(const Plan &q) { return q.chunks == 1 && q.parts == 1; }

struct Args {
    Plan q;
    const void *x, *dy;
    void *out;  // y or dx
    int64_t xs, xp, ds, dp, os, op;
    const float *gamma, *beta;
    float *mean, *rstd;
    float eps;
    int act;
    float2 *part;   // forward: (mean, squared distances) of [sample][group][chunk][part]; backward: (A, B) of [sample][chunk][channel]
    float2 *total;  // backward: (A, B) of [sample][channel]
    float2 *sums;   // backward: (S1, S2) of [sample][group]
    float *dgamma, *dbeta;
};

// What a block works on.
struct Tile {
    int64_t i, chunk, slice, p0, c0;  // sample, chunk, slice, first position, first channel
    int np, nc;                       // positions, channels
    int part;
    int tx, ty;                       // this thread's vector and first position; nc / V <= tx: idle
    __device__ Tile(const Plan &q, int64_t t, int V) {
        slice = t % q.slices;
        chunk = t / q.slices % q.chunks;
        i = t / q.slices / q.chunks;
        p0 = chunk * q.chunk;
        np = (int)(q.p - p0 < q.chunk ? q.p - p0 : q.chunk);
        const int64_t g = q.parts > 1 ? slice / q.parts : 0;
        part = q.parts > 1 ? (int)(slice % q.parts) : 0;
        c0 = q.parts > 1 ? g * q.gc + (int64_t)part * q.cs : slice * q.cs;
        const int64_t end = q.parts > 1 ? (g + 1) * q.gc : q.c;
        nc = (int)(end - c0 < q.cs ? end - c0 : q.cs);
        tx = threadIdx.x % q.tx;
        ty = threadIdx.x / q.tx;
        if (ty >= q.ty) tx = q.tx, ty = 0;  // threads beyond the last whole row of them
    }
    __device__ int groups(const Plan &q) const { return q.parts > 1 ? 1 : nc / (int)q.gc; }
    __device__ int64_t first_group(const Plan &q) const { return c0 / q.gc; }
    __device__ int group_width(const Plan &q) const { return q.parts > 1 ? nc : (int)q.gc; }
};

// Sums K values a thread has for each of its V channels over the threads of a channel, in a fixed order;
// chan[k * cs + channel] gets them.  Ends with a barrier.
template <int K, int V>
__device__ void channel_sums(const Plan &q, const Tile &t, float (&acc)[K][V], float *lds, float *chan) {
    const int cs = q.tx * V;
    int rows = q.ty, row = t.ty;
    bool writes = t.tx < q.tx;
    if (q.tx < 64 && (q.tx & (q.tx - 1)) == 0) {  // a wave holds whole rows: join them in registers first
#pragma unroll
        for (int k = 0; k < K; k++)
#pragma unroll
            for (int v = 0; v < V; v++)
                for (int off = q.tx; off < 64; off *= 2) acc[k][v] += __shfl_xor(acc[k][v], off);
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
    int stride = 1;
    if (rows > 16) {  // many rows: 16 threads a channel where there are enough, in place
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
        for (int y = 0; y < rows; y += stride) s += lds[y * K * cs + at];
        chan[at] = s;
    }
    __syncthreads();
}

// Sums chan (times gamma where given) over each group's channels: a wave a group, lanes strided, then a
// butterfly.  grp[k * kStride + group].  Ends with a barrier.
template <int K>
__device__ void group_sums(const Plan &q, const Tile &t, const float *chan, int cs, const float *gamma, float *grp,
                           int stride) {
    const int ng = t.groups(q), gw = t.group_width(q), lane = threadIdx.x % 64;
    for (int g = threadIdx.x / 64; g < ng; g += q.threads / 64) {
        float s[K] = {};
        for (int j = lane; j < gw; j += 64) {
            const float w = gamma ? gamma[t.c0 + g * gw + j] : 1.0f;
#pragma unroll
            for (int k = 0; k < K; k++) s[k] += w * chan[k * cs + g * gw + j];
        }
#pragma unroll
        for (int k = 0; k < K; k++)
            for (int off = 32; off; off >>= 1) s[k] += __shfl_xor(s[k], off);
        if (lane == 0)
#pragma unroll
            for (int k = 0; k < K; k++) grp[k * stride + g] = s[k];
    }
    __syncthreads();
}

// (count, mean, squared distances) of two sets joined
__device__ __forceinline__ void join(float &na, float &ma, float &qa, float nb, float mb, float qb) {
    const float n = na + nb;
    if (nb == 0.0f) return;
    const float d = mb - ma, f = nb / n;
    ma = na == 0.0f ? mb : ma + d * f;
    qa = na == 0.0f ? qb : qa + qb + d * d * na * f;
    na = n;
}

template <typename T, int V, int R>
__device__ void load_tile(const Tile &t, const Plan &q, const void *base, int64_t sample, int64_t pixel,
                          Pack<T, V> (&v)[R]) {
    const T *at = (const T *)base + t.i * sample + (t.p0 + t.ty) * pixel + t.c0 + t.tx * V;
    const bool mine = t.tx * V < t.nc;
#pragma unroll
    for (int r = 0; r < R; r++) {
        if (mine && t.ty + r * q.ty < t.np)
            v[r] = *(const Pack<T, V> *)(at + (int64_t)r * q.ty * pixel);
        else
#pragma unroll
            for (int k = 0; k < V; k++) v[r].v[k] = (T)0.0f;
    }
}

template <typename T, int V, int R, bool WHOLE>
__global__ __launch_bounds__(kMaxThreads) void norm_forward_kernel(Args a) {
    extern __shared__ float lds[];
    const Plan &q = a.q;
    const int cs = q.cs;
    for (int64_t tile = blockIdx.x; tile < q.tiles; tile += gridDim.x) {
        const Tile t(q, tile, V);
        // chan | group means | group squared distances | reduction's rows
        float *chan = lds, *gmean = chan + cs, *gdist = gmean + cs, *rows = gdist + cs;
        Pack<T, V> x[R];
        load_tile<T, V, R>(t, q, a.x, a.xs, a.xp, x);
        const float inv = 1.0f / ((float)t.np * (float)t.group_width(q));
        float acc[1][V] = {};
#pragma unroll
        for (int r = 0; r < R; r++)
#pragma unroll
            for (int v = 0; v < V; v++) acc[0][v] += (float)x[r].v[v];
        channel_sums<1, V>(q, t, acc, rows, chan);
        group_sums<1>(q, t, chan, cs, nullptr, gmean, cs);
        const bool mine = t.tx * V < t.nc;
        const int gw = t.group_width(q);
        int g[V];
        float m[V];
#pragma unroll
        for (int v = 0; v < V; v++) {
            g[v] = mine ? (t.tx * V + v) / gw : 0;
            m[v] = gmean[g[v]] * inv;
            acc[0][v] = 0.0f;
        }
#pragma unroll
        for (int r = 0; r < R; r++)
            if (mine && t.ty + r * q.ty < t.np)
#pragma unroll
                for (int v = 0; v < V; v++) {
                    const float d = (float)x[r].v[v] - m[v];
                    acc[0][v] += d * d;
                }
        __syncthreads();
        channel_sums<1, V>(q, t, acc, rows, chan);
        group_sums<1>(q, t, chan, cs, nullptr, gdist, cs);
        if constexpr (!WHOLE) {
            for (int j = threadIdx.x; j < t.groups(q); j += q.threads)
                a.part[((t.i * q.groups + t.first_group(q) + j) * q.chunks + t.chunk) * q.parts + t.part] =
                    make_float2(gmean[j] * inv, gdist[j]);
        } else {
            for (int j = threadIdx.x; j < t.groups(q); j += q.threads) {
                a.mean[t.i * q.groups + t.first_group(q) + j] = gmean[j] * inv;
                a.rstd[t.i * q.groups + t.first_group(q) + j] = 1.0f / sqrtf(gdist[j] * inv + a.eps);
            }
            if (mine) {
                float s[V], b[V];
#pragma unroll
                for (int v = 0; v < V; v++) {
                    const int64_t c = t.c0 + t.tx * V + v;
                    s[v] = 1.0f / sqrtf(gdist[g[v]] * inv + a.eps);
                    s[v] *= a.gamma ? a.gamma[c] : 1.0f;
                    b[v] = a.beta ? a.beta[c] : 0.0f;
                }
                T *at = (T *)a.out + t.i * a.os + (t.p0 + t.ty) * a.op + t.c0 + t.tx * V;
                with_act(a.act, [&](auto act) {
#pragma unroll
                    for (int r = 0; r < R; r++)
                        if (t.ty + r * q.ty < t.np) {
                            Pack<T, V> y;
#pragma unroll
                            for (int v = 0; v < V; v++)
                                y.v[v] = round_to<T>(act_value<act.value>(((float)x[r].v[v] - m[v]) * s[v] + b[v]));
                            *(Pack<T, V> *)(at + (int64_t)r * q.ty * a.op) = y;
                        }
                });
            }
        }
        __syncthreads();
    }
}

// Second kernel of a large sample: joins the chunks' statistics, normalises its chunk.
template <typename T, int V, int R>
__global__ __launch_bounds__(512) void norm_apply_kernel(Args a) {
    extern __shared__ float lds[];
    const Plan &q = a.q;
    for (int64_t tile = blockIdx.x; tile < q.tiles; tile += gridDim.x) {
        const Tile t(q, tile, V);
        float *gmean = lds, *grstd = lds + q.cs;
        Pack<T, V> x[R];
        load_tile<T, V, R>(t, q, a.x, a.xs, a.xp, x);
        const int ng = t.groups(q), lane = threadIdx.x % 64;
        const int64_t entries = q.chunks * q.parts;
        for (int g = threadIdx.x / 64; g < ng; g += q.threads / 64) {
            const int64_t group = t.first_group(q) + g;
            float n = 0.0f, m = 0.0f, d = 0.0f;
            for (int64_t e = lane; e < entries; e += 64) {
                const int64_t np = min(q.chunk, q.p - e / q.parts * q.chunk);
                const int64_t nc = q.parts > 1 ? min((int64_t)q.cs, q.gc - e % q.parts * q.cs) : q.gc;
                const float2 v = a.part[(t.i * q.groups + group) * entries + e];
                join(n, m, d, (float)(np * nc), v.x, v.y);
            }
            for (int off = 1; off < 64; off *= 2) {
                // both sides of a pair join in the same order and get the same values
                const float n2 = __shfl_xor(n, off), m2 = __shfl_xor(m, off), d2 = __shfl_xor(d, off);
                if (lane & off) {
                    float n1 = n2, m1 = m2, d1 = d2;
                    join(n1, m1, d1, n, m, d);
                    n = n1, m = m1, d = d1;
                } else {
                    join(n, m, d, n2, m2, d2);
                }
            }
            if (lane == 0) {
                const float rstd = 1.0f / sqrtf(d / ((float)q.p * (float)q.gc) + a.eps);
                gmean[g] = m, grstd[g] = rstd;
                if (t.chunk == 0 && t.part == 0) {
                    a.mean[t.i * q.groups + group] = m;
                    a.rstd[t.i * q.groups + group] = rstd;
                }
            }
        }
        __syncthreads();
        if (t.tx * V < t.nc) {
            const int gw = t.group_width(q);
            float m[V], s[V], b[V];
#pragma unroll
            for (int v = 0; v < V; v++) {
                const int g = (t.tx * V + v) / gw;
                const int64_t c = t.c0 + t.tx * V + v;
                m[v] = gmean[g];
                s[v] = grstd[g] * (a.gamma ? a.gamma[c] : 1.0f);
                b[v] = a.beta ? a.beta[c] : 0.0f;
            }
            T *at = (T *)a.out + t.i * a.os + (t.p0 + t.ty) * a.op + t.c0 + t.tx * V;
            with_act(a.act, [&](auto act) {
#pragma unroll
                for (int r = 0; r < R; r++)
                    if (t.ty + r * q.ty < t.np) {
                        Pack<T, V> y;
#pragma unroll
                        for (int v = 0; v < V; v++)
                            y.v[v] = round_to<T>(act_value<act.value>(((float)x[r].v[v] - m[v]) * s[v] + b[v]));
                        *(Pack<T, V> *)(at + (int64_t)r * q.ty * a.op) = y;
                    }
            });
        }
        __syncthreads();
    }
}

// What a thread needs of its V channels in the backward pass.
template <int V>
struct Channel {
    float m[V], rs[V], gamma[V], beta[V];
    __device__ Channel(const Args &a, const Tile &t) {
        const bool mine = t.tx * V < t.nc;
#pragma unroll
        for (int v = 0; v < V; v++) {
            const int64_t c = t.c0 + (mine ? t.tx * V + v : 0);
            const int64_t g = t.i * a.q.groups + c / a.q.gc;
            m[v] = a.mean[g], rs[v] = a.rstd[g];
            gamma[v] = a.gamma ? a.gamma[c] : 1.0f;
            beta[v] = a.beta ? a.beta[c] : 0.0f;
        }
    }
};

template <typename T, int V, int R>
__device__ void store_dx(const Args &a, const Tile &t, const Channel<V> &ch, const float (&s1)[V], const float (&s2)[V],
                         const Pack<T, V> (&x)[R], const Pack<T, V> (&dy)[R]) {
    T *at = (T *)a.out + t.i * a.os + (t.p0 + t.ty) * a.op + t.c0 + t.tx * V;
    with_act(a.act, [&](auto act) {
#pragma unroll
        for (int r = 0; r < R; r++)
            if (t.ty + r * a.q.ty < t.np) {
                Pack<T, V> d;
#pragma unroll
                for (int v = 0; v < V; v++) {
                    const float xh = ((float)x[r].v[v] - ch.m[v]) * ch.rs[v];
                    const float dz = (float)dy[r].v[v] * act_slope<act.value>(xh * ch.gamma[v] + ch.beta[v]);
                    d.v[v] = round_to<T>(ch.rs[v] * (ch.gamma[v] * dz - s1[v] - xh * s2[v]));
                }
                *(Pack<T, V> *)(at + (int64_t)r * a.q.ty * a.op) = d;
            }
    });
}

// First kernel of the backward pass: the channels' A and B; whole samples: dx too.
template <typename T, int V, int R, bool WHOLE>
__global__ __launch_bounds__(kMaxThreads) void norm_backward_kernel(Args a) {
    extern __shared__ float lds[];
    const Plan &q = a.q;
    const int cs = q.cs;
    for (int64_t tile = blockIdx.x; tile < q.tiles; tile += gridDim.x) {
        const Tile t(q, tile, V);
        float *chan = lds, *grp = chan + 2 * cs, *rows = grp + 2 * cs;
        Pack<T, V> x[R], dy[R];
        load_tile<T, V, R>(t, q, a.x, a.xs, a.xp, x);
        load_tile<T, V, R>(t, q, a.dy, a.ds, a.dp, dy);
        const Channel<V> ch(a, t);
        const bool mine = t.tx * V < t.nc;
        float acc[2][V] = {};
        if (mine)
            with_act(a.act, [&](auto act) {
#pragma unroll
                for (int r = 0; r < R; r++)
                    if (t.ty + r * q.ty < t.np)
#pragma unroll
                        for (int v = 0; v < V; v++) {
                            const float xh = ((float)x[r].v[v] - ch.m[v]) * ch.rs[v];
                            const float dz = (float)dy[r].v[v] * act_slope<act.value>(xh * ch.gamma[v] + ch.beta[v]);
                            acc[0][v] += dz;
                            acc[1][v] += dz * xh;
                        }
            });
        channel_sums<2, V>(q, t, acc, rows, chan);
        float2 *to = WHOLE ? a.total + t.i * q.c : a.part + (t.i * q.chunks + t.chunk) * q.c;
        for (int j = threadIdx.x; j < t.nc; j += q.threads) to[t.c0 + j] = make_float2(chan[j], chan[cs + j]);
        if constexpr (WHOLE) {
            group_sums<2>(q, t, chan, cs, a.gamma, grp, cs);
            if (mine) {
                const float inv = 1.0f / ((float)q.p * (float)q.gc);
                float s1[V], s2[V];
#pragma unroll
                for (int v = 0; v < V; v++) {
                    const int g = (t.tx * V + v) / (int)q.gc;
                    s1[v] = grp[g] * inv, s2[v] = grp[cs + g] * inv;
                }
                store_dx<T, V, R>(a, t, ch, s1, s2, x, dy);
            }
        }
        __syncthreads();
    }
}

// Large samples: adds the chunks' A and B per channel, and S1 and S2 per group.  A block a group and sample.
__global__ __launch_bounds__(256) void norm_backward_totals_kernel(Args a) {
    __shared__ float sums[2][4];
    const Plan &q = a.q;
    for (int64_t ig = blockIdx.x; ig < q.n * q.groups; ig += gridDim.x) {
        const int64_t i = ig / q.groups, g = ig % q.groups;
        // lanes of a channel: as many as fit, each takes chunks in turn
        const int gc = q.gc < 256 ? (int)q.gc : 256, lanes = 256 / gc > 16 ? 16 : 256 / gc;
        __shared__ float2 row[256];
        float s1 = 0.0f, s2 = 0.0f;
        for (int64_t j0 = 0; j0 < q.gc; j0 += gc) {
            const int j = threadIdx.x % gc, lane = threadIdx.x / gc;
            const int64_t c = g * q.gc + j0 + j;
            float A = 0.0f, B = 0.0f;
            if (j0 + j < q.gc && lane < lanes)
                for (int64_t k = lane; k < q.chunks; k += lanes) {
                    const float2 v = a.part[(i * q.chunks + k) * q.c + c];
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
        for (int off = 32; off; off >>= 1) s1 += __shfl_xor(s1, off), s2 += __shfl_xor(s2, off);
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

template <typename T, int V, int R>
__global__ __launch_bounds__(512) void norm_backward_apply_kernel(Args a) {
    const Plan &q = a.q;
    for (int64_t tile = blockIdx.x; tile < q.tiles; tile += gridDim.x) {
        const Tile t(q, tile, V);
        Pack<T, V> x[R], dy[R];
        load_tile<T, V, R>(t, q, a.x, a.xs, a.xp, x);
        load_tile<T, V, R>(t, q, a.dy, a.ds, a.dp, dy);
        const Channel<V> ch(a, t);
        if (t.tx * V < t.nc) {
            float s1[V], s2[V];
#pragma unroll
            for (int v = 0; v < V; v++) {
                const float2 s = a.sums[t.i * q.groups + (t.c0 + t.tx * V + v) / q.gc];
                s1[v] = s.x, s2[v] = s.y;
            }
            store_dx<T, V, R>(a, t, ch, s1, s2, x, dy);
        }
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

// LDS of the reductions: `k` sums a channel, the channels' results and the groups'.
size_t reduction_bytes(const Plan &q, int k, int head) {
    const bool joined = q.tx < 64 && (q.tx & (q.tx - 1)) == 0;
    const size_t rows = joined ? q.threads / 64 : q.ty;
    return sizeof(float) * ((size_t)head * q.cs + rows * k * q.cs);
}

template <typename T, int V, int R>
int launch_forward(const Args &a, hipStream_t s) {
    const size_t lds = reduction_bytes(a.q, 1, 3);
    if (whole(a.q)) {
        norm_forward_kernel<T, V, R, true><<<grid_of(a.q.tiles), a.q.threads, lds, s>>>(a);
    } else if constexpr (R <= 8) {
        norm_forward_kernel<T, V, R, false><<<grid_of(a.q.tiles), a.q.threads, lds, s>>>(a);
        BYZ_HIP(hipGetLastError());
        norm_apply_kernel<T, V, R><<<grid_of(a.q.tiles), a.q.threads, 2 * a.q.cs * sizeof(float), s>>>(a);
    }
    BYZ_HIP(hipGetLastError());
    return BYZ_OK;
}

template <typename T, int V, int R>
int launch_backward(const Args &a, hipStream_t s) {
    const size_t lds = reduction_bytes(a.q, 2, 4);
    if constexpr (R <= 8) {
        if (whole(a.q)) {
            norm_backward_kernel<T, V, R, true><<<grid_of(a.q.tiles), a.q.threads, lds, s>>>(a);
        } else {
            norm_backward_kernel<T, V, R, false><<<grid_of(a.q.tiles), a.q.threads, lds, s>>>(a);
            BYZ_HIP(hipGetLastError());
            norm_backward_totals_kernel<<<grid_of(a.q.n * a.q.groups), 256, 0, s>>>(a);
            BYZ_HIP(hipGetLastError());
            norm_backward_apply_kernel<T, V, R><<<grid_of(a.q.tiles), a.q.threads, 0, s>>>(a);
        }
        BYZ_HIP(hipGetLastError());
    }
    if (a.dgamma) {
        norm_parameters_kernel<<<(unsigned)((a.q.c + 31) / 32), 1024, 0, s>>>(a.total, a.q.n, a.q.c, a.dgamma, a.dbeta);
        BYZ_HIP(hipGetLastError());
    }
    return BYZ_OK;
}

template <typename T, int V, bool FORWARD>
int launch_r(const Args &a, hipStream_t s) {
    switch (a.q.r) {
        case 1: return FORWARD ? launch_forward<T, V, 1>(a, s) : launch_backward<T, V, 1>(a, s);
        case 2: return FORWARD ? launch_forward<T, V, 2>(a, s) : launch_backward<T, V, 2>(a, s);
        case 4: return FORWARD ? launch_forward<T, V, 4>(a, s) : launch_backward<T, V, 4>(a, s);
        case 8: return FORWARD ? launch_forward<T, V, 8>(a, s) : launch_backward<T, V, 8>(a, s);
        default:
            if constexpr (FORWARD) return launch_forward<T, V, 16>(a, s);
            return BYZ_EINTERNAL;
    }
}

template <typename T, bool FORWARD>
int launch_vec(const Args &a, hipStream_t s) {
    constexpr int wide = 16 / sizeof(T), narrow = 4 / sizeof(T);
    if (a.q.vec == wide) return launch_r<T, wide, FORWARD>(a, s);
    if constexpr (narrow > 1)
        if (a.q.vec == narrow) return launch_r<T, narrow, FORWARD>(a, s);
    return launch_r<T, 1, FORWARD>(a, s);
}

template <bool FORWARD>
int launch(const Args &a, int dtype, hipStream_t s) {
    if (dtype == BYZ_F32) return launch_vec<float, FORWARD>(a, s);
    if (dtype == BYZ_BF16) return launch_vec<bf16, FORWARD>(a, s);
    return launch_vec<f16, FORWARD>(a, s);
}

constexpr int kForwardR = 16, kBackwardR = 8;

// Workspace of either direction, for any alignment: the plan with one element a vector has the most chunks or
// parts of those that a call can take.
size_t round_up(size_t bytes) { return (bytes + 255) / 256 * 256; }

bool sizes_ok(int64_t n, int64_t p, int64_t c, int groups, int dtype) {
    int64_t all;
    return n >= 0 && p >= 0 && c >= 1 && groups >= 1 && c % groups == 0 && dtype_known(dtype) && c <= (1 << 24) &&
           !__builtin_mul_overflow(n, p, &all) && !__builtin_mul_overflow(all, c, &all) && all <= (INT64_MAX >> 8);
}

template <typename F>
size_t most_bytes(int elem, int64_t c, F bytes) {
    size_t most = 0;
    for (int vec : {16 / elem, 4 / elem, 1}) {
        if (vec < 1 || c % vec) continue;
        const size_t b = bytes(vec);
        most = b > most ? b : most;
    }
    return most;
}

size_t forward_bytes(const Plan &q) {
    return whole(q) ? 0 : round_up(sizeof(float2) * q.n * q.groups * q.chunks * q.parts);
}

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
    const int elem = (int)dtype_size(dtype);
    return most_bytes(elem, c, [&](int vec) { return forward_bytes(make_plan(n, p, c, groups, elem, vec, kForwardR)); });
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
    const int vec = widest_vec(elem, c, {{x, x_sample, x_pixel}, {y, y_sample, y_pixel}});
    Args a{};
    a.q = make_plan(n, p, c, groups, elem, vec, kForwardR);
    if (forward_bytes(a.q) > workspace_bytes || (forward_bytes(a.q) && !workspace)) return BYZ_ENOMEM;
    a.x = x, a.xs = x_sample, a.xp = x_pixel;
    a.out = y, a.os = y_sample, a.op = y_pixel;
    a.gamma = gamma, a.beta = beta, a.mean = mean, a.rstd = rstd, a.eps = eps, a.act = act;
    a.part = (float2 *)workspace;
    return launch<true>(a, dtype, s);
}

extern "C" size_t byz_group_norm_backward_workspace_bytes(int64_t n, int64_t p, int64_t c, int groups, int dtype) {
    if (!sizes_ok(n, p, c, groups, dtype) || n == 0 || p == 0) return 0;
    const int elem = (int)dtype_size(dtype);
    return most_bytes(elem, c, [&](int vec) { return BackwardLayout(make_plan(n, p, c, groups, elem, vec, kBackwardR)).bytes; });
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
    const int vec = widest_vec(elem, c, {{dy, dy_sample, dy_pixel}, {x, x_sample, x_pixel}, {dx, dx_sample, dx_pixel}});
    a.q = make_plan(n, p, c, groups, elem, vec, kBackwardR);
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

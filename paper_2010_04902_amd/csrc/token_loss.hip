// Losses of tokens' log-probabilities, from logits (gfx950): the log-probabilities themselves, the clipped policy loss with its KL
// term, and the preference loss of pairs of sequences.
//
// All are functions of logp = (z_label - m) / T - log sum exp((z - m) / T), with m the row's largest logit, and all their gradients
// are w (onehot(label) - softmax(z / T)) with one weight w = (d loss / d logp) / T a row.  So there are three steps: a row's
// maximum and sum (one read), what the loss makes of logp (a few values a row, in fp64 from an fp32 sum), and the dense
// gradient (another read, and the write), which needs a row's m, log-sum, w and label and nothing else.
//
// Bound by memory.  The policy step holds rows of up to 256 KB in registers, so that they are read once; the preference step cannot: a
// row's weight depends on all rows of its pair, so its logits are read twice, the last rows first the second time.
//
// 8192 x 131072 bf16 policy step 772 to 826 us (4.3 GB at 5.2 to 5.6 TB/s, vector units busy 0.66); 750 x 32000 fp16 17.8 to 18.5.  6144 x 50021 bf16 preference
// step, a quarter of the rows prompts: sums 96, pairs 6, gradient 182 (5.9 TB/s).  7 x 50021 fp32 loss 7.3, one launch of 1024
// threads a row.
#include <algorithm>
#include <limits>
#include <type_traits>

#include "vocab_rows.h"

using namespace byz_worker;

namespace {

constexpr int64_t kMaxGrid = 1 << 20;

enum Kind { kLogp, kPolicy, kPreference };

// What the gradient needs of a row; w is 0 where there is no token.
struct Terms {
    float m, log_sum, w;
    int32_t label;
};

struct Args {
    const void *logits;
    int64_t rows, vocab, ld;
    const int32_t *label;
    float temperature;
    double per_temperature;  // its inverse: with divisions in fp64 by every thread for its row's weight a step of 8192 x 66000 bf16 took 522 us for 500
    Kind kind;
    // policy
    const float *old, *advantage, *ref;
    float low, high, kl;
    // preference
    const int32_t *bounds;
    int64_t pairs;
    float beta, smoothing;
    // results, each may be absent
    float *loss, *logp, *stats, *sums, *slope;
    // gradient
    const float *dloss, *given_stats, *given_slope;
    void *dlogits;
    int64_t dlogits_ld;
    // workspace
    Terms *terms;
    double *logp64;
    float2 *parts;
};

// log(s) of a sum in fp32, to 2^-24 or 2^-24 of itself; 0 for an empty row's sum
__device__ __forceinline__ double log_of(float s) {
    if (!(s > 0.0f && s < INFINITY)) return s == 0.0f ? 0.0 : (double)s;
    int e = __builtin_amdgcn_frexp_expf(s);
    float f = __builtin_amdgcn_frexp_mantf(s);
    if (f < 0.70710678f) f *= 2.0f, e--;
    return ((double)e + (double)__builtin_amdgcn_logf(f)) * 0.6931471805599453;
}

// exp(d) to some 2^-23 of itself: the whole powers of two exactly, the rest in fp32
__device__ __forceinline__ double exp_of(double d) {
    if (d != d) return d;
    const double y = fmin(fmax(d * 1.4426950408889634, -2000.0), 2000.0), k = rint(y);
    return ldexp((double)__builtin_amdgcn_exp2f((float)(y - k)), (int)k);
}

// exp(g) - 1, and less g: near 0 by the series of the latter.  At infinity, a token banned by the policy, both are infinite, and at
// minus infinity, one banned by the reference, -1 and infinite.
__device__ __forceinline__ void exp_less(double g, double &one, double &both) {
    if (!(fabs(g) < 0.5)) {
        one = exp_of(g) - 1.0, both = one == INFINITY ? one : one - g;
        return;
    }
    double s = 1.0 / 479001600;  // 1 / 12!, and down to 1 / 2!
    double f = 479001600;
#pragma unroll
    for (int n = 12; n > 2; n--) f /= n, s = s * g + 1.0 / f;
    both = s * g * g, one = both + g;
}

// The policy loss of a row and its derivative by logp.
__device__ __forceinline__ void policy(const Args &a, int64_t row, double logp, double &loss, double &slope) {
    const double advantage = a.advantage[row], r = exp_of(logp - (double)a.old[row]);
    const bool above = advantage >= 0.0 && r > (double)a.high, below = !(advantage >= 0.0) && r < (double)a.low;
    loss = -advantage * (above ? (double)a.high : below ? (double)a.low : r);
    slope = above || below ? 0.0 * advantage : -advantage * r;
    if (a.kl != 0.0f) {
        double one, both;
        exp_less((double)a.ref[row] - logp, one, both);
        loss += (double)a.kl * both;
        slope -= (double)a.kl * one;
    }
}

// A row's results from its maximum and sum, by one thread; z is the label's logit.
__device__ __forceinline__ Terms finish(const Args &a, int64_t row, int32_t label, float m, float sum, float z) {
    const bool empty = label < 0;
    if (empty || m == -INFINITY) m = 0.0f;  // no token, or nothing but banned logits (or NaN, which is in the sum)
    const double log_sum = empty ? 0.0 : log_of(sum);
    double logp = empty ? 0.0 : label >= a.vocab ? NAN : ((double)z - (double)m) * a.per_temperature - log_sum;
    Terms t{m, (float)log_sum, 0.0f, label};
    if (a.stats) a.stats[row * 2] = m, a.stats[row * 2 + 1] = (float)log_sum;
    if (a.logp) a.logp[row] = (float)logp;
    if (a.kind == kPolicy) {
        double loss = 0.0, slope = 0.0;
        if (!empty) policy(a, row, logp, loss, slope);
        if (a.loss) a.loss[row] = (float)loss;
        if (a.dloss && !empty) t.w = (float)((double)a.dloss[row] * slope * a.per_temperature);
    }
    if (a.kind == kPreference) a.logp64[row] = logp;
    if (a.terms) a.terms[row] = t;
    return t;
}

// A row's maximum and sum, a block a row.
template <typename T, int NT>
__global__ __launch_bounds__(NT) void rows_kernel(Args a) {
    constexpr int V = 16 / sizeof(T);
    __shared__ double red[32];
    const int tid = threadIdx.x;
    const float c = (float)(1.4426950408889634 / (double)a.temperature);
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const int32_t label = a.label[row];
        RunningSum s;
        float z = 0.0f;
        if (label >= 0) {
            const Row<T> r(a.logits, row, a.ld, a.vocab);
            if (label < a.vocab) z = (float)r.at[label];
            if (tid < r.tail) {
                const float x[1] = {(float)r.at[r.edge(tid)]};
                s.add(x, c);
            }
            auto add_up = [&](auto odd) {
                constexpr int kUnroll = odd.value ? 3 : 4;
                int64_t i = tid;
                for (; i + (kUnroll - 1) * NT < r.vectors; i += kUnroll * NT) {
                    Words<T, V> v[kUnroll];
#pragma unroll
                    for (int u = 0; u < kUnroll; u++) v[u] = r.template vector_of<odd.value>(i + u * NT);
#pragma unroll
                    for (int u = 0; u < kUnroll; u++) {
                        float x[V];
#pragma unroll
                        for (int e = 0; e < V; e++) x[e] = v[u][e];
                        s.add(x, c);
                    }
                }
                for (; i < r.vectors; i += NT) {
                    const Words<T, V> v = r.template vector_of<odd.value>(i);
                    float x[V];
#pragma unroll
                    for (int e = 0; e < V; e++) x[e] = v[e];
                    s.add(x, c);
                }
            };
            if (r.odd())
                add_up(std::true_type{});
            else
                add_up(std::false_type{});
            s = row_join<NT>(s, c, red);
        }
        if (tid == 0) finish(a, row, label, s.m, s.s, z);
    }
}

// Few long rows: `parts` blocks a row, whose maxima and sums join_kernel joins.
template <typename T>
__global__ __launch_bounds__(256) void parts_kernel(Args a, int64_t each) {
    constexpr int V = 16 / sizeof(T);
    __shared__ double red[8];
    const float c = (float)(1.4426950408889634 / (double)a.temperature);
    const int64_t row = blockIdx.y, part = blockIdx.x;
    if (a.label[row] < 0) return;
    const Row<T> r(a.logits, row, a.ld, a.vocab);
    RunningSum s;
    if (part == gridDim.x - 1 && (int)threadIdx.x < r.tail) {
        const float x[1] = {(float)r.at[r.edge(threadIdx.x)]};
        s.add(x, c);
    }
    const int64_t to = std::min(r.vectors, (part + 1) * each);
#pragma unroll 4
    for (int64_t i = part * each + threadIdx.x; i < to; i += 256) {
        const Words<T, V> v = r.vector(i);
        float x[V];
#pragma unroll
        for (int e = 0; e < V; e++) x[e] = v[e];
        s.add(x, c);
    }
    s = row_join<256>(s, c, red);
    if (threadIdx.x == 0) a.parts[row * gridDim.x + part] = make_float2(s.m, s.s);
}

template <typename T>
__global__ __launch_bounds__(64) void join_kernel(Args a, int parts) {
    const float c = (float)(1.4426950408889634 / (double)a.temperature);
    const int64_t row = blockIdx.x;
    const int32_t label = a.label[row];
    RunningSum s;
    float z = 0.0f;
    if (label >= 0) {
        if (label < a.vocab) z = (float)((const T *)a.logits)[row * a.ld + label];
        if ((int)threadIdx.x < parts) {
            const float2 p = a.parts[row * parts + threadIdx.x];
            s.m = p.x, s.s = p.y;
        }
        s = wave_join(s, c);
    }
    if (threadIdx.x == 0) finish(a, row, label, s.m, s.s, z);
}

// What a gradient's own call needs of its rows.
template <typename T>
__global__ __launch_bounds__(256) void terms_kernel(Args a) {
    const int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (row >= a.rows) return;
    const int32_t label = a.label[row];
    Terms t{a.given_stats[row * 2], a.given_stats[row * 2 + 1], 0.0f, label};
    if (label >= a.vocab) {
        t.w = NAN;
    } else if (label >= 0) {
        double slope = 0.0;
        if (a.kind == kLogp) {
            slope = a.dloss[row];
        } else if (a.kind == kPolicy) {
            const double z = (float)((const T *)a.logits)[row * a.ld + label];
            double loss;
            policy(a, row, (z - (double)t.m) * a.per_temperature - (double)t.log_sum, loss, slope);
            slope *= (double)a.dloss[row];
        } else {
            // the last sequence that starts at this row or before; the search ends whatever the bounds are
            int64_t low = 0, high = 2 * a.pairs;
            while (low < high) {
                const int64_t mid = (low + high + 1) / 2;
                if (a.bounds[mid] <= row)
                    low = mid;
                else
                    high = mid - 1;
            }
            if (low < 2 * a.pairs && a.bounds[low] <= row)
                slope = (low % 2 ? -1.0 : 1.0) * (double)a.beta * (double)a.given_slope[low / 2] * (double)a.dloss[low / 2];
        }
        t.w = (float)(slope * a.per_temperature);
    }
    a.terms[row] = t;
}

// A pair's loss, and the weights of its rows.
__global__ __launch_bounds__(256) void pairs_kernel(Args a) {
    __shared__ double red[4];
    for (int64_t pair = blockIdx.x; pair < a.pairs; pair += gridDim.x) {
        const int32_t b0 = a.bounds[2 * pair], b1 = a.bounds[2 * pair + 1], b2 = a.bounds[2 * pair + 2];
        const bool good = 0 <= b0 && b0 <= b1 && b1 <= b2 && b2 <= a.rows;
        auto sum = [&](int64_t from, int64_t to) {
            double s = 0.0;
            for (int64_t i = from + threadIdx.x; i < to; i += 256) s += a.logp64[i];
            return row_sum<256>(s, red);
        };
        const double chosen = good ? sum(b0, b1) : NAN, rejected = good ? sum(b1, b2) : NAN;
        const double ref = a.ref ? (double)a.ref[2 * pair] - (double)a.ref[2 * pair + 1] : 0.0;
        const double margin = (double)a.beta * ((chosen - rejected) - ref);
        const double low = a.smoothing, slope = low - 1.0 / (1.0 + exp(margin));
        if (threadIdx.x == 0) {
            const double small = log1p(exp(-fabs(margin)));
            double loss = margin != margin ? NAN : 0.0;
            if (low != 1.0) loss += (1.0 - low) * (small + fmax(-margin, 0.0));
            if (low != 0.0) loss += low * (small + fmax(margin, 0.0));
            a.loss[pair] = (float)loss;
            if (a.sums) a.sums[2 * pair] = (float)chosen, a.sums[2 * pair + 1] = (float)rejected;
            if (a.slope) a.slope[pair] = (float)slope;
        }
        if (a.dloss && good) {
            const double w = (double)a.beta * slope * (double)a.dloss[pair] * a.per_temperature;
            for (int64_t i = b0 + (int64_t)threadIdx.x; i < b2; i += 256)
                if (a.terms[i].label >= 0) a.terms[i].w = (float)(i < b1 ? w : -w);
        }
    }
}

// The dense gradient: `parts` blocks a row, or a wave each of short rows.  Rows without a token or weight are not read.  The last rows
// come first: they were read for their sums last, the caches still have some of them, and the results go past these.  us, so /
// with results in the caches and the first rows first: preference step on 8192 x 20000 bf16 171 / 195, on 1000 x 200000 192 / 236.
template <typename T, int NT>
__global__ __launch_bounds__(256) void gradient_kernel(Args a, int64_t parts, int64_t each) {
    constexpr int V = 16 / sizeof(T), SLOTS = 256 / NT;
    const int64_t total = a.rows * parts;
    const int slot = SLOTS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / NT) : 0, tid = threadIdx.x % NT;
    for (int64_t unit = (int64_t)blockIdx.x * SLOTS + slot; unit < total; unit += (int64_t)gridDim.x * SLOTS) {
        const int64_t row = a.rows - 1 - unit / parts, part = unit % parts;
        const Terms t = a.terms[row];
        const Row<T> r(a.logits, row, a.ld, a.vocab);
        T *out = (T *)a.dlogits + row * a.dlogits_ld;
        const int64_t from = part * each, to = std::min(r.vectors, from + each);
        const bool last = part == parts - 1 && tid < r.tail;
        const int64_t edge = r.edge(tid);
        if (t.w == 0.0f) {
            for (int64_t i = from + tid; i < to; i += NT) put_words(out + i * V, Words<T, V>::of([](int) { return 0.0f; }));
            if (last) out[edge] = (T)0.0f;
            continue;
        }
        const Softmax<T> q((double)t.m, (double)t.log_sum, (double)a.temperature, -t.w);
        auto write = [&](auto odd) {
            for (int64_t i = from + tid; i < to; i += NT) {
                const Words<T, V> v = r.template vector_of<odd.value>(i);
                const Words<T, V> d = Words<T, V>::of([&](int e) { return q.weighted(v[e]); });
                put_past_caches(out + i * V, d);
                const int64_t at = t.label - i * V;
                if (at >= 0 && at < V) {
                    float x = 0.0f;
#pragma unroll
                    for (int e = 0; e < V; e++) x = at == e ? v[e] : x;
                    out[t.label] = round_to<T>(q.less(x, 1.0f));
                }
            }
        };
        if (r.odd())
            write(std::true_type{});
        else
            write(std::false_type{});
        if (last) {
            const float x = (float)r.at[edge];
            out[edge] = round_to<T>(edge == t.label ? q.less(x, 1.0f) : q.weighted(x));
        }
    }
}

// The largest of G vectors in registers from the `from`-th on, from their bits, so that those of 16 bits need not be unpacked: as signed
// integers the floats from 0 on are in order and above all negative ones, and where there are only these, they are in reverse order as
// unsigned ones.  With a NaN among them it may be any of them, or NaN.
template <int G, typename T, int V, int R>
__device__ __forceinline__ float largest_of(const Words<T, V> (&x)[R], int from) {
    typedef std::conditional_t<sizeof(T) == 2, int16_t, int32_t> Int;
    typedef std::conditional_t<sizeof(T) == 2, uint16_t, uint32_t> Uint;
    constexpr int N = 4 / sizeof(T);
    typedef Int Ints __attribute__((ext_vector_type(N)));
    typedef Uint Uints __attribute__((ext_vector_type(N)));
    auto over = [&](auto join) __attribute__((always_inline)) {
#pragma unroll
        for (int v = from; v < from + G; v++)
#pragma unroll
            for (int i = 0; i < x[v].N; i++) join((uint32_t)x[v].w[i]);
    };
    Ints most = std::numeric_limits<Int>::min();
    over([&](uint32_t w) { most = __builtin_elementwise_max(most, __builtin_bit_cast(Ints, w)); });
    Int a = most[0];
    if constexpr (N == 2) a = std::max(a, most[1]);
    if (__builtin_expect(a < 0, false)) {
        Uints least = std::numeric_limits<Uint>::max();
        over([&](uint32_t w) { least = __builtin_elementwise_min(least, __builtin_bit_cast(Uints, w)); });
        Uint b = least[0];
        if constexpr (N == 2) b = std::min(b, least[1]);
        a = (Int)b;
    }
    return (float)__builtin_bit_cast(T, a);
}

// -inf in all places of a vector
template <typename T, int V>
__device__ __forceinline__ Words<T, V> banned() {
    return Words<T, V>::of([](int) { return -INFINITY; });
}

// A row in the registers of NT threads, R vectors of 16 bytes each, so that it is read once: its maximum and sum, and with STEP the
// gradient of the policy loss.  A block of 1024 threads has a compute unit for itself: as soon as a thread has stored a piece
// of its gradient it loads that piece of its next row, so reads, exponentials and writes overlap, and what the losses are
// made of is left to losses_kernel.  Smaller blocks share a compute unit, and overlap one another; short rows are a wave's, four to
// a block.  ODD: rows of 16-bit values may start at odd multiples of two bytes.
template <typename T, int NT, int R, bool STEP, bool ODD>
__global__ __launch_bounds__(NT == 64 ? 256 : NT, 4) void held_rows_kernel(Args a) {
    constexpr int V = 16 / sizeof(T), SLOTS = NT == 64 ? 4 : 1, G = R > 4 ? 4 : 2;
    constexpr bool kAlone = NT == 1024;
    static_assert(STEP || !kAlone, "");
    __shared__ double red[32];
    const int tid = threadIdx.x % NT;
    const float c = (float)(1.4426950408889634 / (double)a.temperature);
    Words<T, V> x[R];
    word_t next_word[ODD ? R : 1];
    T edge = (T)0.0f;
    // A row here is shorter than 2^31 bytes.  A thread's number is made afresh for each use, or the places of all R vectors would be
    // kept in registers; threads without a v-th vector load the last, without a branch, and leave it.
    auto vector_at = [](auto *base, int number) { return base + (uint32_t)number * (uint32_t)V; };
    // Of an odd row x has the words that hold the values but for the last value's; shifted where the row is begun.
    auto load = [&](const Row<T> &r, int own, int v) __attribute__((always_inline)) {
        const T *from = vector_at(r.at - (ODD && r.odd() ? 1 : 0), std::max(0, std::min(own + v * NT, (int)r.vectors - 1)));
        x[v] = get_words<T, V>(from);
        if constexpr (ODD)
            if (r.odd()) next_word[v] = *(const word_t *)(from + V);
    };
    auto load_row = [&](int64_t row) __attribute__((always_inline)) {
        if (row >= a.rows || a.label[row] < 0) return;
        const Row<T> r(a.logits, row, a.ld, a.vocab);
        const int own = afresh(tid);
        if (NT > 64 || r.vectors > 0) {  // there are none in a row shorter than one
#pragma unroll
            for (int v = 0; v < R; v++) load(r, own, v);
        }
        if (tid < r.tail) edge = r.at[r.edge(tid)];
    };
    if constexpr (kAlone) load_row(blockIdx.x);
    const int slot = SLOTS > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / NT) : 0;
    for (int64_t row = (int64_t)blockIdx.x * SLOTS + slot; row < a.rows; row += (int64_t)gridDim.x * SLOTS) {
        const int32_t label = a.label[row];
        if constexpr (!kAlone) load_row(row);
        const Row<T> r(a.logits, row, a.ld, a.vocab);
        const int vectors = (int)r.vectors;
        const bool has_edge = tid < r.tail;
        float z = 0.0f, w = 0.0f;
        RunningSum s;
        if (label >= 0) {
            if (label < a.vocab) z = (float)r.at[label];
            if constexpr (ODD)
                if (r.odd())
#pragma unroll
                    for (int v = 0; v < R; v++) x[v] = shifted(x[v], next_word[v]);
            // A thread's sum of exp2((x - m) c), G vectors at a time, so that exponentials overlap with the loads behind them and of short
            // rows some are left out.  Its m is the largest value: with one far below that the exponents' rounding would be in the
            // sum.  us of a step of 8192 x 66000 bf16 with all vectors at once 517, so 487.
            s.m = std::numeric_limits<float>::lowest();
            auto raise_to = [&](float top) __attribute__((always_inline)) {
                top = fmaxf(s.m, top);
                s.s *= __builtin_amdgcn_exp2f((s.m - top) * c), s.m = top;
            };
            const int own = afresh(tid);
#pragma unroll
            for (int from = 0; from < R; from += G) {
                if (from > 0 && from * NT >= vectors) break;
                if (__builtin_expect((from + G) * NT > vectors, false)) {  // not for all threads
#pragma unroll
                    for (int v = from; v < from + G; v++)
                        if ((v + 1) * NT > vectors && own + v * NT >= vectors) x[v] = banned<T, V>();
                }
                raise_to(largest_of<G>(x, from));
#pragma unroll
                for (int v = from; v < from + G; v++) {
                    float sum = __builtin_amdgcn_exp2f(less<T, true>(x[v][0], s.m) * c);
#pragma unroll
                    for (int e = 1; e < V; e++) sum += __builtin_amdgcn_exp2f(less<T, true>(x[v][e], s.m) * c);
                    s.s += sum;
                    x[v].keep();
                    __builtin_amdgcn_sched_barrier(0);  // one vector's values in registers at a time
                }
            }
            if (has_edge) {
                raise_to((float)edge);
                s.s += __builtin_amdgcn_exp2f(((float)edge - s.m) * c);
            }
            if (s.s == 0.0f) s.m = -INFINITY;  // nothing, or nothing but -inf
            s = row_join<NT>(s, c, red);
        }
        if constexpr (kAlone) {
            if (tid == 0) a.terms[row] = Terms{s.m, s.s, z, label};
            if (label >= 0) {
                if (s.m == -INFINITY) s.m = 0.0f;
                double loss, slope;  // in the same steps as losses_kernel, so that loss and gradient are clipped alike
                policy(a, row, ((double)z - (double)s.m) * a.per_temperature - log_of(s.s), loss, slope);
                w = label >= a.vocab ? NAN : (float)((double)a.dloss[row] * slope * a.per_temperature);
            }
        } else if constexpr (NT == 64) {
            if (tid == 0) w = finish(a, row, label, s.m, s.s, z).w;
            w = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, w)));
            if (s.m == -INFINITY) s.m = 0.0f;
        } else {
            __syncthreads();
            Terms *const shared = reinterpret_cast<Terms *>(red + 16);
            if (tid == 0) *shared = finish(a, row, label, s.m, s.s, z);
            __syncthreads();
            w = shared->w;
            if (s.m == -INFINITY) s.m = 0.0f;
        }
        if constexpr (!STEP) continue;
        T *out = (T *)a.dlogits + row * a.dlogits_ld;
        const Softmax<T, true> q(s.m, s.s == 0.0f ? 1.0f : s.s, a.temperature, -w, c);
        const int64_t ahead = row + gridDim.x;
        const bool more = kAlone && ahead < a.rows && a.label[ahead] >= 0;
        const Row<T> next(a.logits, more ? ahead : row, a.ld, a.vocab);
        if (has_edge) {
            const int64_t at = r.edge(tid);
            out[at] = w == 0.0f ? (T)0.0f : round_to<T>(at == label ? q.less((float)edge, 1.0f) : q.weighted((float)edge));
            if (more) edge = next.at[next.edge(tid)];
        }
        const int then = afresh(tid);
        auto put_result = [](T *to, const Words<T, V> &v) {
            if constexpr (NT == 64)
                put_words(to, v);
            else
                put_past_caches(to, v);
        };
        const int own_label = (uint32_t)(label / V) % NT == (uint32_t)tid ? label / V / NT : -1;  // which of the thread's vectors has it
        auto pass = [&](auto some, auto loads) __attribute__((always_inline)) {
#pragma unroll
            for (int v = 0; v < R; v++) {
                if (then + v * NT < vectors) {
                    T *const to = vector_at(out, then + v * NT);
                    put_result(to, Words<T, V>::of([&](int e) { return some.value ? q.weighted(x[v][e]) : 0.0f; }));
                    if (some.value && v == own_label) to[label % V] = round_to<T>(q.less(z, 1.0f));
                }
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (loads.value) {
                    load(next, then, v);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        };
        if (more) {
            if (w == 0.0f)
                pass(std::false_type{}, std::true_type{});
            else
                pass(std::true_type{}, std::true_type{});
        } else if (w == 0.0f) {
            pass(std::false_type{}, std::false_type{});
        } else {
            pass(std::true_type{}, std::false_type{});
        }
    }
}

// The losses of rows whose maxima and sums held_rows_kernel has left.
__global__ __launch_bounds__(256) void losses_kernel(Args a) {
    const int64_t row = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (row >= a.rows) return;
    const Terms t = a.terms[row];
    Args only = a;
    only.dloss = nullptr, only.terms = nullptr;
    finish(only, row, t.label, t.m, t.log_sum, t.w);
}

// ------------------------------------------------------------------ launches

constexpr int kCus = 256;  // compute units

template <typename T>
int64_t vectors_of(int64_t vocab) {
    return vocab * (int64_t)sizeof(T) / 16;
}

// Whether rows of 16-bit values may start at odd multiples of two bytes.
template <typename T>
bool may_be_odd(const Args &a) {
    return sizeof(T) == 2 && (((uintptr_t)a.logits & 2) || (a.ld & 1));
}

template <typename T, int NT, int R, bool STEP>
int launch_held(const Args &a, hipStream_t s) {
    constexpr int slots = NT == 64 ? 4 : 1;
    const unsigned grid = (unsigned)std::min((a.rows + slots - 1) / slots, NT == 1024 ? (int64_t)kCus : kMaxGrid);
    if (may_be_odd<T>(a)) {
        if constexpr (sizeof(T) == 2) held_rows_kernel<T, NT, R, STEP, true><<<grid, NT * slots, 0, s>>>(a);
    } else {
        held_rows_kernel<T, NT, R, STEP, false><<<grid, NT * slots, 0, s>>>(a);
    }
    BYZ_HIP(hipGetLastError());
    return BYZ_OK;
}

// The policy loss' step of rows that registers hold; of more than 128 KB where there is one for every other compute unit at least.
// Blocks of 1024 threads were slower up to there: 8192 x 50000 bf16 370 us for 331 in blocks of 512.
template <typename T>
bool step_is_held(const Args &a) {
    return vectors_of<T>(a.vocab) <= 512 * 16 || (vectors_of<T>(a.vocab) <= 1024 * 16 && a.rows >= kCus / 2);
}

template <typename T>
int launch_step(const Args &a, hipStream_t s) {
    const int64_t vectors = vectors_of<T>(a.vocab);
    if (vectors <= 64 * 4) return launch_held<T, 64, 4, true>(a, s);
    if (vectors <= 64 * 16) return launch_held<T, 64, 16, true>(a, s);
    if (vectors <= 256 * 8) return launch_held<T, 256, 8, true>(a, s);
    if (vectors <= 256 * 16) return launch_held<T, 256, 16, true>(a, s);
    if (vectors <= 512 * 16) return launch_held<T, 512, 16, true>(a, s);
    const int rc = launch_held<T, 1024, 16, true>(a, s);
    if (rc != BYZ_OK) return rc;
    losses_kernel<<<(unsigned)((a.rows + 255) / 256), 256, 0, s>>>(a);
    BYZ_HIP(hipGetLastError());
    return BYZ_OK;
}

// Blocks of a row: of few rows of 256 KB and more, so many that there are some for every compute unit, each with 16 KB at least.
int64_t row_parts(int64_t rows, int64_t vectors) {
    if (rows >= kCus / 2 || vectors < 16384) return 1;
    return std::min<int64_t>({64, vectors / 1024, (2 * kCus + rows - 1) / rows});
}

size_t terms_bytes(int64_t rows) { return (size_t)rows * sizeof(Terms); }
size_t workspace_of(int64_t rows, int64_t vocab, int dtype) {
    const int64_t parts = row_parts(rows, vocab * (int64_t)dtype_size(dtype) / 16);
    return terms_bytes(rows) + (size_t)rows * sizeof(double) + (parts > 1 ? (size_t)(rows * parts) * sizeof(float2) : 0);
}

template <typename T>
int launch_rows(const Args &a, hipStream_t s) {
    const int64_t vectors = vectors_of<T>(a.vocab), parts = row_parts(a.rows, vectors);
    if (vectors <= 64 * 4) return launch_held<T, 64, 4, false>(a, s);
    if (vectors <= 64 * 16) return launch_held<T, 64, 16, false>(a, s);
    if (parts > 1) {
        parts_kernel<T><<<dim3((unsigned)parts, (unsigned)a.rows), 256, 0, s>>>(a, (vectors + parts - 1) / parts);
        BYZ_HIP(hipGetLastError());
        join_kernel<T><<<(unsigned)a.rows, 64, 0, s>>>(a, (int)parts);
        BYZ_HIP(hipGetLastError());
        return BYZ_OK;
    }
    if (a.rows < kCus / 2)
        rows_kernel<T, 1024><<<(unsigned)a.rows, 1024, 0, s>>>(a);
    else
        rows_kernel<T, 256><<<(unsigned)std::min(a.rows, kMaxGrid), 256, 0, s>>>(a);
    BYZ_HIP(hipGetLastError());
    return BYZ_OK;
}

template <typename T>
int launch_gradient(const Args &a, hipStream_t s) {
    const int64_t vectors = vectors_of<T>(a.vocab), each = 1024;
    if (vectors <= 256) {
        gradient_kernel<T, 64><<<(unsigned)std::min((a.rows + 3) / 4, kMaxGrid), 256, 0, s>>>(a, 1, vectors);
    } else {
        const int64_t parts = (vectors + each - 1) / each;
        gradient_kernel<T, 256><<<(unsigned)std::min(a.rows * parts, kMaxGrid), 256, 0, s>>>(a, parts, each);
    }
    BYZ_HIP(hipGetLastError());
    return BYZ_OK;
}

template <typename T>
int launch_terms(const Args &a, hipStream_t s) {
    terms_kernel<T><<<(unsigned)((a.rows + 255) / 256), 256, 0, s>>>(a);
    BYZ_HIP(hipGetLastError());
    return BYZ_OK;
}

int launch_pairs(const Args &a, hipStream_t s) {
    if (a.pairs == 0) return BYZ_OK;
    pairs_kernel<<<(unsigned)std::min(a.pairs, kMaxGrid), 256, 0, s>>>(a);
    BYZ_HIP(hipGetLastError());
    return BYZ_OK;
}

// Rows, then pairs where there are any, then the gradient where it is wanted.
template <typename T>
int launch_all(const Args &a, hipStream_t s) {
    int rc = BYZ_OK;
    if (a.rows && a.kind == kPolicy && a.dlogits && !a.given_stats && step_is_held<T>(a)) return launch_step<T>(a, s);
    if (a.rows) rc = a.given_stats ? launch_terms<T>(a, s) : launch_rows<T>(a, s);
    if (rc == BYZ_OK && a.kind == kPreference && !a.given_stats) rc = launch_pairs(a, s);
    if (rc == BYZ_OK && a.rows && a.dlogits) rc = launch_gradient<T>(a, s);
    return rc;
}

int launch(const Args &a, int dtype, void *stream) {
    const hipStream_t s = (hipStream_t)stream;
    return dtype == BYZ_F32 ? launch_all<float>(a, s) : dtype == BYZ_BF16 ? launch_all<bf16>(a, s) : launch_all<f16>(a, s);
}

bool sizes_ok(int64_t rows, int64_t vocab, int dtype) {
    return rows >= 0 && rows <= ((int64_t)1 << 38) && vocab >= 1 && vocab <= INT32_MAX && dtype_known(dtype);
}
bool real(float v) { return v > -INFINITY && v < INFINITY; }
bool floats_ok(const float *p) { return aligned(p, 4); }

Args args_of(const void *logits, int64_t rows, int64_t vocab, int64_t ld, const int32_t *label, float temperature, Kind kind) {
    Args a{};
    a.logits = logits, a.rows = rows, a.vocab = vocab, a.ld = ld, a.label = label, a.temperature = temperature, a.kind = kind;
    a.per_temperature = 1.0 / (double)temperature;
    return a;
}

// The checks that all calls share, and the workspace's parts.
int check(Args &a, int dtype, bool gradient, void *workspace, size_t bytes) {
    // colder by some 2^-24, log2(e) / T in two parts times a banned logit's difference passes fp32's range
    if (!sizes_ok(a.rows, a.vocab, dtype) || !(a.temperature >= 0x1p-64f) || !real(a.temperature)) return BYZ_EINVAL;
    if (a.rows == 0) return BYZ_OK;
    if (!a.logits || !a.label || !aligned(a.logits, dtype_size(dtype)) || !aligned(a.label, 4) || a.ld < a.vocab ||
        !extent_ok(a.rows, a.ld, a.vocab) || !floats_ok(a.stats) || !floats_ok(a.given_stats))
        return BYZ_EINVAL;
    if (gradient && (!a.dlogits || !a.dloss || !floats_ok(a.dloss) || !aligned(a.dlogits, dtype_size(dtype)) || a.dlogits_ld < a.vocab ||
                     !extent_ok(a.rows, a.dlogits_ld, a.vocab)))
        return BYZ_EINVAL;
    if (!workspace || !aligned(workspace, 16) || bytes < workspace_of(a.rows, a.vocab, dtype)) return BYZ_ENOMEM;
    a.terms = (Terms *)workspace;
    a.logp64 = (double *)((char *)workspace + terms_bytes(a.rows));
    a.parts = (float2 *)(a.logp64 + a.rows);
    return BYZ_OK;
}

bool policy_ok(const Args &a, float clip_low, float clip_high) {
    return clip_low >= 0.0f && clip_low <= 1.0f && clip_high >= 0.0f && real(clip_high) && a.kl >= 0.0f && real(a.kl) &&
           (a.rows == 0 || (a.old && a.advantage && (a.ref || a.kl == 0.0f) && floats_ok(a.old) && floats_ok(a.advantage) && floats_ok(a.ref)));
}
void set_policy(Args &a, const float *old, const float *advantage, const float *ref, float clip_low, float clip_high, float kl) {
    a.old = old, a.advantage = advantage, a.ref = ref, a.kl = kl;
    a.low = 1.0f - clip_low, a.high = 1.0f + clip_high;
}
bool preference_ok(const Args &a) {
    return a.pairs >= 0 && a.pairs <= (1 << 29) && real(a.beta) && a.smoothing >= 0.0f && a.smoothing <= 1.0f && floats_ok(a.ref) &&
           floats_ok(a.sums) && floats_ok(a.slope) && (a.pairs == 0 || (a.bounds && aligned(a.bounds, 4)));
}
void set_preference(Args &a, const int32_t *bounds, int64_t pairs, const float *ref, float beta, float smoothing) {
    a.bounds = bounds, a.pairs = pairs, a.ref = ref, a.beta = beta, a.smoothing = smoothing;
}

}  // namespace

extern "C" size_t byz_token_loss_workspace_bytes(int64_t rows, int64_t vocab, int dtype) {
    return sizes_ok(rows, vocab, dtype) ? workspace_of(rows, vocab, dtype) : 0;
}

extern "C" int byz_token_logp(const void *logits, int64_t rows, int64_t vocab, int64_t ld, int dtype, const int32_t *label,
                              float temperature, float *logp, float *stats, void *workspace, size_t workspace_bytes, void *stream) {
    Args a = args_of(logits, rows, vocab, ld, label, temperature, kLogp);
    a.logp = logp, a.stats = stats;
    const int rc = check(a, dtype, false, workspace, workspace_bytes);
    if (rc != BYZ_OK || rows == 0) return rc;
    if (!logp || !floats_ok(logp)) return BYZ_EINVAL;
    return launch(a, dtype, stream);
}

extern "C" int byz_token_logp_backward(const float *dlogp, const void *logits, int64_t rows, int64_t vocab, int64_t ld, int dtype,
                                       const int32_t *label, const float *stats, float temperature, void *dlogits,
                                       int64_t dlogits_ld, void *workspace, size_t workspace_bytes, void *stream) {
    Args a = args_of(logits, rows, vocab, ld, label, temperature, kLogp);
    a.dloss = dlogp, a.given_stats = stats, a.dlogits = dlogits, a.dlogits_ld = dlogits_ld;
    const int rc = check(a, dtype, true, workspace, workspace_bytes);
    if (rc != BYZ_OK || rows == 0) return rc;
    if (!stats) return BYZ_EINVAL;
    return launch(a, dtype, stream);
}

extern "C" int byz_policy_loss(const void *logits, int64_t rows, int64_t vocab, int64_t ld, int dtype, const int32_t *label,
                               const float *old, const float *advantage, const float *ref, float clip_low, float clip_high, float kl,
                               float temperature, float *loss, float *logp, float *stats, void *workspace, size_t workspace_bytes,
                               void *stream) {
    Args a = args_of(logits, rows, vocab, ld, label, temperature, kPolicy);
    set_policy(a, old, advantage, ref, clip_low, clip_high, kl);
    a.loss = loss, a.logp = logp, a.stats = stats;
    const int rc = check(a, dtype, false, workspace, workspace_bytes);
    if (rc == BYZ_EINVAL || !policy_ok(a, clip_low, clip_high)) return BYZ_EINVAL;
    if (rc != BYZ_OK || rows == 0) return rc;
    if (!loss || !floats_ok(loss) || !floats_ok(logp)) return BYZ_EINVAL;
    return launch(a, dtype, stream);
}

extern "C" int byz_policy_loss_backward(const float *dloss, const void *logits, int64_t rows, int64_t vocab, int64_t ld, int dtype,
                                        const int32_t *label, const float *old, const float *advantage, const float *ref,
                                        float clip_low, float clip_high, float kl, float temperature, const float *stats,
                                        void *dlogits, int64_t dlogits_ld, void *workspace, size_t workspace_bytes, void *stream) {
    Args a = args_of(logits, rows, vocab, ld, label, temperature, kPolicy);
    set_policy(a, old, advantage, ref, clip_low, clip_high, kl);
    a.dloss = dloss, a.given_stats = stats, a.dlogits = dlogits, a.dlogits_ld = dlogits_ld;
    const int rc = check(a, dtype, true, workspace, workspace_bytes);
    if (rc == BYZ_EINVAL || !policy_ok(a, clip_low, clip_high)) return BYZ_EINVAL;
    if (rc != BYZ_OK || rows == 0) return rc;
    if (!stats) return BYZ_EINVAL;
    return launch(a, dtype, stream);
}

extern "C" int byz_policy_loss_step(const float *dloss, const void *logits, int64_t rows, int64_t vocab, int64_t ld, int dtype,
                                    const int32_t *label, const float *old, const float *advantage, const float *ref, float clip_low,
                                    float clip_high, float kl, float temperature, float *loss, float *logp, void *dlogits,
                                    int64_t dlogits_ld, void *workspace, size_t workspace_bytes, void *stream) {
    Args a = args_of(logits, rows, vocab, ld, label, temperature, kPolicy);
    set_policy(a, old, advantage, ref, clip_low, clip_high, kl);
    a.dloss = dloss, a.loss = loss, a.logp = logp, a.dlogits = dlogits, a.dlogits_ld = dlogits_ld;
    const int rc = check(a, dtype, true, workspace, workspace_bytes);
    if (rc == BYZ_EINVAL || !policy_ok(a, clip_low, clip_high)) return BYZ_EINVAL;
    if (rc != BYZ_OK || rows == 0) return rc;
    if (!loss || !floats_ok(loss) || !floats_ok(logp)) return BYZ_EINVAL;
    return launch(a, dtype, stream);
}

extern "C" int byz_preference_loss(const void *logits, int64_t rows, int64_t vocab, int64_t ld, int dtype, const int32_t *label,
                                   const int32_t *bounds, int64_t pairs, const float *ref, float beta, float smoothing,
                                   float temperature, float *loss, float *sums, float *slope, float *stats, void *workspace,
                                   size_t workspace_bytes, void *stream) {
    Args a = args_of(logits, rows, vocab, ld, label, temperature, kPreference);
    set_preference(a, bounds, pairs, ref, beta, smoothing);
    a.loss = loss, a.sums = sums, a.slope = slope, a.stats = stats;
    const int rc = check(a, dtype, false, workspace, workspace_bytes);
    if (rc == BYZ_EINVAL || !preference_ok(a) || (pairs > 0 && (!loss || !floats_ok(loss)))) return BYZ_EINVAL;
    if (rc != BYZ_OK) return rc;
    return launch(a, dtype, stream);
}

extern "C" int byz_preference_loss_backward(const float *dloss, const void *logits, int64_t rows, int64_t vocab, int64_t ld, int dtype,
                                            const int32_t *label, const int32_t *bounds, int64_t pairs, const float *slope, float beta,
                                            float temperature, const float *stats, void *dlogits, int64_t dlogits_ld, void *workspace,
                                            size_t workspace_bytes, void *stream) {
    Args a = args_of(logits, rows, vocab, ld, label, temperature, kPreference);
    set_preference(a, bounds, pairs, nullptr, beta, 0.0f);
    a.dloss = dloss, a.given_slope = slope, a.given_stats = stats, a.dlogits = dlogits, a.dlogits_ld = dlogits_ld;
    const int rc = check(a, dtype, pairs > 0, workspace, workspace_bytes);
    if (rc == BYZ_EINVAL || !preference_ok(a) || !floats_ok(slope) || (pairs > 0 && !slope)) return BYZ_EINVAL;
    if (rc != BYZ_OK || rows == 0) return rc;
    if (!stats || !dlogits || !aligned(dlogits, dtype_size(dtype)) || dlogits_ld < vocab || !extent_ok(rows, dlogits_ld, vocab)) return BYZ_EINVAL;
    return launch(a, dtype, stream);
}

extern "C" int byz_preference_loss_step(const float *dloss, const void *logits, int64_t rows, int64_t vocab, int64_t ld, int dtype,
                                        const int32_t *label, const int32_t *bounds, int64_t pairs, const float *ref, float beta,
                                        float smoothing, float temperature, float *loss, float *sums, void *dlogits,
                                        int64_t dlogits_ld, void *workspace, size_t workspace_bytes, void *stream) {
    Args a = args_of(logits, rows, vocab, ld, label, temperature, kPreference);
    set_preference(a, bounds, pairs, ref, beta, smoothing);
    a.dloss = dloss, a.loss = loss, a.sums = sums, a.dlogits = dlogits, a.dlogits_ld = dlogits_ld;
    const int rc = check(a, dtype, pairs > 0, workspace, workspace_bytes);
    if (rc == BYZ_EINVAL || !preference_ok(a) || (pairs > 0 && (!loss || !floats_ok(loss) || !dloss || !floats_ok(dloss)))) return BYZ_EINVAL;
    if (rc != BYZ_OK) return rc;
    if (rows > 0 && (!dlogits || !aligned(dlogits, dtype_size(dtype)) || dlogits_ld < vocab || !extent_ok(rows, dlogits_ld, vocab)))
        return BYZ_EINVAL;
    return launch(a, dtype, stream);
}

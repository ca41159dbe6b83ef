// Distillation from a teacher's top logits: loss, gradient, or both in one pass (gfx950).
//
// A row's loss needs two sums: the teacher's softmax over its k entries, done in fp64 (a loss near 0 is a
// difference of larger terms, and k values cost nothing next to the vocabulary), and the student's
// log-sum-exp over the vocabulary, joined over the row's threads in a fixed order.  The gradient is dense, dloss T q_v,
// with the few places of the teacher's entries written again after it (each thread that owns an entry adds up all
// p at its place, so entries at one place write one value).  A thread's values are counted from the row's start, wherever that
// lies: the bits of a row do not depend on its address.
//
// Bound by memory: logits in, gradients out.  Loss and gradient in one call hold a long row in registers ("resident"): it
// is read once, and as soon as a thread has stored a piece of its gradient it loads that piece of its next row, so reads,
// the two exponentials of a value and writes overlap although a row fills a compute unit's registers.  Nothing else is
// in that kernel: the teacher's softmax, fp64 functions and the few places are kernels before and behind it (places
// written in it, behind a barrier, cost 17 % of its time).  Short rows are a wave's.  Rows between, too long ones and the other
// calls stream: with a running maximum m and a sum of exp((s - m) / T).
//
// 8192 x 131072 bf16, loss and gradient: resident 818 us (4.3 GB at 5.3 TB/s, a copy reaches 6.5; vector instructions issue
// 0.51 of the time), teacher 29, places 18.  8192 x 20000, twice read: loss 83, loss and gradient 174, gradient alone 140.
// 30 x 10 and 750 x 1000: 6.0 us a call, one launch, bound by the host; through LDS and barriers 7.2 and 8.1.
#include <algorithm>
#include <type_traits>

#include "worker_internal.h"

using namespace byz_worker;

namespace {

constexpr int64_t kMaxGrid = 1 << 20;
constexpr int kCus = 256;  // compute units
constexpr int kManyRows = 4 * kCus;
constexpr int kShortBytes = 16384;  // of a row that a wave holds at most

enum Mode { kLoss, kGradient, kStep };

struct Args {
    const void *logits;
    int64_t rows, vocab, ld;
    const float *teacher;
    const int32_t *index;
    int k;
    int64_t teacher_ld;
    float temperature;
    const float *dloss;
    float *loss, *lse;  // gradient alone: lse is read
    void *dlogits;
    int64_t dlogits_ld;
};

// A sum of positive terms in fp32: a thread adds some hundred of them at most, and the threads' sums are joined pairwise, so it
// is good to some 2^-23 of itself, of which the loss has the logarithm.  In fp64 it would be ten times nearer, for a conversion
// and an fp64 addition a value.
struct RunningSum {
    float m = -INFINITY, s = 0.0f;  // maximum of the raw logits, sum of exp2((x - m) c)
    template <int N>
    __device__ __forceinline__ void add(const float (&x)[N], float c) {
        float top = m;
#pragma unroll
        for (int i = 0; i < N; i++) top = fmaxf(top, x[i]);
        if (top == -INFINITY) {  // nothing but -inf so far, or NaN, which has to stay
#pragma unroll
            for (int i = 0; i < N; i++) s += x[i] == -INFINITY ? 0.0f : x[i];
            return;
        }
        float sum = s * __builtin_amdgcn_exp2f((m - top) * c);
#pragma unroll
        for (int i = 0; i < N; i++) sum += __builtin_amdgcn_exp2f((x[i] - top) * c);
        s = sum, m = top;
    }
    // The power is taken in halves: a sum of the resident kernel can be 2^117 of its m and weigh something where the power itself is
    // less than fp32 has.
    __device__ __forceinline__ void join(float m2, float s2, float c) {
        const float top = fmaxf(m, m2), half = 0.5f * c;
        const float a = __builtin_amdgcn_exp2f((m - top) * half), b = __builtin_amdgcn_exp2f((m2 - top) * half);
        s = (m == -INFINITY ? s : s * a * a) + (m2 == -INFINITY ? s2 : s2 * b * b), m = top;
    }
};

// Reductions over the NT threads of a row: in the wave, then every wave does one over the waves' results.
// `lds` has room for NT / 64 doubles.  Every thread gets the result.
__device__ __forceinline__ RunningSum wave_join(RunningSum r, float c) {
    return wave_reduce(r, [&](RunningSum a, const RunningSum &b) {
        a.join(b.m, b.s, c);
        return a;
    });
}

template <int NT>
__device__ __forceinline__ RunningSum row_join(RunningSum r, float c, double *lds) {
    constexpr int waves = NT / 64;
    r = wave_join(r, c);
    if constexpr (waves > 1) {
        float *f = reinterpret_cast<float *>(lds);
        __syncthreads();
        if (threadIdx.x % 64 == 0) f[threadIdx.x / 64 * 2] = r.m, f[threadIdx.x / 64 * 2 + 1] = r.s;
        __syncthreads();
        const int from = threadIdx.x % 64;
        r = RunningSum();
        if (from < waves) r.m = f[2 * from], r.s = f[2 * from + 1];
        r = wave_join(r, c);
    }
    return r;
}

template <int NT, typename F>
__device__ __forceinline__ double row_reduce(double v, double nothing, double *lds, F join) {
    constexpr int waves = NT / 64;
    v = wave_reduce(v, join);
    if constexpr (waves > 1) {
        __syncthreads();
        if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
        __syncthreads();
        const int from = threadIdx.x % 64;
        v = wave_reduce(from < waves ? lds[from] : nothing, join);
    }
    return v;
}
template <int NT>
__device__ __forceinline__ double row_sum(double v, double *lds) {
    return row_reduce<NT>(v, 0.0, lds, [](double a, double b) { return a + b; });
}
template <int NT>
__device__ __forceinline__ double row_max(double v, double *lds) {
    return row_reduce<NT>(v, -INFINITY, lds, [](double a, double b) { return fmax(a, b); });
}

// The values that start in the middle of v's first word and end in that of `next`.
template <typename T, int V>
__device__ __forceinline__ Words<T, V> shifted(Words<T, V> v, word_t next) {
#pragma unroll
    for (int w = 0; w < v.N; w++) v.w[w] = __builtin_amdgcn_alignbit(w + 1 < v.N ? v.w[w + 1] : next, v.w[w], 16);
    return v;
}

// A row's vocabulary as vectors of 16 bytes from its start on, wherever that lies, and a few single elements behind them.
template <typename T>
struct Row {
    static constexpr int V = 16 / sizeof(T);
    const T *at;
    int tail;
    int64_t vectors;
    __device__ Row(const void *base, int64_t row, int64_t ld, int64_t vocab) {
        at = (const T *)base + row * ld;
        vectors = vocab / V;
        tail = (int)(vocab - vectors * V);
    }
    __device__ __forceinline__ Words<T, V> vector(int64_t i) const { return get_words<T, V>(at + i * V); }
    // A row that starts at an odd multiple of two bytes: the hardware is slower to load vectors there than at whole words, so the
    // words that hold their values are loaded and shifted.  us on 8192 x 50016 bf16 as it comes / shifted: loss 176 / 149
    // (aligned 152), step 418 / 385 (354).  The half words beside the row that are loaded too are in one word with its values.
    __device__ __forceinline__ bool odd() const { return sizeof(T) == 2 && ((uintptr_t)at & 2) != 0; }
    template <bool ODD>
    __device__ __forceinline__ Words<T, V> vector_of(int64_t i) const {
        if constexpr (ODD && sizeof(T) == 2) {
            return shifted(get_words<T, V>(at + i * V - 1), *(const word_t *)(at + i * V + V - 1));
        } else {
            return vector(i);
        }
    }
    __device__ int64_t edge(int t) const { return vectors * V + t; }  // the t-th single element
};

// A row's teacher in LDS: places (-1: no entry), exp(z - top), p, and the student's logits there.
struct Teacher {
    double *weight;
    int32_t *index;
    float *p, *student;
    double top, total;
    bool some;  // an entry at all
    __device__ Teacher(char *lds, int k) {
        weight = (double *)lds, index = (int32_t *)(weight + k), p = (float *)(index + k), student = p + k;
    }
};

constexpr int kTeacherBytes = 20;  // of an entry
__host__ __device__ inline size_t teacher_bytes(int k) { return ((size_t)k * kTeacherBytes + 15) / 16 * 16; }

// Softmax over the entries that are there; `at`: the student's row.  Starts with a barrier (of the row's threads).
template <typename T, int NT>
__device__ __forceinline__ void read_teacher(const Args &a, int64_t row, const T *at, Teacher &t, int tid, double *red) {
    const double tau = a.temperature;
    double top = -INFINITY, total = 0.0;
    __syncthreads();
#pragma unroll 1
    for (int j = tid; j < a.k; j += NT) {
        const int32_t i = a.index[row * a.teacher_ld + j];
        const double z = (double)a.teacher[row * a.teacher_ld + j] / tau;
        const bool in = i >= 0 && i < a.vocab;
        if (in) top = fmax(top, z);
        t.index[j] = in ? i : -1;
        t.weight[j] = z;
        t.student[j] = in ? (float)at[i] : 0.0f;
        if (i >= a.vocab || (i >= 0 && z != z)) total = NAN;
    }
    t.top = row_max<NT>(top, red);
    const double shift = t.top > -INFINITY ? t.top : 0.0;
#pragma unroll 1
    for (int j = tid; j < a.k; j += NT)
        if (t.index[j] >= 0) total += t.weight[j] = exp(t.weight[j] - shift);
    t.total = row_sum<NT>(total, red);
    t.some = t.total > 0.0 || t.total != t.total;
}

// p, and the loss with the student's log-sum-exp m / tau + log_sum.  Logits are taken less m first: next to an m of 10^30 no
// other term has a bit.
template <int NT>
__device__ __forceinline__ double loss_of(const Args &a, Teacher &t, double m, double log_sum, int tid, double *red) {
    const double tau = a.temperature;
    double part = 0.0;
#pragma unroll 1
    for (int j = tid; j < a.k; j += NT) {
        const double p = t.index[j] < 0 ? 0.0 : t.weight[j] / t.total;
        t.p[j] = (float)p;
        if (p > 0.0) part += p * (log(p) - (((double)t.student[j] - m) / tau - log_sum));
        if (p != p) part = NAN;
    }
    part = row_sum<NT>(part, red);
    return !t.some ? 0.0 : t.total != t.total ? NAN : tau * tau * part;
}

// q_v times a weight, from a logit.  The exponent is (x - m) c - l, with c = log2(e) / T in two parts where the result is fp32.
// The instruction's exp2 gives 0 below 2^-126, where a product with the weight still has a value: there the
// exponent is raised by 32 and the product lowered by it.
template <typename T>
struct Softmax {
    float m, c, c_low, l, w;
    __device__ Softmax(double m_, double log_sum, double temperature, float weight) {
        const double s = 1.4426950408889634 / temperature;
        m = (float)m_, c = (float)s, c_low = (float)(s - (double)c), l = (float)(log_sum * 1.4426950408889634), w = weight;
    }
    // from a maximum and a sum in fp32; c is log2(e) / T
    __device__ Softmax(float m_, float sum, float temperature, float weight, float c_) {
        m = m_, c = c_, l = __builtin_amdgcn_logf(sum), w = weight;
        // what c is short of: log2(e) = hi + lo, and the remainder of hi - c T
        c_low = sizeof(T) == 4 ? (fmaf(-c, temperature, 0x1.715476p+0f) + 0x1.4ae0c0p-26f) / temperature : 0.0f;
    }
    __device__ __forceinline__ float weighted(float x) const { return less(x, 0.0f); }
    // w (q - p)
    __device__ __forceinline__ float less(float x, float p) const {
        const float d = x - m;
        if constexpr (sizeof(T) == 4) {
            // c_low can be 0 or less: the small term of a banned entry, d = -inf, is that of a finite d, or the sum would be NaN
            const float e = fmaf(d, c, fmaf(fmaxf(d, -0x1p64f), c_low, -l));
            const bool low = e < -100.0f;
            const float q = __builtin_amdgcn_exp2f(low ? e + 32.0f : e);
            return low ? (q - p * 0x1p32f) * (w * 0x1p-32f) : (q - p) * w;
        } else {
            return (__builtin_amdgcn_exp2f(fmaf(d, c, 32.0f - l)) - p * 0x1p32f) * (w * 0x1p-32f);
        }
    }
};

// The same from a row's sum of exp2(x c - m), for the resident kernel.
template <typename T>
struct ScaledSoftmax;
template <>
struct ScaledSoftmax<float> : Softmax<float> {
    using Softmax<float>::Softmax;
};
// 16-bit types: the exponent in one operation, x c - high.  m can be large (fp16 logits reach 65504) where q has 11 bits, so
// only what is exact or accounted for is added to it: the sum's whole powers of two; what the addition's rounding took and
// the sum's mantissa make a factor.  With m + log2(sum) rounded to fp32 instead q was 0.27 % off at logits of 60000.
template <typename T>
struct ScaledSoftmax {
    float c, high, share, w;
    __device__ ScaledSoftmax(float m, float sum, float, float weight, float c_) {
        const float t = (float)(__builtin_amdgcn_frexp_expf(sum) - 32);
        c = c_, high = m + t;
        const float back = high - m, lost = (m - (high - back)) + (t - back);
        share = __builtin_amdgcn_exp2f(-lost) / __builtin_amdgcn_frexp_mantf(sum), w = weight * 0x1p-32f;
    }
    __device__ __forceinline__ float less(float x, float p) const {
        return (__builtin_amdgcn_exp2f(fmaf(x, c, -high)) * share - p * 0x1p32f) * w;
    }
    __device__ __forceinline__ float weighted(float x) const { return __builtin_amdgcn_exp2f(fmaf(x, c, -high)) * (share * w); }
};

// The gradient by its own call has a row's log-sum-exp in fp32, half a step of which is a share of q.  Up to here that is
// 2^-19 of q, as much as the other terms' rounding; a row beyond (logits far from 0, or all of a mask's value) is summed again.
__device__ __forceinline__ bool lse_is_good(float lse) { return fabsf(lse) <= 64.0f; }

// The gradient at the teacher's places; the dense part is written.
template <typename T, int NT>
__device__ __forceinline__ void write_places(const Args &a, const Teacher &t, const Softmax<T> &q, T *out, int tid) {
#pragma unroll 1
    for (int j = tid; j < a.k; j += NT) {
        const int32_t i = t.index[j];
        if (i < 0) continue;
        float p = 0.0f;
#pragma unroll 1
        for (int l = 0; l < a.k; l++) p += t.index[l] == i ? t.p[l] : 0.0f;
        out[i] = round_to<T>(q.less(t.student[j], p));
    }
}

// The step of 256 threads in 96 registers, five blocks a compute unit: 8192 x 20000 fp16 takes 176 us so, 192 with three more.
// bf16 does without being told, and is slower told (20011 words 188 us for 178).
template <typename T, int NT, Mode MODE>
__global__ __launch_bounds__(NT, MODE == kStep && NT == 256 && (std::is_same_v<T, f16>) ? 5 : NT / 256) void distill_kernel(Args a) {
    extern __shared__ char lds_raw[];
    __shared__ double red[32];
    constexpr int V = 16 / sizeof(T);
    const int tid = threadIdx.x;
    const double tau = a.temperature;
    const float c = (float)(1.4426950408889634 / tau);
    Teacher t(lds_raw, a.k);
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const Row<T> r(a.logits, row, a.ld, a.vocab);
        // sent ahead of the teacher's chain; in the step, which is at its registers' end, later
        const float given = MODE == kGradient ? a.lse[row] : 0.0f, early = MODE == kGradient ? a.dloss[row] : 0.0f;
        read_teacher<T, NT>(a, row, r.at, t, tid, red);
        double m, log_sum;  // the student's log-sum-exp is m / tau + log_sum
        if (MODE != kGradient || !lse_is_good(given)) {
            RunningSum s;
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
            if constexpr (MODE == kGradient) {
                // the exception, in few registers, or all rows would have fewer waves
#pragma unroll 1
                for (int64_t i = tid; i < r.vectors * (V / 4); i += NT) {
                    const Words<T, 4> v = get_words<T, 4>(r.at + i * 4);
                    float x[4];
#pragma unroll
                    for (int e = 0; e < 4; e++) x[e] = v[e];
                    s.add(x, c);
                }
            } else if (r.odd()) {
                add_up(std::true_type{});
            } else {
                add_up(std::false_type{});
            }
            s = row_join<NT>(s, c, red);
            // the gradient's needs no more than fp32; a logarithm in fp64 would cost all rows two waves
            m = s.m, log_sum = MODE == kGradient ? (double)(__builtin_amdgcn_logf(s.s) * 0.69314718f) : log((double)s.s);
        } else {
            m = (float)(given * tau), log_sum = given - m / tau;
        }
        if constexpr (MODE != kGradient) {
            const double loss = loss_of<NT>(a, t, m, log_sum, tid, red);
            if (tid == 0) {
                a.loss[row] = (float)loss;
                if (a.lse) a.lse[row] = (float)(m / tau + log_sum);
            }
        } else {
#pragma unroll 1
            for (int j = tid; j < a.k; j += NT) t.p[j] = t.index[j] < 0 ? 0.0f : (float)(t.weight[j] / t.total);
        }
        if constexpr (MODE != kLoss) {
            const Softmax<T> q(m, log_sum, tau, t.total != t.total ? NAN : a.temperature * (MODE == kGradient ? early : a.dloss[row]));
            T *out = (T *)a.dlogits + row * a.dlogits_ld;
            __syncthreads();  // the logits at the teacher's places are read: they may be written now
            if (tid < r.tail) {
                const int64_t e = r.edge(tid);
                out[e] = t.some ? round_to<T>(q.weighted((float)r.at[e])) : (T)0.0f;
            }
            auto write = [&](auto odd) {
                for (int64_t i = tid; i < r.vectors; i += NT) {
                    const Words<T, V> v = r.template vector_of<odd.value>(i);
                    put_words(out + i * V, Words<T, V>::of([&](int e) { return t.some ? q.weighted(v[e]) : 0.0f; }));
                }
            };
            if (r.odd())
                write(std::true_type{});
            else
                write(std::false_type{});
            __syncthreads();  // the dense part is written: the teacher's places again
            if (t.some) write_places<T, NT>(a, t, q, out, tid);
        }
    }
}

// Short rows, R KB and 64 E entries of the teacher at most: a wave a row, everything in its registers, all loads sent
// first.  Bound by one chain: places, the student there, fp64 functions and four reductions.
template <typename T, Mode MODE, int R, int E>
__global__ __launch_bounds__(256) void distill_short_kernel(Args a) {
    constexpr int V = 16 / sizeof(T);
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const double tau = a.temperature, inv = 1.0 / tau;
    const float c = (float)(1.4426950408889634 / tau);
    for (int64_t row = (int64_t)blockIdx.x * 4 + wave; row < a.rows; row += (int64_t)gridDim.x * 4) {
        const Row<T> r(a.logits, row, a.ld, a.vocab);
        int32_t index[E];
        float t[E], student[E];
#pragma unroll
        for (int e = 0; e < E; e++) {
            const int j = e * 64 + lane;
            index[e] = -1, t[e] = 0.0f;
            if (j < a.k) index[e] = a.index[row * a.teacher_ld + j], t[e] = a.teacher[row * a.teacher_ld + j];
        }
        Words<T, V> x[R];
#pragma unroll
        for (int v = 0; v < R; v++)
            if (v * 64 + lane < r.vectors) x[v] = get_words<T, V>(r.at + (uint32_t)(v * 64 + lane) * V);
        const bool has_edge = lane < r.tail;
        T edge = (T)0.0f;
        if (has_edge) edge = r.at[r.edge(lane)];
        const float given = MODE == kGradient ? a.lse[row] : 0.0f, dloss = MODE == kLoss ? 0.0f : a.dloss[row];
        float first = -INFINITY;
        bool broken = false;
#pragma unroll
        for (int e = 0; e < E; e++) {
            const bool in = index[e] >= 0 && index[e] < a.vocab;
            student[e] = in ? (float)r.at[index[e]] : 0.0f;
            if (in) first = fmaxf(first, t[e]);
            broken = broken || index[e] >= a.vocab || (in && t[e] != t[e]);
        }
        first = wave_reduce(first, [](float p, float q) { return fmaxf(p, q); });
        const double top = first > -INFINITY ? (double)first : 0.0;
        double weight[E], total = 0.0;
#pragma unroll
        for (int e = 0; e < E; e++) {
            weight[e] = index[e] >= 0 ? exp(((double)t[e] - top) * inv) : 0.0;
            total += weight[e];
        }
        total = row_sum<64>(total, nullptr);
        if (__ballot(broken) != 0) total = NAN;
        const bool some = total > 0.0 || total != total;
#pragma unroll
        for (int e = 0; e < E; e++) weight[e] = index[e] < 0 ? 0.0 : weight[e] / total;
        double m, log_sum;
        if (MODE != kGradient || !lse_is_good(given)) {
            RunningSum s;
            if (has_edge) {
                const float y[1] = {(float)edge};
                s.add(y, c);
            }
#pragma unroll
            for (int v = 0; v < R; v++)
                if (v * 64 + lane < r.vectors) {
                    float y[V];
#pragma unroll
                    for (int i = 0; i < V; i++) y[i] = x[v][i];
                    s.add(y, c);
                }
            s = wave_join(s, c);
            m = s.m, log_sum = log((double)s.s);
        } else {
            m = (float)(given * tau), log_sum = given - m * inv;
        }
        if constexpr (MODE != kGradient) {
            const double log_total = log(total);
            double part = 0.0;
#pragma unroll
            for (int e = 0; e < E; e++)
                if (weight[e] > 0.0) part += weight[e] * ((((double)t[e] - top) - ((double)student[e] - m)) * inv - log_total + log_sum);
            part = row_sum<64>(part, nullptr);
            if (lane == 0) {
                a.loss[row] = !some ? 0.0f : total != total ? NAN : (float)(tau * tau * part);
                if (a.lse) a.lse[row] = (float)(m * inv + log_sum);
            }
        }
        if constexpr (MODE != kLoss) {
            float p[E] = {};
#pragma unroll
            for (int f = 0; f < E; f++) {
                const int end = std::min(64, a.k - f * 64), own = __builtin_bit_cast(int, (float)weight[f]);
                for (int l = 0; l < end; l++) {
                    const int il = __builtin_amdgcn_readlane(index[f], l);
                    const float pl = __builtin_bit_cast(float, __builtin_amdgcn_readlane(own, l));
#pragma unroll
                    for (int e = 0; e < E; e++) p[e] += il == index[e] ? pl : 0.0f;
                }
            }
            const Softmax<T> q(m, log_sum, tau, total != total ? NAN : a.temperature * dloss);
            T *out = (T *)a.dlogits + row * a.dlogits_ld;
            if (has_edge) out[r.edge(lane)] = some ? round_to<T>(q.weighted((float)edge)) : (T)0.0f;
#pragma unroll
            for (int v = 0; v < R; v++)
                if (v * 64 + lane < r.vectors)
                    put_words(out + (uint32_t)(v * 64 + lane) * V, Words<T, V>::of([&](int i) { return some ? q.weighted(x[v][i]) : 0.0f; }));
            // the dense part is written, in the wave's order: the teacher's places again
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int e = 0; e < E; e++)
                if (some && index[e] >= 0 && index[e] < a.vocab) out[index[e]] = round_to<T>(q.less(student[e], p[e]));
        }
    }
}

// A row's part of the workspace of the resident kernel, beside its k places.
struct RowSums {
    double entropy;  // sum of p log p
    double dot, ps;  // sums of p (s - at) and p over the places
    float m, s;      // the student's maximum (16-bit types: times c) and sum
    int flags;       // kSome: an entry at all; kBroken: the row is NaN
    float at;        // the largest s of the places with weight: differences of logits keep what a sum of large ones loses
};
struct Place {
    float p, student;  // of all entries at the place; the student's logit
};
enum { kSome = 1, kBroken = 2 };

// The teacher's softmax and what the student has at its places, a wave a row.
template <typename T>
__global__ __launch_bounds__(256) void distill_teacher_kernel(Args a, Place *places, RowSums *sums) {
    extern __shared__ double own[];
    const double tau = a.temperature;
    const int lane = threadIdx.x % 64;
    double *const each = own + threadIdx.x / 64 * a.k;  // a lane reads what it has written itself
    for (int64_t row = (int64_t)blockIdx.x * 4 + threadIdx.x / 64; row < a.rows; row += (int64_t)gridDim.x * 4) {
        const float *t = a.teacher + row * a.teacher_ld;
        const int32_t *index = a.index + row * a.teacher_ld;
        const T *logits = (const T *)a.logits + row * a.ld;
        double top = -INFINITY, total = 0.0, entropy = 0.0, dot = 0.0, ps = 0.0;
        bool broken = false;
        for (int j = lane; j < a.k; j += 64)
            if (index[j] >= 0) {
                const double z = (double)t[j] / tau;
                top = fmax(top, z);
                broken = broken || z != z || index[j] >= a.vocab;
            }
        top = row_max<64>(top, nullptr);
        const double shift = top > -INFINITY ? top : 0.0;
        for (int j = lane; j < a.k; j += 64) {
            const int32_t i = index[j];
            const float s = i >= 0 && i < a.vocab ? (float)logits[i] : 0.0f;
            const double e = i >= 0 ? exp((double)t[j] / tau - shift) : 0.0;
            total += e;
            each[j] = e;
            places[row * a.k + j].student = s;
        }
        total = row_sum<64>(total, nullptr);
        broken = __ballot(broken) != 0 || total != total;
        const bool some = total > 0.0 || broken;
        float at = -INFINITY;
        for (int j = lane; j < a.k; j += 64) {
            const double w = index[j] < 0 || !some ? 0.0 : broken ? NAN : each[j] / total;
            each[j] = w;
            if (w > 0.0) at = fmaxf(at, places[row * a.k + j].student);
        }
        at = wave_reduce(at, [](float p, float q) { return fmaxf(p, q); });
        if (at == -INFINITY) at = 0.0f;
        for (int j = lane; j < a.k; j += 64) {
            const double w = each[j];
            if (w > 0.0) entropy += w * log(w), dot += w * ((double)places[row * a.k + j].student - (double)at), ps += w;
        }
        entropy = row_sum<64>(entropy, nullptr);
        dot = row_sum<64>(dot, nullptr);
        ps = row_sum<64>(ps, nullptr);
        if (lane == 0) {
            sums[row].entropy = entropy, sums[row].dot = dot, sums[row].ps = ps;
            sums[row].flags = (some ? kSome : 0) | (broken ? kBroken : 0), sums[row].at = at;
        }
        for (int j0 = 0; j0 < a.k; j0 += 64) {
            const int32_t i = j0 + lane < a.k ? index[j0 + lane] : -1;
            float p = 0.0f;
            for (int l0 = 0; l0 < a.k; l0 += 64) {
                const int32_t il = l0 + lane < a.k ? index[l0 + lane] : -1;
                const float pl = l0 + lane < a.k ? (float)each[l0 + lane] : 0.0f;
                const int end = std::min(64, a.k - l0);
                for (int l = 0; l < end; l++) {
                    const float pj = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, pl), l));
                    p += __builtin_amdgcn_readlane(il, l) == i ? pj : 0.0f;
                }
            }
            if (j0 + lane < a.k) places[row * a.k + j0 + lane].p = p;
        }
    }
}

// Rows whose maximum in c times a value is not small beside 2^31: the rounding of such a product is no small power of two, and
// past 2^128 there is no product (16-bit types; a row that is all banned, or masked with the type's lowest value).
template <typename T>
__device__ __forceinline__ bool is_far(float m) {
    return sizeof(T) == 2 && !(fabsf(m) < 0x1p28f);
}

// A far row, of which the resident kernel has written nothing: its sum about its maximum and, where the teacher has an entry, its
// dense gradient, by a wave.
template <typename T>
__device__ __forceinline__ Softmax<T> far_row(const Args &a, int64_t row, bool some, float weight, float c, RunningSum &s, int lane) {
    constexpr int V = 16 / sizeof(T);
    const Row<T> r(a.logits, row, a.ld, a.vocab);
    const bool has_edge = lane < r.tail;
    s = RunningSum();
    if (has_edge) {
        const float x[1] = {(float)r.at[r.edge(lane)]};
        s.add(x, c);
    }
    for (int64_t i = lane; i < r.vectors; i += 64) {
        const Words<T, V> v = r.vector(i);
        float x[V];
#pragma unroll
        for (int e = 0; e < V; e++) x[e] = v[e];
        s.add(x, c);
    }
    s = wave_join(s, c);
    const Softmax<T> q(s.m, log((double)s.s), a.temperature, weight);
    if (some) {
        T *out = (T *)a.dlogits + row * a.dlogits_ld;
        if (has_edge) out[r.edge(lane)] = round_to<T>(q.weighted((float)r.at[r.edge(lane)]));
        for (int64_t i = lane; i < r.vectors; i += 64) {
            const Words<T, V> v = r.vector(i);
            put_words(out + i * V, Words<T, V>::of([&](int e) { return q.weighted(v[e]); }));
        }
        // written, in the wave's order, before the teacher's places
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
        __builtin_amdgcn_wave_barrier();
    }
    return q;
}

// The losses, and the gradient at the teacher's places (the dense part is written), a wave a row.
template <typename T>
__global__ __launch_bounds__(256) void distill_places_kernel(Args a, const Place *places, const RowSums *sums) {
    const double tau = a.temperature;
    const float c = (float)(1.4426950408889634 / tau);
    const int lane = threadIdx.x % 64;
    for (int64_t row = (int64_t)blockIdx.x * 4 + threadIdx.x / 64; row < a.rows; row += (int64_t)gridDim.x * 4) {
        const RowSums r = sums[row];
        const bool some = r.flags & kSome;
        const float weight = r.flags & kBroken ? NAN : a.temperature * a.dloss[row];
        auto finish = [&](double m, float s, const auto &q) {
            if (lane == 0) {
                const double log_sum = log((double)s);
                a.loss[row] = r.flags & kBroken ? NAN
                              : some            ? (float)(tau * tau * (r.entropy - (r.dot + r.ps * ((double)r.at - m)) / tau + r.ps * log_sum))
                                                : 0.0f;
                if (a.lse) a.lse[row] = (float)(m / tau + log_sum);
            }
            if (!some) return;
            T *out = (T *)a.dlogits + row * a.dlogits_ld;
            for (int j = lane; j < a.k; j += 64) {
                const int32_t i = a.index[row * a.teacher_ld + j];
                const Place at = places[row * a.k + j];
                if (i >= 0 && i < a.vocab) out[i] = round_to<T>(q.less(at.student, at.p));
            }
        };
        if (is_far<T>(r.m)) {
            RunningSum s;
            const Softmax<T> q = far_row<T>(a, row, some, weight, c, s, lane);
            finish(s.m, s.s, q);
        } else {
            finish(sizeof(T) == 4 ? (double)r.m : (double)r.m / (double)c, r.s, ScaledSoftmax<T>(r.m, r.s, a.temperature, weight, c));
        }
    }
}

// The dense gradients and the student's sums.  R vectors of a row in each of 1024 threads' registers.
template <typename T, int R>
__global__ __launch_bounds__(1024) void distill_resident_kernel(Args a, RowSums *sums) {
    constexpr int V = 16 / sizeof(T), NT = 1024;
    __shared__ double red[32];
    const int tid = threadIdx.x;
    const float c = (float)(1.4426950408889634 / (double)a.temperature);
    Words<T, V> x[R];
    T edge = (T)0.0f;
    // A row here is shorter than 2^31 bytes.  A thread's number `own` is made afresh for each use, or the places of all R
    // vectors would be kept in registers; threads without a v-th vector load the last, without a branch, and leave it.
    auto vector_at = [](auto *base, int number) { return base + (uint32_t)number * (uint32_t)V; };
    // Of an odd row x has the words that hold the values but for the last value's; shifted where the row is begun.
    word_t next_word[R];
    auto load = [&](const Row<T> &r, int own, int v) {
        const T *from = vector_at(r.at - (r.odd() ? 1 : 0), std::min(own + v * NT, (int)r.vectors - 1));
        x[v] = get_words<T, V>(from);
        if (r.odd()) next_word[v] = *(const word_t *)(from + V);
    };
    // 16-bit types: sums are of exp2(x c - m) with m = c times a value, rounded: one operation for the exponent
    constexpr bool kScaled = sizeof(T) == 2;
    const float unit = kScaled ? 1.0f : c;
    auto scaled = [&](float v) { return kScaled ? v * c : v; };
    auto load_edge = [&](const Row<T> &r) {
        if (tid < r.tail) edge = r.at[r.edge(tid)];
    };
    {
        const Row<T> r(a.logits, blockIdx.x, a.ld, a.vocab);
#pragma unroll
        for (int v = 0; v < R; v++) load(r, tid, v);
        load_edge(r);
    }
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const Row<T> r(a.logits, row, a.ld, a.vocab);
        if constexpr (sizeof(T) == 2)
            if (r.odd())
#pragma unroll
                for (int v = 0; v < R; v++) x[v] = shifted(x[v], next_word[v]);
        // A thread's sum of exp2((x - m) c).  The maximum of its first values is m.  The row's sum of 1024 such sums has to stay
        // below fp32's 2^128, so what reaches 2^117 (or is not finite) is summed again from the maximum of all.
        const bool has_edge = tid < r.tail;
        RunningSum s;
        if (tid < r.vectors) {
            float top = x[0][0];
#pragma unroll
            for (int e = 1; e < V; e++) top = fmaxf(top, x[0][e]);
            s.m = scaled(top);
        } else if (has_edge) {
            s.m = scaled((float)edge);
        }
        // of 16-bit values to a rounded product m: the product's rounding is in the sum, which the gradient takes into account
        auto power = [&](float v, float m) { return __builtin_amdgcn_exp2f(kScaled ? fmaf(v, c, -m) : (v - m) * c); };
        const int vectors = (int)r.vectors, own = afresh(tid);
        auto add_up = [&](float m) {
            float all = 0.0f;
#pragma unroll
            for (int v = 0; v < R; v++) {
                float sum = 0.0f;
#pragma unroll
                for (int e = 0; e < V; e++) sum += power(x[v][e], m);
                all += own + v * NT < vectors ? sum : 0.0f;
                x[v].keep();
                __builtin_amdgcn_sched_barrier(0);  // one vector's values in registers at a time
            }
            return has_edge ? all + power((float)edge, m) : all;
        };
        s.s = add_up(s.m);
        if (!(s.s < 0x1p117f)) {
            float top = has_edge ? fmaxf((float)edge, -INFINITY) : -INFINITY;
#pragma unroll
            for (int v = 0; v < R; v++) {
#pragma unroll
                for (int e = 0; e < V; e++) top = own + v * NT < vectors ? fmaxf(top, x[v][e]) : top;
                x[v].keep();
                __builtin_amdgcn_sched_barrier(0);
            }
            s.m = scaled(top);
            // nothing but -inf (or NaN, which has to stay) adds up to 0, and so does what is far below: the row is far itself or has more
            s.s = add_up(s.m == -INFINITY || is_far<T>(s.m) ? 0.0f : s.m);
        }
        s = row_join<NT>(s, unit, red);
        const int flags = sums[row].flags;
        if (tid == 0) sums[row].m = s.m, sums[row].s = s.s;
        const bool some = flags & kSome;
        const ScaledSoftmax<T> q(s.m, s.s, a.temperature, flags & kBroken ? NAN : a.temperature * a.dloss[row], c);
        T *out = (T *)a.dlogits + row * a.dlogits_ld;
        const bool left = some && __builtin_amdgcn_readfirstlane((int)is_far<T>(s.m));  // to the places' kernel
        if (has_edge && !left) {
            const int64_t e = r.edge(tid);
            out[e] = some ? round_to<T>(q.weighted((float)edge)) : (T)0.0f;
        }
        const int then = afresh(tid);
        auto pass = [&](auto gradient, auto store, auto more, const Row<T> &next) {
#pragma unroll
            for (int v = 0; v < R; v++) {
                if (store.value && then + v * NT < vectors)
                    put_past_caches(vector_at(out, then + v * NT), Words<T, V>::of([&](int e) { return gradient(x[v][e]); }));
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (more.value) {
                    load(next, then, v);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        };
        auto weighted = [&](float v) { return q.weighted(v); };
        auto none = [](float) { return 0.0f; };
        if (row + gridDim.x < a.rows) {
            const Row<T> next(a.logits, row + gridDim.x, a.ld, a.vocab);
            load_edge(next);
            if (left)
                pass(none, std::false_type{}, std::true_type{}, next);
            else if (some)
                pass(weighted, std::true_type{}, std::true_type{}, next);
            else
                pass(none, std::true_type{}, std::true_type{}, next);
        } else if (left) {
        } else if (some) {
            pass(weighted, std::true_type{}, std::false_type{}, r);
        } else {
            pass(none, std::true_type{}, std::false_type{}, r);
        }
    }
}

template <typename T, int NT, Mode MODE>
int launch_threads(const Args &a, hipStream_t s) {
    distill_kernel<T, NT, MODE><<<(unsigned)std::min(a.rows, kMaxGrid), NT, teacher_bytes(a.k), s>>>(a);
    BYZ_HIP(hipGetLastError());
    return BYZ_OK;
}

template <typename T, Mode MODE, int R>
int launch_short(const Args &a, hipStream_t s) {
    const unsigned grid = (unsigned)std::min((a.rows + 3) / 4, kMaxGrid);
    if (a.k <= 64)
        distill_short_kernel<T, MODE, R, 1><<<grid, 256, 0, s>>>(a);
    else
        distill_short_kernel<T, MODE, R, 4><<<grid, 256, 0, s>>>(a);
    BYZ_HIP(hipGetLastError());
    return BYZ_OK;
}

// Rows that the resident kernel takes: their threads' vectors fit, and there is one for every compute unit.
constexpr int kResident = 16;  // vectors of a thread
bool fits_resident(int64_t rows, int64_t vocab, int dtype) {
    const int64_t vectors = vocab * (int64_t)dtype_size(dtype) / 16;
    return vectors >= 1024 * 4 && vectors <= 1024 * kResident && rows >= kCus / 2;
}

size_t resident_bytes(int64_t rows, int k) { return (size_t)rows * (sizeof(RowSums) + (size_t)k * sizeof(Place)); }

template <typename T>
int launch_resident(const Args &a, void *workspace, hipStream_t s) {
    RowSums *sums = (RowSums *)workspace;
    Place *places = (Place *)(sums + a.rows);
    const unsigned waves = (unsigned)std::min<int64_t>((a.rows + 3) / 4, kMaxGrid), grid = (unsigned)std::min<int64_t>(a.rows, kCus);
    distill_teacher_kernel<T><<<waves, 256, 4 * a.k * sizeof(double), s>>>(a, places, sums);
    BYZ_HIP(hipGetLastError());
    if (a.vocab * (int64_t)sizeof(T) / 16 <= 1024 * kResident / 2)
        distill_resident_kernel<T, kResident / 2><<<grid, 1024, 0, s>>>(a, sums);
    else
        distill_resident_kernel<T, kResident><<<grid, 1024, 0, s>>>(a, sums);
    BYZ_HIP(hipGetLastError());
    distill_places_kernel<T><<<waves, 256, 0, s>>>(a, places, sums);
    BYZ_HIP(hipGetLastError());
    return BYZ_OK;
}

template <typename T, Mode MODE>
int launch_mode(const Args &a, hipStream_t s) {
    const int64_t bytes = a.vocab * (int64_t)sizeof(T);
    if (bytes <= kShortBytes && a.k <= 256) return bytes <= 4096 ? launch_short<T, MODE, 4>(a, s) : launch_short<T, MODE, 16>(a, s);
    // Blocks of 256 threads where every compute unit has rows for several, whose chains then overlap, or where a row is short.
    // us, blocks of 1024 / 256: loss of 8192 x 20000 bf16 261 / 80, of 8192 x 50000 322 / 152, step on 8192 x 20000 342 / 184.
    // A wave a row against a block of 256: step on 8192 x 3000 bf16 33.6 / 66.2, loss of 8192 x 5000 22.4 / 49.3.
    if (bytes <= 32768 || a.rows >= kManyRows) return launch_threads<T, 256, MODE>(a, s);
    return launch_threads<T, 1024, MODE>(a, s);
}

template <Mode MODE>
int launch(const Args &a, int dtype, hipStream_t s) {
    if (dtype == BYZ_F32) return launch_mode<float, MODE>(a, s);
    if (dtype == BYZ_BF16) return launch_mode<bf16, MODE>(a, s);
    return launch_mode<f16, MODE>(a, s);
}

bool sizes_ok(int64_t rows, int64_t vocab, int k, int dtype) {
    return rows >= 0 && vocab >= 1 && vocab <= INT32_MAX && k >= 1 && k <= BYZ_MAX_TEACHER && dtype_known(dtype);
}

int check(const Args &a, int dtype) {
    if (!sizes_ok(a.rows, a.vocab, a.k, dtype) || !(a.temperature > 0.0f) || !(a.temperature < INFINITY)) return BYZ_EINVAL;
    if (a.rows == 0) return BYZ_OK;
    if (!a.logits || !a.teacher || !a.index || !aligned(a.logits, dtype_size(dtype))) return BYZ_EINVAL;
    if (a.ld < a.vocab || !extent_ok(a.rows, a.ld, a.vocab) || a.teacher_ld < a.k || !extent_ok(a.rows, a.teacher_ld, a.k))
        return BYZ_EINVAL;
    return BYZ_OK;
}

int check_gradient(const Args &a, int dtype) {
    const int rc = check(a, dtype);
    if (rc != BYZ_OK || a.rows == 0) return rc;
    if (!a.dloss || !a.dlogits || !aligned(a.dlogits, dtype_size(dtype)) || a.dlogits_ld < a.vocab ||
        !extent_ok(a.rows, a.dlogits_ld, a.vocab))
        return BYZ_EINVAL;
    return BYZ_OK;
}

}  // namespace

extern "C" size_t byz_distill_loss_step_workspace_bytes(int64_t rows, int64_t vocab, int k, int dtype) {
    return sizes_ok(rows, vocab, k, dtype) && fits_resident(rows, vocab, dtype) ? resident_bytes(rows, k) : 0;
}

extern "C" int byz_distill_loss(const void *logits, int64_t rows, int64_t vocab, int64_t ld, int dtype,
                                const float *teacher, const int32_t *index, int k, int64_t teacher_ld,
                                float temperature, float *loss, float *lse, void *stream) {
    const Args a{logits, rows, vocab, ld, teacher, index, k, teacher_ld, temperature, nullptr, loss, lse, nullptr, 0};
    const int rc = check(a, dtype);
    if (rc != BYZ_OK || rows == 0) return rc;
    if (!loss) return BYZ_EINVAL;
    return launch<kLoss>(a, dtype, (hipStream_t)stream);
}

extern "C" int byz_distill_loss_backward(const float *dloss, const void *logits, int64_t rows, int64_t vocab,
                                         int64_t ld, int dtype, const float *teacher, const int32_t *index, int k,
                                         int64_t teacher_ld, const float *lse, float temperature, void *dlogits,
                                         int64_t dlogits_ld, void *stream) {
    const Args a{logits,     rows,        vocab, ld,      teacher,                   index,   k,
                 teacher_ld, temperature, dloss, nullptr, const_cast<float *>(lse), dlogits, dlogits_ld};
    const int rc = check_gradient(a, dtype);
    if (rc != BYZ_OK || rows == 0) return rc;
    if (!lse) return BYZ_EINVAL;
    return launch<kGradient>(a, dtype, (hipStream_t)stream);
}

extern "C" int byz_distill_loss_step(const void *logits, int64_t rows, int64_t vocab, int64_t ld, int dtype,
                                     const float *teacher, const int32_t *index, int k, int64_t teacher_ld,
                                     const float *dloss, float temperature, float *loss, float *lse, void *dlogits,
                                     int64_t dlogits_ld, void *workspace, size_t workspace_bytes, void *stream) {
    const Args a{logits, rows, vocab, ld, teacher, index, k, teacher_ld, temperature, dloss, loss, lse, dlogits, dlogits_ld};
    const int rc = check_gradient(a, dtype);
    if (rc != BYZ_OK || rows == 0) return rc;
    if (!loss) return BYZ_EINVAL;
    if (fits_resident(rows, vocab, dtype)) {
        if (workspace_bytes < resident_bytes(rows, k) || !workspace || !aligned(workspace, 16)) return BYZ_ENOMEM;
        const hipStream_t s = (hipStream_t)stream;
        return dtype == BYZ_F32 ? launch_resident<float>(a, workspace, s)
               : dtype == BYZ_BF16 ? launch_resident<bf16>(a, workspace, s) : launch_resident<f16>(a, workspace, s);
    }
    return launch<kStep>(a, dtype, (hipStream_t)stream);
}

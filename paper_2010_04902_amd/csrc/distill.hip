// Distillation from a teacher's top logits: loss, gradient, or both in one pass (gfx950).
//
// A row's loss needs two sums: the teacher's softmax over its k entries, done in fp64 (a loss near 0 is a
// difference of larger terms, and k values cost nothing next to the vocabulary), and the student's
// log-sum-exp over the vocabulary: one pass with a running maximum m and a sum S of exp((s - m) / T) per
// thread, joined over the row's threads in a fixed order.  The gradient is dense, dloss T q_v, with the
// few places of the teacher's entries written again after it (each thread that owns an entry adds up all
// p at its place, so entries at one place write one value).  Bound by memory: logits in, gradients out.
#include <algorithm>

#include "worker_internal.h"

using namespace byz_worker;

namespace {

constexpr int64_t kMaxGrid = 1 << 20;

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
    __device__ __forceinline__ void join(float m2, float s2, float c) {
        const float top = fmaxf(m, m2);
        const float a = m == -INFINITY ? s : s * __builtin_amdgcn_exp2f((m - top) * c);
        const float b = m2 == -INFINITY ? s2 : s2 * __builtin_amdgcn_exp2f((m2 - top) * c);
        s = a + b, m = top;
    }
};

// Reductions over the NT threads of a row: a butterfly in the wave, then the waves in order.  `lds` has room
// for 2 * NT / 64 doubles.  Every thread gets the result.
template <int NT>
__device__ RunningSum row_join(RunningSum r, float c, double *lds) {
    for (int off = 1; off < 64; off *= 2) {
        // both sides of a pair join lower lane first and get the same bits
        const float m2 = __shfl_xor(r.m, off), s2 = __shfl_xor(r.s, off);
        RunningSum lo = r;
        if (threadIdx.x & off) {
            lo.m = m2, lo.s = s2;
            lo.join(r.m, r.s, c);
        } else {
            lo.join(m2, s2, c);
        }
        r = lo;
    }
    if constexpr (NT > 64) {
        float *f = reinterpret_cast<float *>(lds);
        __syncthreads();
        if (threadIdx.x % 64 == 0) f[threadIdx.x / 64 * 2] = r.m, f[threadIdx.x / 64 * 2 + 1] = r.s;
        __syncthreads();
        RunningSum all;
        for (int w = 0; w < NT / 64; w++) all.join(f[2 * w], f[2 * w + 1], c);
        r = all;
    }
    return r;
}

template <int NT>
__device__ double row_sum(double v, double *lds) {
    for (int off = 32; off; off >>= 1) v += __shfl_xor(v, off);
    if constexpr (NT > 64) {
        __syncthreads();
        if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
        __syncthreads();
        v = 0.0;
        for (int w = 0; w < NT / 64; w++) v += lds[w];
    }
    return v;
}

template <int NT>
__device__ double row_max(double v, double *lds) {
    for (int off = 32; off; off >>= 1) v = fmax(v, __shfl_xor(v, off));
    if constexpr (NT > 64) {
        __syncthreads();
        if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
        __syncthreads();
        v = lds[0];
        for (int w = 1; w < NT / 64; w++) v = fmax(v, lds[w]);
    }
    return v;
}

// A row's teacher in LDS: places, p, and the student's logits there.
struct Teacher {
    int32_t *index;
    float *p, *student;
    double top, total;
    bool some;
};

size_t teacher_bytes(int k) { return ((size_t)k * 12 + 15) / 16 * 16; }

// A row's vocabulary as 16-byte vectors between a few single elements on either side.
template <typename T>
struct Row {
    static constexpr int V = 16 / sizeof(T);
    const T *at;
    int head, tail;
    int64_t vectors;
    __device__ Row(const void *base, int64_t row, int64_t ld, int64_t vocab) {
        at = (const T *)base + row * ld;
        const int off = (int)((16 - ((uintptr_t)at & 15)) & 15) / (int)sizeof(T);
        head = vocab < off ? (int)vocab : off;
        vectors = (vocab - head) / V;
        tail = (int)(vocab - head - vectors * V);
    }
    __device__ int64_t edge(int t) const { return t < head ? t : vectors * V + t; }  // the t-th single element
};

template <typename T, int NT, Mode MODE>
__global__ __launch_bounds__(NT == 64 ? 256 : NT) void distill_kernel(Args a) {
    extern __shared__ char lds_raw[];
    __shared__ double red[32];
    constexpr int V = 16 / sizeof(T), kRows = NT == 64 ? 4 : 1, kUnroll = 4;
    const int tid = threadIdx.x % NT, sub = threadIdx.x / NT;
    const double tau = a.temperature;
    const float c = (float)(1.0 / tau * 1.4426950408889634);
    Teacher t;
    char *mine = lds_raw + sub * (((size_t)a.k * 12 + 15) / 16 * 16);
    t.index = (int32_t *)mine, t.p = (float *)(t.index + a.k), t.student = t.p + a.k;
    for (int64_t row0 = (int64_t)blockIdx.x * kRows; row0 < a.rows; row0 += (int64_t)gridDim.x * kRows) {
        // a wave whose row lies behind the last works on the last one again and writes nothing
        const bool there = row0 + sub < a.rows;
        const int64_t row = there ? row0 + sub : a.rows - 1;
        const Row<T> r(a.logits, row, a.ld, a.vocab);
        __syncthreads();
        // teacher: softmax over the entries that are there
        double top = -INFINITY, total = 0.0;
        for (int j = tid; j < a.k; j += NT) {
            const int32_t i = a.index[row * a.teacher_ld + j];
            const double z = (double)a.teacher[row * a.teacher_ld + j] / tau;
            if (i >= 0 && i < a.vocab) top = fmax(top, z);
            t.index[j] = i < a.vocab ? i : -1;
            t.student[j] = i >= 0 && i < a.vocab ? (float)r.at[i] : 0.0f;
            if (i >= a.vocab || (i >= 0 && z != z)) total = NAN;
        }
        top = row_max<NT>(top, red);
        const double shift = top > -INFINITY ? top : 0.0;
        for (int j = tid; j < a.k; j += NT)
            if (t.index[j] >= 0) total += exp((double)a.teacher[row * a.teacher_ld + j] / tau - shift);
        total = row_sum<NT>(total, red);
        t.some = total > 0.0 || total != total;
        double m, log_sum;  // the student's log-sum-exp is m / tau + log_sum
        if constexpr (MODE != kGradient) {
            RunningSum s;
            if (tid < r.head + r.tail) {
                const float x[1] = {(float)r.at[r.edge(tid)]};
                s.add(x, c);
            }
            const Pack<T, V> *at = (const Pack<T, V> *)(r.at + r.head);
            int64_t i = tid;
            for (; i + (kUnroll - 1) * NT < r.vectors; i += kUnroll * NT) {
                Pack<T, V> v[kUnroll];
#pragma unroll
                for (int u = 0; u < kUnroll; u++) v[u] = at[i + u * NT];
#pragma unroll
                for (int u = 0; u < kUnroll; u++) {
                    float x[V];
#pragma unroll
                    for (int e = 0; e < V; e++) x[e] = (float)v[u].v[e];
                    s.add(x, c);
                }
            }
            for (; i < r.vectors; i += NT) {
                const Pack<T, V> v = at[i];
                float x[V];
#pragma unroll
                for (int e = 0; e < V; e++) x[e] = (float)v.v[e];
                s.add(x, c);
            }
            s = row_join<NT>(s, c, red);
            m = s.m, log_sum = log((double)s.s);
            double part = 0.0;
            for (int j = tid; j < a.k; j += NT) {
                const double p = t.index[j] < 0 ? 0.0 : exp((double)a.teacher[row * a.teacher_ld + j] / tau - shift) / total;
                t.p[j] = (float)p;
                if (p > 0.0) part += p * (log(p) - (((double)t.student[j] - m) / tau - log_sum));
                if (p != p) part = NAN;
            }
            part = row_sum<NT>(part, red);
            if (there && tid == 0) {
                a.loss[row] = t.some ? (total != total ? NAN : (float)(tau * tau * part)) : 0.0f;
                if (a.lse) a.lse[row] = (float)(m / tau + log_sum);
            }
        } else {
            m = 0.0, log_sum = a.lse[row];
            for (int j = tid; j < a.k; j += NT)
                t.p[j] = t.index[j] < 0 ? 0.0f : (float)(exp((double)a.teacher[row * a.teacher_ld + j] / tau - shift) / total);
        }
        if constexpr (MODE != kLoss) {
            // q is taken times 2^32 and the weight times 2^-32: the instruction's exp2 gives 0 below 2^-126, where
            // a product with the weight still has a value
            const float w = total != total ? NAN : a.temperature * a.dloss[row] * 0x1p-32f;
            const float m0 = (float)m, ls = (float)(log_sum * 1.4426950408889634) - 32.0f;
            auto q = [&](float x) { return __builtin_amdgcn_exp2f((x - m0) * c - ls); };
            T *out = (T *)a.dlogits + row * a.dlogits_ld;
            const bool pieces = (((uintptr_t)out ^ (uintptr_t)r.at) & 15) == 0;
            __syncthreads();  // the logits at the teacher's places are read: they may be written now
            if (there && tid < r.head + r.tail) {
                const int64_t e = r.edge(tid);
                out[e] = t.some ? round_to<T>(w * q((float)r.at[e])) : (T)0.0f;
            }
            const Pack<T, V> *at = (const Pack<T, V> *)(r.at + r.head);
            for (int64_t i = tid; there && i < r.vectors; i += NT) {
                const Pack<T, V> v = at[i];
                Pack<T, V> d;
#pragma unroll
                for (int e = 0; e < V; e++) d.v[e] = t.some ? round_to<T>(w * q((float)v.v[e])) : (T)0.0f;
                if (pieces) {
                    ((Pack<T, V> *)(out + r.head))[i] = d;
                } else {
#pragma unroll
                    for (int e = 0; e < V; e++) out[r.head + i * V + e] = d.v[e];
                }
            }
            __syncthreads();  // the dense part is written: the teacher's places again
            if (there && t.some)
                for (int j = tid; j < a.k; j += NT) {
                    const int32_t i = t.index[j];
                    if (i < 0) continue;
                    float p = 0.0f;
                    for (int l = 0; l < a.k; l++) p += t.index[l] == i ? t.p[l] : 0.0f;
                    out[i] = round_to<T>(w * (q(t.student[j]) - p * 0x1p32f));
                }
        }
    }
}

template <typename T, int NT, Mode MODE>
int launch_threads(const Args &a, hipStream_t s) {
    constexpr int rows = NT == 64 ? 4 : 1;
    const int64_t blocks = (a.rows + rows - 1) / rows;
    distill_kernel<T, NT, MODE><<<(unsigned)std::min(blocks, kMaxGrid), NT == 64 ? 256 : NT, rows * teacher_bytes(a.k), s>>>(a);
    BYZ_HIP(hipGetLastError());
    return BYZ_OK;
}

template <typename T, Mode MODE>
int launch_mode(const Args &a, hipStream_t s) {
    if (a.vocab * (int64_t)sizeof(T) <= 4096 && a.k <= 256) return launch_threads<T, 64, MODE>(a, s);
    if (a.vocab * (int64_t)sizeof(T) <= 32768) return launch_threads<T, 256, MODE>(a, s);
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

extern "C" size_t byz_distill_loss_workspace_bytes(int64_t rows, int64_t vocab, int k, int dtype) { return 0; }

extern "C" int byz_distill_loss(const void *logits, int64_t rows, int64_t vocab, int64_t ld, int dtype,
                                const float *teacher, const int32_t *index, int k, int64_t teacher_ld,
                                float temperature, float *loss, float *lse, void *workspace, size_t workspace_bytes,
                                void *stream) {
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
    return launch<kStep>(a, dtype, (hipStream_t)stream);
}

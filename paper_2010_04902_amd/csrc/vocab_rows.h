// Rows over a vocabulary, shared by the losses that take logits (not part of the C-ABI): their sums of exponentials, their vectors,
// and the gradient's softmax.
#ifndef BYZ_VOCAB_ROWS_H
#define BYZ_VOCAB_ROWS_H

#include "worker_internal.h"

namespace byz_worker {

// A sum of positive terms in fp32.  A vector's terms are added among themselves first, so that small ones are not lost one by one
// beside a large sum; the threads' sums are joined pairwise.  A thread's is off by 2^-24 of itself for each of its vectors at most, which
// are 98 for 200003 logits of 16 bits over 256 threads.  The loss has the logarithm.  In fp64 it would cost a conversion and an
// fp64 addition a value.
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
        float sum = __builtin_amdgcn_exp2f((x[0] - top) * c);
#pragma unroll
        for (int i = 1; i < N; i++) sum += __builtin_amdgcn_exp2f((x[i] - top) * c);
        s = fmaf(s, __builtin_amdgcn_exp2f((m - top) * c), sum), m = top;
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

// x - m for an x that was just unpacked.  FUSED: of fp16 as x 1 - m with a 1 that the compiler does not know, because a fused product takes
// a half from where it lies; the same number for an instruction less a value.  Where rows are held in registers that counts (policy
// step of 750 x 32000 17.8 us for 18.7), where they stream past it does not (distillation step of 8192 x 20000 173 us for 171).
template <typename T, bool FUSED>
__device__ __forceinline__ float less(float x, float m) {
    if constexpr (FUSED && std::is_same_v<T, f16>) {
        float one = 1.0f;
        asm("" : "+s"(one));
        return fmaf(x, one, -m);
    } else {
        return x - m;
    }
}

// q_v times a weight, from a logit.  The exponent is (x - m) c - l, with c = log2(e) / T in two parts where the result is fp32.
// The instruction's exp2 gives 0 below 2^-126, where a product with the weight still has a value: there the
// exponent is raised by 32 and the product lowered by it.
template <typename T, bool FUSED = false>
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
        const float d = byz_worker::less<T, FUSED>(x, m);
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

}  // namespace byz_worker

#endif

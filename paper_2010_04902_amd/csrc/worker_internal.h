// Shared by the operators of a worker's step (not part of the C-ABI): element types, vector loads and
// stores, activations, reductions in a fixed order.
#ifndef BYZ_WORKER_INTERNAL_H
#define BYZ_WORKER_INTERNAL_H

#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>
#include <type_traits>

#include "byz_internal.h"
#include "byzshield_worker.h"

#define BYZ_HIP(call)                              \
    do {                                           \
        hipError_t e_ = (call);                    \
        if (e_ != hipSuccess) {                    \
            byz_internal_set_hip_error((int)e_);   \
            return BYZ_EDEVICE;                    \
        }                                          \
    } while (0)

namespace byz_worker {

typedef _Float16 f16;
typedef __bf16 bf16;

inline size_t dtype_size(int dtype) { return dtype == BYZ_F32 ? 4 : 2; }
inline bool dtype_known(int dtype) { return dtype == BYZ_F32 || dtype == BYZ_BF16 || dtype == BYZ_F16; }
inline bool act_known(int act) { return act >= BYZ_ACT_NONE && act <= BYZ_ACT_SIGMOID; }

// V neighbouring values of type T as they lie in memory, loaded and stored in one piece.
template <typename T, int V>
struct alignas(sizeof(T) * V) Pack {
    T v[V];
};

// Stores a pack as one vector.  Assigned as a struct beside a branch that stores single elements, the compiler (ROCm 7.2) joins a
// store of each side to one and has lost the last element of packs in tiles that end early.
template <typename T, int V>
__device__ __forceinline__ void put(T *to, const Pack<T, V> &v) {
    typedef uint32_t words __attribute__((ext_vector_type(sizeof(T) * V / 4), may_alias));
    *(words *)to = __builtin_bit_cast(words, v);
}

// The same, held as 32-bit words: values of 16 bits that live over a loop or a barrier as such would take a register
// each.
typedef uint32_t __attribute__((may_alias)) word_t;
typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef f16 f16x2 __attribute__((ext_vector_type(2)));
typedef float floatx2 __attribute__((ext_vector_type(2)));

template <typename T, int V>
struct alignas(sizeof(T) * V) Words {
    static constexpr int N = sizeof(T) * V / 4;
    word_t w[N];
    __device__ __forceinline__ float operator[](int e) const {
        if constexpr (sizeof(T) == 4) {
            return __builtin_bit_cast(float, (uint32_t)w[e]);
        } else if constexpr (std::is_same_v<T, bf16>) {
            return __builtin_bit_cast(float, e % 2 ? (uint32_t)w[e / 2] & 0xffff0000u : (uint32_t)w[e / 2] << 16);
        } else {
            return (float)__builtin_bit_cast(f16x2, (uint32_t)w[e / 2])[e % 2];
        }
    }
    // the values f(0) .. f(V - 1), rounded to the nearest, ties to even
    template <typename F>
    static __device__ __forceinline__ Words of(F f) {
        Words r;
#pragma unroll
        for (int i = 0; i < N; i++) {
            if constexpr (sizeof(T) == 4) {
                r.w[i] = __builtin_bit_cast(uint32_t, (float)f(i));
            } else {
                const floatx2 x = {f(2 * i), f(2 * i + 1)};
                if constexpr (std::is_same_v<T, bf16>)
                    r.w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
                else
                    r.w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, f16x2));
            }
        }
        return r;
    }
    // The compiler takes what it has made of the words (values widened to fp32) for lost, and makes it again where it is used.
    __device__ __forceinline__ void keep() {
#pragma unroll
        for (int i = 0; i < N; i++) {
            uint32_t x = w[i];
            asm volatile("" : "+v"(x));
            w[i] = x;
        }
    }
};

template <typename T>
struct Words<T, 1> {
    T t;
    __device__ __forceinline__ float operator[](int) const { return (float)t; }
    template <typename F>
    static __device__ __forceinline__ Words of(F f) {
        return Words{(T)f(0)};
    }
    __device__ __forceinline__ void keep() {}
};

// Loaded and stored in one piece at any address of a T: the hardware takes vectors at an element's alignment, so which values
// a thread holds, and with it the order of sums, need not depend on where a tensor lies.
template <typename T, int V>
__device__ __forceinline__ Words<T, V> get_words(const T *from) {
    Words<T, V> v;
    __builtin_memcpy(&v, from, sizeof(v));
    return v;
}
template <typename T, int V>
__device__ __forceinline__ void put_words(T *to, const Words<T, V> &v) {
    __builtin_memcpy(to, &v, sizeof(v));
}

// Stored past the caches: for results larger than these, in whose place they keep the inputs, which are read again.
template <typename T, int V>
__device__ __forceinline__ void put_past_caches(T *to, const Words<T, V> &v) {
    if constexpr (sizeof(v) == 16) {
        typedef uint32_t words4 __attribute__((ext_vector_type(4), aligned(2), may_alias));
        __builtin_nontemporal_store(__builtin_bit_cast(words4, v), (words4 *)to);
    } else {
        put_words(to, v);
    }
}

// fp32 -> T, to the nearest, ties to even
template <typename T>
__device__ __forceinline__ T round_to(float x) {
    return (T)x;
}

__device__ __forceinline__ float sigmoidf(float z) { return __builtin_amdgcn_rcpf(1.0f + __expf(-z)); }

// The same number, of which the compiler knows nothing: what is computed from it is not kept over a loop, where the
// registers are wanted for other things.
__device__ __forceinline__ int afresh(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

// The normal distribution's upper tail at |z|, from e = exp(-z^2 / 2): the rational approximation 7.1.26 of
// Abramowitz and Stegun for erfc(|z| / sqrt 2) / 2, good to 7.5e-8.
__device__ __forceinline__ float normal_tail(float z, float e) {
    const float t = __builtin_amdgcn_rcpf(1.0f + 0.23164190f * fabsf(z));  // 0.3275911 / sqrt 2
    return ((((0.5307027145f * t - 0.7265760130f) * t + 0.7107068705f) * t - 0.1422483680f) * t + 0.1274147960f) * t * e;
}

template <int ACT>
__device__ __forceinline__ float act_value(float z) {
    if constexpr (ACT == BYZ_ACT_RELU) return z < 0.0f ? 0.0f : z;
    if constexpr (ACT == BYZ_ACT_SILU) return z * sigmoidf(z);
    if constexpr (ACT == BYZ_ACT_GELU) {
        const float tail = normal_tail(z, __expf(-0.5f * z * z));
        return z * (z < 0.0f ? tail : 1.0f - tail);
    }
    if constexpr (ACT == BYZ_ACT_SIGMOID) return sigmoidf(z);
    return z;
}

template <int ACT>
__device__ __forceinline__ float act_slope(float z) {
    if constexpr (ACT == BYZ_ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
    if constexpr (ACT == BYZ_ACT_SILU) {
        const float s = sigmoidf(z);
        return s * (1.0f + z * (1.0f - s));
    }
    if constexpr (ACT == BYZ_ACT_GELU) {
        const float e = __expf(-0.5f * z * z), tail = normal_tail(z, e);
        return (z < 0.0f ? tail : 1.0f - tail) + z * e * 0.39894228040143268f;
    }
    if constexpr (ACT == BYZ_ACT_SIGMOID) {
        const float s = sigmoidf(z);
        return s * (1.0f - s);
    }
    return 1.0f;
}

// Calls fn with the activation as a compile-time constant.
template <typename F>
__device__ __forceinline__ void with_act(int act, F fn) {
    switch (act) {
        case BYZ_ACT_RELU: fn(std::integral_constant<int, BYZ_ACT_RELU>{}); break;
        case BYZ_ACT_SILU: fn(std::integral_constant<int, BYZ_ACT_SILU>{}); break;
        case BYZ_ACT_GELU: fn(std::integral_constant<int, BYZ_ACT_GELU>{}); break;
        case BYZ_ACT_SIGMOID: fn(std::integral_constant<int, BYZ_ACT_SIGMOID>{}); break;
        default: fn(std::integral_constant<int, BYZ_ACT_NONE>{});
    }
}

// What a lane and the lane 2^STEP away (in the exclusive-or of their numbers) hold: a row of 16 lanes is turned by DPP, rows and
// halves are exchanged; a tenth of the latency of a shuffle through LDS.  Steps 2 and 3 turn the row by 4 and 8, which is the
// partner's value where the steps above have been taken.  Steps 4 and 5 give the lower lane's value first, others the lane's own.
template <int STEP, typename V>
__device__ __forceinline__ void wave_pair(const V &v, V &a, V &b) {
    static_assert(sizeof(V) % 4 == 0, "");
    struct Bits {
        uint32_t w[sizeof(V) / 4];
    };
    const Bits in = __builtin_bit_cast(Bits, v);
    Bits x = in, y;
#pragma unroll
    for (size_t i = 0; i < sizeof(V) / 4; i++) {
        if constexpr (STEP < 4) {
            constexpr int control[4] = {0xB1, 0x4E, 0x124, 0x128};  // lanes 1 0 3 2; 2 3 0 1; row turned by 4; by 8
            y.w[i] = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)in.w[i], control[STEP], 0xf, 0xf, true);
        } else {
            const auto r = STEP == 4 ? __builtin_amdgcn_permlane16_swap(in.w[i], in.w[i], false, false)
                                     : __builtin_amdgcn_permlane32_swap(in.w[i], in.w[i], false, false);
            x.w[i] = r[0], y.w[i] = r[1];
        }
    }
    a = __builtin_bit_cast(V, x), b = __builtin_bit_cast(V, y);
}

// fn(step) for the steps that join lanes `first` and more apart, first a power of two
template <typename F>
__device__ __forceinline__ void wave_steps(int first, F fn) {
    if (first <= 32) fn(std::integral_constant<int, 5>{});
    if (first <= 16) fn(std::integral_constant<int, 4>{});
    if (first <= 8) fn(std::integral_constant<int, 3>{});
    if (first <= 4) fn(std::integral_constant<int, 2>{});
    if (first <= 2) fn(std::integral_constant<int, 1>{});
    if (first <= 1) fn(std::integral_constant<int, 0>{});
}

// join(a, b) over the wave's lanes, for a join whose operands can be exchanged; every lane gets the same bits.
template <typename V, typename F>
__device__ __forceinline__ V wave_reduce(V v, F join) {
    wave_steps(1, [&](auto step) {
        V a, b;
        wave_pair<step.value>(v, a, b);
        v = join(a, b);
    });
    return v;
}

inline bool aligned(const void *p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

// first + (rows - 1) * pitch + width elements can be counted, and addressed with 64 bits
inline bool extent_ok(int64_t count, int64_t stride, int64_t more) {
    int64_t span;
    return stride >= 0 && more >= 0 && !__builtin_mul_overflow(count > 0 ? count - 1 : 0, stride, &span) &&
           !__builtin_add_overflow(span, more, &span) && span <= (INT64_MAX >> 4);
}

}  // namespace byz_worker

#endif

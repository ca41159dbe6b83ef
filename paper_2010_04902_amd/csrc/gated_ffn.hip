// Gated feed-forward block: both projections, activation and product in one kernel, and its gradients
// (gfx950, bf16 and fp16 with fp32 sums on the matrix cores).
//
// One tile kernel does all products.  Forward, the rows of B in a tile are half gate and half up weights of the same
// outputs, laid out so that a wave holds both sums of an output in the same lane and register: the epilogue needs no
// exchange.  Backward, one pass over dh and the saved sums writes dgate | dup, and
//     dx = dgate w_gate + dup w_up  is one product summed over 2n,   dw_gate = dgate^T x and dw_up = dup^T x  one launch.
// Operands whose summed index is not contiguous are turned by the loads from LDS, nothing is transposed in memory.
// The saved sums are fp32: rounded to bf16 they would be a third rounding on the way to a weight's gradient (2.9e-3
// off its 64-bit value instead of 2.35e-3; dgate's and the result's own are the others).
//
// Few tokens: the weights' bytes bound the call; a wave multiplies 16 rows of each weight with up to 16 tokens,
// straight from memory into the matrix instruction's registers, the waves of a block split k and join in LDS.
#include <algorithm>
#include <type_traits>

#include "worker_internal.h"

using namespace byz_worker;

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

template <typename T>
struct Frag;  // eight values of the summed index, an operand's share of a lane
template <>
struct Frag<bf16> {
    typedef bf16 type __attribute__((ext_vector_type(8)));
};
template <>
struct Frag<f16> {
    typedef f16 type __attribute__((ext_vector_type(8)));
};

__device__ __forceinline__ f32x16 mma32(Frag<bf16>::type a, Frag<bf16>::type b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma32(Frag<f16>::type a, Frag<f16>::type b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma16(Frag<bf16>::type a, Frag<bf16>::type b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma16(Frag<f16>::type a, Frag<f16>::type b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// C[i, j] = sum_k A[i, k] B[j, k].  An operand lies in memory either by rows of its outer index, k contiguous ("rows"),
// or by rows of k, the outer index contiguous ("columns"):
//   kForward  x by rows; tiles of B are half w_gate's rows, half w_up's of the same outputs (k: the input width)
//   kInput    dx: [dgate | dup] by rows; w_gate's rows then w_up's are the summed index: by columns
//   kWeight   dw_gate, dw_up: both operands by columns, summed over the tokens
enum Kind { kForward, kInput, kWeight };

struct Product {
    const void *a, *b, *b2;
    int64_t a_ld, b_ld;
    int64_t m, n, k;         // outputs m x n (kForward: n of each weight); summed index
    int64_t a_outer, b_outer;  // outer indices that can be read: rows, or columns in whole pieces of eight
    int64_t turn;            // kInput: summed index where w_up starts; kWeight: columns of a where dup starts
    void *out, *out2;        // kWeight: out2 is dw_up
    int64_t out_ld;
    float *gate, *up;        // kForward: saved sums
    int64_t gate_ld;
    int act;
    int tiles_m, tiles_n;
    bool direct;             // whole steps go from memory to LDS without registers
};

// A step of the sum is 32 values of k.  In LDS an operand by rows has 64 bytes a row, in four 16-byte pieces; by columns 32
// rows (of k) of a tile's width.  A wave's load instruction fills 1024 bytes in lane order, so pieces are exchanged on
// the way by the global addresses: without that, lanes that read one piece of 16 rows, or four rows of k, would meet
// in the same banks.
constexpr int kStep = 32;

template <int WIDTH>
__device__ __forceinline__ int row_piece(int row, int piece) {  // by rows: byte of a piece
    return row * 64 + ((piece ^ ((row >> 2) & 3)) * 16);
}
template <int WIDTH>
__device__ __forceinline__ int column_turn(int row) {  // by columns: what the 64-byte slots of a row of k are exchanged by
    return WIDTH >= 128 ? row & 3 : (row >> 1) & 1;
}

// 1024 bytes from memory to LDS without registers: lane i's 16 bytes at `from` go to lds + 16 i.  Written out
// because the compiler, where it sees such a load, lets every turned read from LDS wait for all of them.  It has no
// output register, so nothing of the compiler's can meet it in flight; vmcnt counts it, which makes the compiler's own
// waits only longer.  Nothing else here uses m0.
__device__ __forceinline__ void load_to_lds(const void *from, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                 :
                 : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(from)
                 : "memory");
}

// One operand's tile of WIDTH outer indices.
template <typename T, int WIDTH, bool COLUMNS>
struct Side {
    using frag = typename Frag<T>::type;
    static constexpr int kBytes = WIDTH * 64, kChunks = WIDTH / 16;

    // Byte offset from the tile's corner of what lane `lane` of chunk `chunk` loads.  `outer`: outer indices from
    // the corner on; rows and pieces past the end load the last, and their products are not stored.
    static __device__ __forceinline__ uint32_t offset(int chunk, int lane, int64_t outer, int64_t ld) {
        if constexpr (COLUMNS) {
            constexpr int pieces = WIDTH / 8, rows = 64 / pieces;
            const int row = chunk * rows + lane / pieces, at = lane % pieces;
            const int piece = (((at >> 2) ^ column_turn<WIDTH>(row)) << 2) | (at & 3);
            return (uint32_t)((row * ld + std::min<int64_t>(piece * 8, outer - 8)) * sizeof(T));
        }
        const int row = chunk * 16 + lane / 4, piece = (lane % 4) ^ ((row >> 2) & 3);
        return (uint32_t)((std::min<int64_t>(row, outer - 1) * ld + piece * 8) * sizeof(T));
    }

    // One 16-byte piece through registers, zeros from `ks` values of k on.  `at`: the step's corner.
    static __device__ __forceinline__ void copy_piece(const T *at, int64_t ld, int64_t outer, int64_t ks, int number, char *lds) {
        frag v = {};
        if constexpr (COLUMNS) {
            constexpr int pieces = WIDTH / 8;
            const int row = number / pieces, piece = number % pieces;
            if (row < ks) v = *(const frag *)(at + row * ld + std::min<int64_t>(piece * 8, outer - 8));
            *(frag *)(lds + row * WIDTH * 2 + (((piece >> 2) ^ column_turn<WIDTH>(row)) << 6) + (piece & 3) * 16) = v;
        } else {
            const int row = number / 4, piece = number % 4;
            if (piece * 8 < ks) v = *(const frag *)(at + std::min<int64_t>(row, outer - 1) * ld + piece * 8);
            *(frag *)(lds + row_piece<WIDTH>(row, piece)) = v;
        }
    }

    // Byte of this lane's first piece of the fragment of 32 outer indices that starts at `first`.
    static __device__ __forceinline__ int fragment(int first, int lane) {
        if constexpr (COLUMNS) {
            const int q = lane % 16 / 4;  // the row of four that the lane reads for its group of 16
            return (lane / 32 * 8 + q) * WIDTH * 2 + (((first / 32) ^ column_turn<WIDTH>(q)) << 6) + lane / 16 % 2 * 32 + lane % 4 * 8;
        }
        return row_piece<WIDTH>(first + lane % 32, lane / 32);
    }

    // Values 16 half .. 16 half + 15 of the step: lane l has outer index l % 32 and k = 8 (l / 32) .. + 7.
    static __device__ __forceinline__ frag read(const char *lds, int at, int half) {
        if constexpr (COLUMNS) {
            // four rows of k, 16 outer indices, turned by the load: a lane gets its index's four values
            typedef short s4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s4 *ptr;
            struct {
                s4 v[2];
            } two;
#pragma unroll
            for (int i = 0; i < 2; i++) two.v[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ptr)(lds + at + (half * 16 + i * 4) * WIDTH * 2));
            return __builtin_bit_cast(frag, two);
        }
        return *(const frag *)(lds + (at ^ (half * 32)));
    }
};

template <typename T, int BM, int BN, int WM, int WN, Kind KIND, int STAGES>
__global__ __launch_bounds__(WM * WN * 64) void product_kernel(Product p) {
    using frag = typename Frag<T>::type;
    using A = Side<T, BM, KIND == kWeight>;
    using B = Side<T, KIND == kForward ? BN / 2 : BN, KIND != kForward>;  // kForward: two sides, w_gate's and w_up's
    constexpr int kWaves = WM * WN, FM = BM / WM / 32, FN = BN / WN / 32, kBytes = (BM + BN) * 64;
    constexpr int kLoads = (BM + BN) / 16 / kWaves, kOut = KIND == kForward ? BN / 2 : BN;
    static_assert((BM + BN) / 16 % kWaves == 0 && STAGES >= 3, "");
    extern __shared__ char lds[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, wm = wave / WN, wn = wave % WN;
    int tile = blockIdx.x;
    const T *a = (const T *)p.a;
    T *out = (T *)p.out;
    if (KIND == kWeight && tile >= p.tiles_m * p.tiles_n) {
        tile -= p.tiles_m * p.tiles_n;
        a += p.turn;
        out = (T *)p.out2;
    }
    const int64_t m0 = (int64_t)(tile % p.tiles_m) * BM, n0 = (int64_t)(tile / p.tiles_m) * kOut;
    // corners of the tile's sides in memory, and what a step moves them by
    const T *corner_a = KIND == kWeight ? a + m0 : a + m0 * p.a_ld;
    const T *corner_b = KIND == kForward ? (const T *)p.b + n0 * p.b_ld : (const T *)p.b + n0;
    const T *corner_b2 = KIND == kForward ? (const T *)p.b2 + n0 * p.b_ld : KIND == kInput ? (const T *)p.b2 + n0 : nullptr;
    const int64_t move_a = KIND == kWeight ? kStep * p.a_ld : kStep, move_b = KIND == kForward ? kStep : kStep * p.b_ld;
    const int64_t outer_a = p.a_outer - m0, outer_b = p.b_outer - n0;

    uint32_t offset[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; i++) {
        const int chunk = i * kWaves + wave;
        offset[i] = chunk < A::kChunks ? A::offset(chunk, lane, outer_a, p.a_ld)
                                       : B::offset((chunk - A::kChunks) % B::kChunks, lane, outer_b, p.b_ld);
    }
    // kInput: steps of w_gate, then of w_up; `turn` is a multiple of the step
    const int steps = (int)((p.k + kStep - 1) / kStep), turn = KIND == kInput ? (int)(p.turn / kStep) : steps;
    auto corner_of_b = [&](int t) { return KIND == kInput && t >= turn ? corner_b2 + (t - turn) * move_b : corner_b + t * move_b; };
    // values of k that step t has
    auto values = [&](int t) -> int64_t {
        if (KIND == kInput) return std::min<int64_t>(kStep, std::max<int64_t>(0, p.k - p.turn - (int64_t)(t >= turn ? t - turn : t) * kStep));
        return std::min<int64_t>(kStep, p.k - (int64_t)t * kStep);
    };
    // whole steps from memory to LDS without registers
    const int whole = !p.direct ? 0 : (int)((KIND == kInput ? p.k - p.turn : p.k) / kStep);
    auto is_direct = [&](int t) { return t < steps && (t >= turn ? t - turn : t) < whole; };
    const uint32_t lds_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
    auto load_direct = [&](int t) {
        const T *at_a = corner_a + t * move_a, *at_b = corner_of_b(t), *at_b2 = corner_b2 + (KIND == kForward ? t * move_b : 0);
        const uint32_t to = lds_at + t % STAGES * kBytes;
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const int chunk = i * kWaves + wave;
            const T *at = chunk < A::kChunks ? at_a : KIND == kForward && chunk >= A::kChunks + B::kChunks ? at_b2 : at_b;
            load_to_lds((const char *)at + offset[i], to + chunk * 1024);
        }
    };
    auto load = [&](int t) {
        if (is_direct(t)) {
            load_direct(t);
        } else if (t < steps) {
            const T *at_a = corner_a + t * move_a, *at_b = corner_of_b(t);
            char *to = lds + t % STAGES * kBytes;
            const int64_t ks = values(t);
            for (int i = threadIdx.x; i < BM * 4; i += kWaves * 64) A::copy_piece(at_a, p.a_ld, outer_a, ks, i, to);
            for (int i = threadIdx.x; i < BN * 4; i += kWaves * 64) {
                const bool second = KIND == kForward && i >= BN * 2;
                B::copy_piece(second ? corner_b2 + t * move_b : at_b, p.b_ld, outer_b, ks, second ? i - BN * 2 : i,
                              to + BM * 64 + (second ? BN * 32 : 0));
            }
        }
    };
    int place_a[FM], place_b[FN];
#pragma unroll
    for (int i = 0; i < FM; i++) place_a[i] = A::fragment((wm * FM + i) * 32, lane);
#pragma unroll
    for (int j = 0; j < FN; j++)
        place_b[j] = BM * 64 + (KIND == kForward ? j % 2 * (BN * 32) + B::fragment((wn * (FN / 2) + j / 2) * 32, lane)
                                                 : B::fragment((wn * FN + j) * 32, lane));
    auto read = [&](frag(&fa)[FM], frag(&fb)[FN], int t, int half) {
        const char *at = lds + t % STAGES * kBytes;
#pragma unroll
        for (int i = 0; i < FM; i++) fa[i] = A::read(at, place_a[i], half);
#pragma unroll
        for (int j = 0; j < FN; j++) fb[j] = B::read(at, place_b[j], half);
    };
    f32x16 acc[FM][FN] = {};
    auto multiply = [&](frag(&fa)[FM], frag(&fb)[FN]) {
#pragma unroll
        for (int i = 0; i < FM; i++)
#pragma unroll
            for (int j = 0; j < FN; j++) acc[i][j] = mma32(fa[i], fb[j], acc[i][j]);
    };
    // Steps t + 1 .. t + STAGES - 1 are on their way while step t is multiplied, and fragments are read half a step ahead:
    // two sets of registers.  Before half a step is multiplied, the reads that its fragments came by are
    // waited for; before the second half also step t + 1's loads, then a barrier: step t + 1 is there for
    // everybody, and everybody has read step t - 1, whose place the next load takes.
    auto barrier = [&] {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    frag a0[FM], b0[FN], a1[FM], b1[FN];
    auto step = [&](int t, auto fast) {  // fast: steps t + 2 .. t + STAGES - 1 are there and direct
        __builtin_amdgcn_s_waitcnt(0xC07F);  // lgkmcnt(0)
        __builtin_amdgcn_sched_barrier(0);
        read(a1, b1, t, 1);
        __builtin_amdgcn_sched_barrier(0);
        multiply(a0, b0);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0xC07F);
        if constexpr (fast.value)
            asm volatile("s_waitcnt vmcnt(%0)" : : "n"((STAGES - 3) * kLoads) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
        barrier();
        if constexpr (fast.value) {
            load_direct(t + STAGES - 1);
            read(a0, b0, t + 1, 0);
        } else {
            load(t + STAGES - 1);
            if (t + 1 < steps) read(a0, b0, t + 1, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
        multiply(a1, b1);
        __builtin_amdgcn_sched_barrier(0);
    };
    // end of the fast steps that t is among
    auto fast_end = [&](int t) {
        if (KIND == kInput && whole == turn) return 2 * whole - (STAGES - 1);
        return (KIND == kInput && t + 2 >= turn ? turn : 0) + whole - (STAGES - 1);
    };
    if (steps > 0) {
        for (int t = 0; t < STAGES - 1; t++) load(t);
        __builtin_amdgcn_s_waitcnt(0xC07F);
        if (whole >= STAGES - 1)
            asm volatile("s_waitcnt vmcnt(%0)" : : "n"((STAGES - 2) * kLoads) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
        barrier();
        read(a0, b0, 0, 0);
        for (int t = 0; t < steps;) {
            for (const int end = fast_end(t); t < end; t++) step(t, std::true_type{});
            if (t < steps) step(t++, std::false_type{});
        }
    }
    // a lane holds one column and, of a fragment, rows 8 * (r / 4) + 4 * (lane / 32) + r % 4
    auto each = [&](auto fn) {
#pragma unroll
        for (int i = 0; i < FM; i++)
#pragma unroll
            for (int r = 0; r < 16; r++) {
                const int64_t row = m0 + (wm * FM + i) * 32 + (r / 4) * 8 + (lane / 32) * 4 + r % 4;
                if (row < p.m) fn(i, r, row);
            }
    };
    if constexpr (KIND == kForward) {
        with_act(p.act, [&](auto act) {
            each([&](int i, int r, int64_t row) {
#pragma unroll
                for (int j = 0; j < FN; j += 2) {
                    const int64_t col = n0 + (wn * (FN / 2) + j / 2) * 32 + lane % 32;
                    if (col >= p.n) continue;
                    const float g = acc[i][j][r], u = acc[i][j + 1][r];
                    out[row * p.out_ld + col] = round_to<T>(act_value<act.value>(g) * u);
                    if (p.gate) {
                        p.gate[row * p.gate_ld + col] = g;
                        p.up[row * p.gate_ld + col] = u;
                    }
                }
            });
        });
    } else {
        each([&](int i, int r, int64_t row) {
#pragma unroll
            for (int j = 0; j < FN; j++) {
                const int64_t col = n0 + (wn * FN + j) * 32 + lane % 32;
                if (col < p.n) out[row * p.out_ld + col] = round_to<T>(acc[i][j][r]);
            }
        });
    }
}

// Up to 16 tokens.  Block: 16 outputs, kSkinnyWaves shares of k.
constexpr int kSkinnyWaves = 8;
template <typename T>
__global__ __launch_bounds__(kSkinnyWaves * 64) void skinny_kernel(Product p) {
    using frag = typename Frag<T>::type;
    __shared__ f32x4 part[2][kSkinnyWaves][64];
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64;
    const int64_t n0 = (int64_t)blockIdx.x * 16, n = std::min<int64_t>(n0 + lane % 16, p.n - 1);
    const T *g = (const T *)p.b + n * p.b_ld, *u = (const T *)p.b2 + n * p.b_ld;
    const bool token = lane % 16 < p.m;
    const T *x = (const T *)p.a + (token ? lane % 16 : 0) * p.a_ld;
    f32x4 accg = {}, accu = {};
    auto piece = [&](const T *src, int64_t k) {
        frag v;
        if (p.direct && k + 8 <= p.k) {
            v = *(const frag *)(src + k);
        } else {
#pragma unroll
            for (int e = 0; e < 8; e++) v[e] = k + e < p.k ? src[k + e] : (T)0.0f;
        }
        return v;
    };
    // steps of 32 values, dealt to the waves in turn
    for (int64_t k0 = wave * 32; k0 < p.k; k0 += kSkinnyWaves * 32) {
        const int64_t k = k0 + lane / 16 * 8;
        frag a = piece(x, k), bg = piece(g, k), bu = piece(u, k);
        if (!token) a = frag{};
        accg = mma16(a, bg, accg);
        accu = mma16(a, bu, accu);
    }
    part[0][wave][lane] = accg, part[1][wave][lane] = accu;
    __syncthreads();
    if (wave == 0) {
        for (int w = 1; w < kSkinnyWaves; w++) accg += part[0][w][lane], accu += part[1][w][lane];
        const int64_t col = n0 + lane % 16;
        with_act(p.act, [&](auto act) {
#pragma unroll
            for (int r = 0; r < 4; r++) {
                const int64_t row = lane / 16 * 4 + r;
                if (row >= p.m || col >= p.n) continue;
                ((T *)p.out)[row * p.out_ld + col] = round_to<T>(act_value<act.value>(accg[r]) * accu[r]);
                if (p.gate) {
                    p.gate[row * p.gate_ld + col] = accg[r];
                    p.up[row * p.gate_ld + col] = accu[r];
                }
            }
        });
    }
}

// dgate | dup from dh, gate and up: `d` is [m][2 np] (dgate, then dup), zeros in the padding.
struct Slopes {
    const void *dh;
    const float *gate, *up;
    int64_t dh_ld, gate_ld, m, n, np;
    void *d;
    int act;
};

// Four values a thread, rows of np / 4 threads.
template <typename T, bool WIDE>
__global__ __launch_bounds__(256) void slopes_kernel(Slopes s) {
    const int64_t across = s.np / 4, all = s.m * across;
    with_act(s.act, [&](auto act) {
        for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < all; at += (int64_t)gridDim.x * 256) {
            const int64_t i = at / across, j = (at - i * across) * 4;
            const T *dh = (const T *)s.dh + i * s.dh_ld + j;
            const float *gate = s.gate + i * s.gate_ld + j, *up = s.up + i * s.gate_ld + j;
            Pack<T, 4> h, dg, du;
            Pack<float, 4> g, u;
            if (WIDE && j + 4 <= s.n) {
                h = *(const Pack<T, 4> *)dh;
                g = *(const Pack<float, 4> *)gate;
                u = *(const Pack<float, 4> *)up;
            } else {
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const bool in = j + e < s.n;
                    h.v[e] = in ? dh[e] : (T)0.0f;
                    g.v[e] = in ? gate[e] : 0.0f;
                    u.v[e] = in ? up[e] : 0.0f;
                }
            }
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const float d = (float)h.v[e];
                dg.v[e] = round_to<T>(d * u.v[e] * act_slope<act.value>(g.v[e]));
                du.v[e] = round_to<T>(d * act_value<act.value>(g.v[e]));
            }
            *(Pack<T, 4> *)((T *)s.d + i * 2 * s.np + j) = dg;
            *(Pack<T, 4> *)((T *)s.d + i * 2 * s.np + s.np + j) = du;
        }
    });
}

// A matrix whose rows do not start at 16-byte boundaries, copied to rows of `out_ld`, zeros behind its columns.
template <typename T>
__global__ __launch_bounds__(256) void align_kernel(const T *in, int64_t in_ld, int64_t rows, int64_t cols, T *out, int64_t out_ld) {
    const int64_t across = out_ld / 8, all = rows * across;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < all; at += (int64_t)gridDim.x * 256) {
        const int64_t i = at / across, j = (at - i * across) * 8;
        Pack<T, 8> v;
#pragma unroll
        for (int e = 0; e < 8; e++) v.v[e] = j + e < cols ? in[i * in_ld + j + e] : (T)0.0f;
        *(Pack<T, 8> *)(out + i * out_ld + j) = v;
    }
}

unsigned grid_of(int64_t threads) { return (unsigned)std::min<int64_t>((threads + 255) / 256, 8192); }

template <typename T, int BM, int BN, int WM, int WN, Kind KIND, int STAGES>
int launch_tile(Product p, hipStream_t s) {
    constexpr int kOut = KIND == kForward ? BN / 2 : BN, kThreads = WM * WN * 64, kLds = STAGES * (BM + BN) * 64;
    const int64_t tm = (p.m + BM - 1) / BM, tn = (p.n + kOut - 1) / kOut, blocks = tm * tn * (KIND == kWeight ? 2 : 1);
    if (blocks > INT32_MAX / kThreads) return BYZ_EUNSUPPORTED;
    p.tiles_m = (int)tm, p.tiles_n = (int)tn;
    // a lane's place in a tile's side is a 32-bit offset
    const int64_t most = INT32_MAX / (int64_t)sizeof(T);
    p.direct = (KIND == kWeight ? kStep : BM) * p.a_ld + BM < most && (KIND == kForward ? BN : kStep) * p.b_ld + BN < most;
    auto *kernel = &product_kernel<T, BM, BN, WM, WN, KIND, STAGES>;
    BYZ_HIP(hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kLds));
    kernel<<<(unsigned)blocks, kThreads, kLds, s>>>(p);
    BYZ_HIP(hipGetLastError());
    return BYZ_OK;
}

// Operands' rows start at 16-byte boundaries and have whole 16-byte pieces.
template <typename T, Kind KIND>
int launch_product(const Product &p, hipStream_t s) {
    const int64_t across = KIND == kInput ? p.n : 2 * p.n;
    auto tiles = [&](int bm, int bn) { return ((p.m + bm - 1) / bm) * ((across + bn - 1) / bn); };
    if (tiles(256, 256) >= 192) return launch_tile<T, 256, 256, 2, 4, KIND, 4>(p, s);
    if (tiles(128, 128) >= 192) return launch_tile<T, 128, 128, 2, 2, KIND, 4>(p, s);
    return launch_tile<T, 64, 128, 2, 2, KIND, 4>(p, s);
}

int64_t padded(int64_t v) { return (v + 63) / 64 * 64; }

bool sizes_ok(int64_t m, int64_t k, int64_t n) {
    const int64_t most = (int64_t)1 << 31;
    return m >= 0 && k >= 0 && n >= 0 && m < most && k < most && n < most;
}

// Whether the tile kernel reads a matrix as it lies: pieces of 16 bytes, none of them beyond the columns.
bool pieces(const void *at, int64_t cols, int64_t ld) { return aligned(at, 16) && cols % 8 == 0 && ld % 8 == 0; }

// Workspace, in elements: matrices that have to be copied, and for the backward pass dgate | dup.
struct Layout {
    int64_t np, kp;
    int64_t x, w, d, all;
    Layout(int64_t m, int64_t k, int64_t n, bool backward) : np(padded(n)), kp((k + 7) / 8 * 8) {
        x = 0;
        w = x + m * kp;
        d = w + 2 * n * kp;
        all = d + (backward ? m * 2 * np : 0);
    }
};

constexpr int kSkinny = 16;  // most tokens of the kernel for few

struct Call {
    const void *x, *w_gate, *w_up;
    int64_t x_ld, w_ld, m, k, n;
    int act;
    void *ws;
};

template <typename T>
int align(const void **at, int64_t *ld, int64_t rows, int64_t cols, T *to, int64_t to_ld, hipStream_t s) {
    align_kernel<T><<<grid_of(rows * (to_ld / 8)), 256, 0, s>>>((const T *)*at, *ld, rows, cols, to, to_ld);
    BYZ_HIP(hipGetLastError());
    *at = to, *ld = to_ld;
    return BYZ_OK;
}

// Copies x and the weights where the tile kernel cannot read them: rows of whole pieces, zeros behind k.
template <typename T>
int align_operands(Call &c, const Layout &lay, bool x, bool w, hipStream_t s) {
    const bool good_x = !x || c.m == 0 || pieces(c.x, c.k, c.x_ld);
    const bool good_w = !w || c.n == 0 || (pieces(c.w_gate, c.k, c.w_ld) && pieces(c.w_up, c.k, c.w_ld));
    if (c.k == 0 || (good_x && good_w)) return BYZ_OK;
    T *ws = (T *)c.ws;
    int rc = BYZ_OK;
    if (!good_x) rc = align<T>(&c.x, &c.x_ld, c.m, c.k, ws + lay.x, lay.kp, s);
    if (rc == BYZ_OK && !good_w) {
        int64_t ld = c.w_ld;
        rc = align<T>(&c.w_gate, &ld, c.n, c.k, ws + lay.w, lay.kp, s);
        if (rc == BYZ_OK) rc = align<T>(&c.w_up, &c.w_ld, c.n, c.k, ws + lay.w + c.n * lay.kp, lay.kp, s);
    }
    return rc;
}

size_t forward_bytes(const Call &c) {
    const bool good = pieces(c.x, c.k, c.x_ld) && pieces(c.w_gate, c.k, c.w_ld) && pieces(c.w_up, c.k, c.w_ld);
    return c.m <= kSkinny || good ? 0 : (size_t)Layout(c.m, c.k, c.n, false).all * 2;
}

template <typename T>
int forward(Call c, Product p, hipStream_t s) {
    if (c.m > kSkinny) {
        const int rc = align_operands<T>(c, Layout(c.m, c.k, c.n, false), true, true, s);
        if (rc != BYZ_OK) return rc;
    }
    p.a = c.x, p.a_ld = c.x_ld, p.b = c.w_gate, p.b2 = c.w_up, p.b_ld = c.w_ld;
    p.m = c.m, p.n = c.n, p.k = c.k, p.act = c.act;
    if (c.m > kSkinny) {
        p.k = (p.k + 7) / 8 * 8, p.a_outer = p.m, p.b_outer = p.n;
        return launch_product<T, kForward>(p, s);
    }
    p.direct = pieces(c.x, 8, c.x_ld) && pieces(c.w_gate, 8, c.w_ld) && pieces(c.w_up, 8, c.w_ld);
    skinny_kernel<T><<<(unsigned)((p.n + 15) / 16), kSkinnyWaves * 64, 0, s>>>(p);
    BYZ_HIP(hipGetLastError());
    return BYZ_OK;
}

struct Gradients {
    const void *dh;
    const float *gate, *up;
    int64_t dh_ld, gate_ld;
    void *dx, *dw_gate, *dw_up;
    int64_t dx_ld, dw_ld;
};

template <typename T>
int backward(Call c, const Gradients &g, hipStream_t s) {
    const Layout lay(c.m, c.k, c.n, true);
    T *d = (T *)c.ws + lay.d;
    const int64_t cols = c.k;
    const bool dx = g.dx && c.m > 0 && c.k > 0, dw = g.dw_gate && c.n > 0 && c.k > 0;
    if (c.m > 0 && c.n > 0) {
        const Slopes v{g.dh, g.gate, g.up, g.dh_ld, g.gate_ld, c.m, c.n, lay.np, d, c.act};
        const bool wide = aligned(g.dh, 8) && g.dh_ld % 4 == 0 && aligned(g.gate, 16) && aligned(g.up, 16) && g.gate_ld % 4 == 0;
        const unsigned grid = grid_of(c.m * (lay.np / 4));
        if (wide)
            slopes_kernel<T, true><<<grid, 256, 0, s>>>(v);
        else
            slopes_kernel<T, false><<<grid, 256, 0, s>>>(v);
        BYZ_HIP(hipGetLastError());
    }
    int rc = align_operands<T>(c, lay, dw, dx, s);
    if (rc == BYZ_OK && dx) {
        Product p{};
        p.a = d, p.a_ld = 2 * lay.np, p.b = c.w_gate, p.b2 = c.w_up, p.b_ld = c.w_ld;
        p.m = c.m, p.n = cols, p.turn = lay.np, p.k = lay.np + c.n, p.out = g.dx, p.out_ld = g.dx_ld;
        p.a_outer = c.m, p.b_outer = lay.kp;
        rc = launch_product<T, kInput>(p, s);
    }
    if (rc == BYZ_OK && dw) {
        Product p{};
        p.a = d, p.a_ld = 2 * lay.np, p.turn = lay.np, p.b = c.x, p.b_ld = c.x_ld;
        p.m = c.n, p.n = cols, p.k = c.m, p.out = g.dw_gate, p.out2 = g.dw_up, p.out_ld = g.dw_ld;
        p.a_outer = lay.np, p.b_outer = lay.kp;
        rc = launch_product<T, kWeight>(p, s);
    }
    return rc;
}

bool matrix_ok(const void *at, int64_t rows, int64_t cols, int64_t ld, int elem = 2) {
    return rows == 0 || cols == 0 || (at && aligned(at, elem) && ld >= cols && extent_ok(rows, ld, cols));
}

}  // namespace

extern "C" size_t byz_gated_ffn_workspace_bytes(int64_t m, int64_t k, int64_t n, int dtype) {
    if (!sizes_ok(m, k, n) || (dtype != BYZ_BF16 && dtype != BYZ_F16) || m <= kSkinny) return 0;
    return (size_t)Layout(m, k, n, false).all * 2;
}

extern "C" int byz_gated_ffn(const void *x, int64_t x_ld, const void *w_gate, const void *w_up, int64_t w_ld,
                             int64_t m, int64_t k, int64_t n, int dtype, int act, void *h, int64_t h_ld,
                             float *gate_out, float *up_out, int64_t gate_ld, void *workspace, size_t workspace_bytes,
                             void *stream) {
    if (!sizes_ok(m, k, n) || !dtype_known(dtype) || !act_known(act) || !gate_out != !up_out) return BYZ_EINVAL;
    if (dtype == BYZ_F32) return BYZ_EUNSUPPORTED;
    if (!matrix_ok(x, m, k, x_ld) || !matrix_ok(w_gate, n, k, w_ld) || !matrix_ok(w_up, n, k, w_ld) || !matrix_ok(h, m, n, h_ld) ||
        (gate_out && (!matrix_ok(gate_out, m, n, gate_ld, 4) || !matrix_ok(up_out, m, n, gate_ld, 4))))
        return BYZ_EINVAL;
    if (m == 0 || n == 0) return BYZ_OK;
    const Call c{x, w_gate, w_up, x_ld, w_ld, m, k, n, act, workspace};
    const size_t need = forward_bytes(c);
    if (need && (!workspace || !aligned(workspace, 16) || workspace_bytes < need)) return BYZ_ENOMEM;
    Product p{};
    p.out = h, p.out_ld = h_ld, p.gate = gate_out, p.up = up_out, p.gate_ld = gate_ld;
    return dtype == BYZ_BF16 ? forward<bf16>(c, p, (hipStream_t)stream) : forward<f16>(c, p, (hipStream_t)stream);
}

extern "C" size_t byz_gated_ffn_backward_workspace_bytes(int64_t m, int64_t k, int64_t n, int dtype) {
    if (!sizes_ok(m, k, n) || (dtype != BYZ_BF16 && dtype != BYZ_F16)) return 0;
    return (size_t)Layout(m, k, n, true).all * 2;
}

extern "C" int byz_gated_ffn_backward(const void *dh, int64_t dh_ld, const void *x, int64_t x_ld, const void *w_gate,
                                      const void *w_up, int64_t w_ld, const float *gate, const float *up,
                                      int64_t gate_ld, int64_t m, int64_t k, int64_t n, int dtype, int act, void *dx,
                                      int64_t dx_ld, void *dw_gate, void *dw_up, int64_t dw_ld, void *workspace,
                                      size_t workspace_bytes, void *stream) {
    if (!sizes_ok(m, k, n) || !dtype_known(dtype) || !act_known(act) || !dw_gate != !dw_up) return BYZ_EINVAL;
    if (dtype == BYZ_F32) return BYZ_EUNSUPPORTED;
    if (!matrix_ok(dh, m, n, dh_ld) || !matrix_ok(gate, m, n, gate_ld, 4) || !matrix_ok(up, m, n, gate_ld, 4) ||
        (dx && (!matrix_ok(w_gate, n, k, w_ld) || !matrix_ok(w_up, n, k, w_ld) || !matrix_ok(dx, m, k, dx_ld))) ||
        (dw_gate && (!matrix_ok(x, m, k, x_ld) || !matrix_ok(dw_gate, n, k, dw_ld) || !matrix_ok(dw_up, n, k, dw_ld))))
        return BYZ_EINVAL;
    const size_t need = (size_t)Layout(m, k, n, true).all * 2;
    if (workspace_bytes < need || (need && (!workspace || !aligned(workspace, 16)))) return BYZ_ENOMEM;
    const Call c{x, w_gate, w_up, x_ld, w_ld, m, k, n, act, workspace};
    const Gradients g{dh, gate, up, dh_ld, gate_ld, dx, dw_gate, dw_up, dx_ld, dw_ld};
    return dtype == BYZ_BF16 ? backward<bf16>(c, g, (hipStream_t)stream) : backward<f16>(c, g, (hipStream_t)stream);
}

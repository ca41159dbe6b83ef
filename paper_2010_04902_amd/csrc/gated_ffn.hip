// Gated feed-forward block: both projections, activation and product in one kernel, and its gradients
// (gfx950, bf16 and fp16 with fp32 sums on the matrix cores).
//
// One tile kernel does all products.  Forward, the rows of B in a tile are half gate and half up weights of the same
// outputs, laid out so that a wave holds both sums of an output in the same lane and register: the epilogue needs no
// exchange.  Backward, one pass over dh and the saved sums writes dgate | dup, and
//     dx = dgate w_gate + dup w_up  is one product summed over 2n,   dw_gate = dgate^T x and dw_up = dup^T x  one launch.
// dx of few tokens has few tiles and a long sum: blocks share it and a kernel adds their sums in order (us of the backward pass
// without / with that: 40 x 4096 x 10944 198 / 111, 64 x 1024 x 2752 36 / 23, 333 x 1000 x 2731 59 / 48).
// Operands whose summed index is not contiguous are turned by the loads from LDS, nothing is transposed in memory.
// The saved sums are fp32: rounded to bf16 they would be a third rounding on the way to a weight's gradient (2.9e-3
// off its 64-bit value instead of 2.35e-3; dgate's and the result's own are the others).
//
// Few tokens: the weights' bytes bound the call; a wave multiplies 16 rows of each weight with up to 16 tokens,
// straight from memory into the matrix instruction's registers, the waves of a block split k and join in LDS.
//
// us, traced (TFLOP/s; a large library product reaches 1161 in bf16): 8192 x 4096 x 10944 bf16 forward with saved sums 1349 (1089),
// dgate | dup 261, dx 1212 (1212), both dw 1349 (1089).  1920 x 512 x 1376: 18.2, 8.7, 19.3, 14.6, short products on less than
// two blocks a compute unit.  333 x 1000 x 2731 fp16 forward 18: 129 blocks of 16 steps.  One token of 2048 -> 5504: 9.3 (45 MB,
// 4.9 TB/s).
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
    int splits, split_steps;  // kInput: blocks that share a tile's sum, and steps of each; their sums go to
    float *partial;           // [splits][m][partial_ld]
    int64_t partial_ld;
    bool direct;             // whole steps go from memory to LDS without registers
    bool out_wide, gate_wide;  // rows of results start at 16-byte boundaries
};

// A step of the sum is 64 values of k.  In LDS an operand by rows has 128 bytes a row, in eight 16-byte pieces; by columns
// 64 rows (of k) of a tile's width.  A wave's load instruction fills 1024 bytes in lane order, so pieces are exchanged
// on the way by the global addresses: without that, lanes that read one piece of 16 rows, or four rows of k, would
// meet in the same banks.
constexpr int kStep = 64;

__device__ __forceinline__ int row_piece(int row, int piece) {  // by rows: byte of a piece
    return row * 128 + ((piece ^ ((row >> 1) & 7)) * 16);
}
template <int WIDTH>
__device__ __forceinline__ int column_turn(int row) {  // by columns: what the 64-byte slots of a row of k are exchanged by
    return WIDTH >= 128 ? row & 3 : (row >> 1) & 1;
}

// 1024 bytes from memory to LDS without registers: lane i's 16 bytes at `from` go to lds + 16 i.  Written out
// because the compiler, where it sees such a load, lets every turned read from LDS wait for all of them.  It has no
// output register, so nothing of the compiler's can meet it in flight; vmcnt counts it, which makes the compiler's own
// waits only longer.  The compiler reserves m0: it keeps no value in it from one statement to another (and takes no word that
// one changes it); nothing else in these kernels uses it, as their listing shows.
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
    static constexpr int kChunks = WIDTH / 8;  // load instructions of a step

    // Byte offset from the tile's corner of what lane `lane` of chunk `chunk` loads.  `outer`: outer indices from
    // the corner on; rows and pieces past the end load the last, and their products are not stored.
    static __device__ __forceinline__ uint32_t offset(int chunk, int lane, int64_t outer, int64_t ld) {
        if constexpr (COLUMNS) {
            constexpr int pieces = WIDTH / 8, rows = 64 / pieces;
            const int row = chunk * rows + lane / pieces, at = lane % pieces;
            const int piece = (((at >> 2) ^ column_turn<WIDTH>(row)) << 2) | (at & 3);
            return (uint32_t)((row * ld + std::min<int64_t>(piece * 8, outer - 8)) * sizeof(T));
        }
        const int row = chunk * 8 + lane / 8, piece = (lane % 8) ^ ((row >> 1) & 7);
        return (uint32_t)((std::min<int64_t>(row, outer - 1) * ld + piece * 8) * sizeof(T));
    }

    // The number-th 16-byte piece of a step, zeros from `ks` values of k on, and its byte in LDS.  `at`: the step's corner.
    static __device__ __forceinline__ frag piece(const T *at, int64_t ld, int64_t outer, int64_t ks, int number) {
        frag v = {};
        if constexpr (COLUMNS) {
            constexpr int pieces = WIDTH / 8;
            const int row = number / pieces, piece = number % pieces;
            if (row < ks) v = *(const frag *)(at + row * ld + std::min<int64_t>(piece * 8, outer - 8));
        } else {
            const int row = number / 8, piece = number % 8;
            if (piece * 8 < ks) v = *(const frag *)(at + std::min<int64_t>(row, outer - 1) * ld + piece * 8);
        }
        return v;
    }
    static __device__ __forceinline__ int place(int number) {
        if constexpr (COLUMNS) {
            constexpr int pieces = WIDTH / 8;
            const int row = number / pieces, piece = number % pieces;
            return row * WIDTH * 2 + (((piece >> 2) ^ column_turn<WIDTH>(row)) << 6) + (piece & 3) * 16;
        }
        return row_piece(number / 8, number % 8);
    }

    // Byte of this lane's first piece of the fragment of 32 outer indices that starts at `first`.
    static __device__ __forceinline__ int fragment(int first, int lane) {
        if constexpr (COLUMNS) {
            const int q = lane % 16 / 4;  // the row of four that the lane reads for its group of 16
            return (lane / 32 * 8 + q) * WIDTH * 2 + (((first / 32) ^ column_turn<WIDTH>(q)) << 6) + lane / 16 % 2 * 32 + lane % 4 * 8;
        }
        return row_piece(first + lane % 32, lane / 32);
    }

    // Values 16 quarter .. 16 quarter + 15 of the step: lane l has outer index l % 32 and k = 8 (l / 32) .. + 7.
    static __device__ __forceinline__ frag read(const char *lds, int at, int quarter) {
        if constexpr (COLUMNS) {
            // four rows of k, 16 outer indices, turned by the load: a lane gets its index's four values
            typedef short s4 __attribute__((ext_vector_type(4)));
            typedef __attribute__((address_space(3))) s4 *ptr;
            struct {
                s4 v[2];
            } two;
#pragma unroll
            for (int i = 0; i < 2; i++)
                two.v[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ptr)(lds + at + (quarter * 16 + i * 4) * WIDTH * 2));
            return __builtin_bit_cast(frag, two);
        }
        return *(const frag *)(lds + (at ^ (quarter * 32)));
    }
};

// A block's place among the output tiles, and what its loads need.
template <typename T, int BM, int BN, int WM, int WN, Kind KIND>
struct Place {
    using A = Side<T, BM, KIND == kWeight>;
    using B = Side<T, KIND == kForward ? BN / 2 : BN, KIND != kForward>;  // kForward: two sides, w_gate's and w_up's
    static constexpr int kWaves = WM * WN, kLoads = (BM + BN) / 8 / kWaves, kOut = KIND == kForward ? BN / 2 : BN;
    int64_t m0, n0, outer_a, outer_b;
    const T *corner_a, *corner_b, *corner_b2;  // corners of the tile's sides in memory
    T *out;
    uint32_t offset[kLoads];

    __device__ __forceinline__ Place(const Product &p, int tile, int wave, int lane) {
        const T *a = (const T *)p.a;
        out = (T *)p.out;
        if (KIND == kWeight && tile >= p.tiles_m * p.tiles_n) {
            tile -= p.tiles_m * p.tiles_n;
            a += p.turn;
            out = (T *)p.out2;
        }
        const int across = tile / p.tiles_m;
        m0 = (int64_t)(tile - across * p.tiles_m) * BM, n0 = (int64_t)across * kOut;
        corner_a = KIND == kWeight ? a + m0 : a + m0 * p.a_ld;
        corner_b = KIND == kForward ? (const T *)p.b + n0 * p.b_ld : (const T *)p.b + n0;
        corner_b2 = KIND == kForward ? (const T *)p.b2 + n0 * p.b_ld : KIND == kInput ? (const T *)p.b2 + n0 : nullptr;
        outer_a = p.a_outer - m0, outer_b = p.b_outer - n0;
#pragma unroll
        for (int i = 0; i < kLoads; i++) {
            const int chunk = i * kWaves + wave;
            offset[i] = i * kWaves < A::kChunks ? A::offset(chunk, lane, outer_a, p.a_ld)
                                                : B::offset((chunk - A::kChunks) % B::kChunks, lane, outer_b, p.b_ld);
        }
    }
};

// A block a tile: while its results drain the next block on the compute unit is at its loads already.  (Blocks that stay
// and send the next tile's first steps before they store were 2 % slower on 8192 x 4096 x 10944: loads are counted
// off behind the stores, so the first steps wait for all of them.)
template <typename T, int BM, int BN, int WM, int WN, Kind KIND, int STAGES>
__global__ __launch_bounds__(WM * WN * 64) void product_kernel(Product p) {
    using frag = typename Frag<T>::type;
    using Pl = Place<T, BM, BN, WM, WN, KIND>;
    using A = typename Pl::A;
    using B = typename Pl::B;
    constexpr int kWaves = WM * WN, FM = BM / WM / 32, FN = BN / WN / 32, kBytes = (BM + BN) * 128, kLoads = Pl::kLoads;
    constexpr int kWide = (KIND == kForward ? FN / 2 : FN) * 32;  // outputs of a wave across
    static_assert(A::kChunks % kWaves == 0 && B::kChunks % kWaves == 0 && (kWide == 32 || kWide == 64) && STAGES >= 2 && STAGES * kLoads < 64, "");
    extern __shared__ char lds[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), lane = threadIdx.x % 64, wm = wave / WN, wn = wave % WN;
    const uint32_t lds_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
    // this wave's, for turning results: in the stages' place, which nobody reads behind the last step's barrier
    char *const scratch = lds + wave * 4096;
    static_assert(kWaves * 4096 <= STAGES * kBytes, "");
    const int64_t move_a = KIND == kWeight ? kStep * p.a_ld : kStep, move_b = KIND == kForward ? kStep : kStep * p.b_ld;
    // kInput: steps of w_gate, then of w_up; `turn` is a multiple of the step
    const int all = (int)((p.k + kStep - 1) / kStep), turn = KIND == kInput ? (int)(p.turn / kStep) : all;
    // this block's: all, or its share of them
    const bool split = KIND == kInput && p.splits > 1;
    const int share = split ? (int)blockIdx.x / (p.tiles_m * p.tiles_n) : 0, first = share * p.split_steps;
    const int steps = split ? std::min(all, first + p.split_steps) : all;
    // whole steps go from memory to LDS without registers
    const int whole = !p.direct ? 0 : (int)((KIND == kInput ? p.k - p.turn : p.k) / kStep);
    auto is_direct = [&](int t) { return t < steps && (t >= turn ? t - turn : t) < whole; };
    // values of k that step t has
    auto values = [&](int t) -> int64_t {
        if (KIND == kInput) return std::min<int64_t>(kStep, std::max<int64_t>(0, p.k - p.turn - (int64_t)(t >= turn ? t - turn : t) * kStep));
        return std::min<int64_t>(kStep, p.k - (int64_t)t * kStep);
    };
    int place_a[FM], place_b[FN];
#pragma unroll
    for (int i = 0; i < FM; i++) place_a[i] = A::fragment((wm * FM + i) * 32, lane);
#pragma unroll
    for (int j = 0; j < FN; j++)
        place_b[j] = BM * 128 + (KIND == kForward ? j % 2 * (BN * 64) + B::fragment((wn * (FN / 2) + j / 2) * 32, lane)
                                                  : B::fragment((wn * FN + j) * 32, lane));
    const Pl at(p, split ? (int)blockIdx.x - share * p.tiles_m * p.tiles_n : (int)blockIdx.x, wave, lane);
    // Addresses of this thread's loads of a step; which operand a load is of goes by its number, for all waves.
    const T *from[kLoads];
    auto address = [&](int t) {
        const T *at_a = at.corner_a + t * move_a;
        const T *at_b = KIND == kInput && t >= turn ? at.corner_b2 + (t - turn) * move_b : at.corner_b + t * move_b;
        const T *at_b2 = KIND == kForward ? at.corner_b2 + t * move_b : nullptr;
#pragma unroll
        for (int i = 0; i < kLoads; i++)
            from[i] = (const T *)((const char *)(i * kWaves < A::kChunks ? at_a
                                                 : KIND == kForward && i * kWaves >= A::kChunks + B::kChunks ? at_b2 : at_b) +
                                  at.offset[i]);
    };
    auto load_direct = [&](int t) {
        const uint32_t to = lds_at + t % STAGES * kBytes;
#pragma unroll
        for (int i = 0; i < kLoads; i++) load_to_lds(from[i], to + (i * kWaves + wave) * 1024);
    };
    auto load = [&](int t) {
        if (is_direct(t)) {
            address(t);
            load_direct(t);
        } else if (t < steps) {
            const T *at_a = at.corner_a + t * move_a;
            const T *at_b = KIND == kInput && t >= turn ? at.corner_b2 + (t - turn) * move_b : at.corner_b + t * move_b;
            char *to = lds + t % STAGES * kBytes;
            const int64_t ks = values(t);
            const int thread = afresh(threadIdx.x);
            // a thread's kLoads pieces, up to four at a time
            constexpr int kBatch = BM == 256 ? 2 : kLoads % 4 == 0 ? 4 : 3, kPiecesA = BM * 8, kPiecesB = B::kChunks * 64;
            static_assert(kLoads % kBatch == 0 && kPiecesA % (kWaves * 64) == 0 && kPiecesB % (kWaves * 64) == 0, "");
#pragma unroll
            for (int i0 = 0; i0 < kLoads; i0 += kBatch) {
                frag v[kBatch];
#pragma unroll
                for (int u = 0; u < kBatch; u++) {
                    const int first = (i0 + u) * kWaves * 64;
                    if (first < kPiecesA)
                        v[u] = A::piece(at_a, p.a_ld, at.outer_a, ks, first + thread);
                    else
                        v[u] = B::piece(first < kPiecesA + kPiecesB ? at_b : at.corner_b2 + t * move_b, p.b_ld, at.outer_b, ks,
                                        (first - kPiecesA) % kPiecesB + thread);
                }
#pragma unroll
                for (int u = 0; u < kBatch; u++) {
                    const int first = (i0 + u) * kWaves * 64;
                    char *side = to + (first < kPiecesA ? 0 : first < kPiecesA + kPiecesB ? kPiecesA * 16 : (kPiecesA + kPiecesB) * 16);
                    const int number = first < kPiecesA ? first : (first - kPiecesA) % kPiecesB;
                    *(frag *)(side + (first < kPiecesA ? A::place(number + thread) : B::place(number + thread))) = v[u];
                }
            }
        }
    };
    auto read = [&](frag(&fa)[FM], frag(&fb)[FN], int t, int quarter) {
        const char *from = lds + t % STAGES * kBytes;
#pragma unroll
        for (int i = 0; i < FM; i++) fa[i] = A::read(from, place_a[i], quarter);
#pragma unroll
        for (int j = 0; j < FN; j++) fb[j] = B::read(from, place_b[j], quarter);
    };
    f32x16 acc[FM][FN] = {};
    auto multiply = [&](frag(&fa)[FM], frag(&fb)[FN]) {
#pragma unroll
        for (int i = 0; i < FM; i++)
#pragma unroll
            for (int j = 0; j < FN; j++) acc[i][j] = mma32(fb[j], fa[i], acc[i][j]);
    };
    auto barrier = [&] {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    auto done_reading = [&] { __builtin_amdgcn_s_waitcnt(0xC07F); };  // lgkmcnt(0)
    auto keep_order = [&] { __builtin_amdgcn_sched_barrier(0); };

    frag a0[FM], b0[FN], a1[FM], b1[FN];
    // Fragments are read a quarter of a step ahead, into two sets of registers, and a quarter's own reads are waited for
    // before the next are sent.  Before the last quarter everybody's reads of step t are done and step t + 1 is
    // there (its loads were sent STAGES - 1 steps ago): one barrier, then step t + STAGES is sent to step t's place.
    auto step = [&](int t, auto fast) {  // fast: steps up to t + STAGES are there and direct
        done_reading(), keep_order();
        read(a1, b1, t, 1), keep_order();
        multiply(a0, b0), keep_order();
        done_reading(), keep_order();
        read(a0, b0, t, 2), keep_order();
        multiply(a1, b1), keep_order();
        done_reading(), keep_order();
        read(a1, b1, t, 3), keep_order();
        multiply(a0, b0), keep_order();
        done_reading();
        if constexpr (fast.value) {
            asm volatile("s_waitcnt vmcnt(%0)" : : "n"((STAGES - 2) * kLoads) : "memory");
            barrier();
            load_direct(t + STAGES);
#pragma unroll
            for (int i = 0; i < kLoads; i++) from[i] += i * kWaves < A::kChunks ? move_a : move_b;
            read(a0, b0, t + 1, 0);
        } else {
            asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
            barrier();
            load(t + STAGES);
            if (t + 1 < steps) read(a0, b0, t + 1, 0);
        }
        keep_order();
        multiply(a1, b1), keep_order();
    };
    // end of the fast steps that t is among: those behind t that are counted off are direct, too, and their loads
    // move on in one operand
    auto fast_end = [&](int t) {
        if (KIND != kInput || t + STAGES < turn) return std::min(whole, steps) - STAGES;
        return whole == turn || t + 2 >= turn ? std::min(turn + whole, steps) - STAGES : t;
    };
    if (steps > first) {
        bool ahead = true;  // the first steps are all there and direct
        for (int t = first; t < first + STAGES; t++) ahead = ahead && is_direct(t), load(t);
        done_reading();
        if (ahead)
            asm volatile("s_waitcnt vmcnt(%0)" : : "n"((STAGES - 1) * kLoads) : "memory");
        else
            asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
        barrier();
        read(a0, b0, first, 0);
        for (int t = first; t < steps;) {
            const int end = fast_end(t);
            if (t < end) address(t + STAGES);
            for (; t < end; t++) step(t, std::true_type{});
            if (t < steps) step(t++, std::false_type{});
        }
    }
    const int64_t m0 = at.m0 + wm * FM * 32, n0 = at.n0 + wn * kWide;
    T *const out = at.out;
    // Results: of a fragment, lane l holds row l % 32 and columns 8 (r / 4) + 4 (l / 32) + r % 4.  32 rows at a time
    // go through the wave's scratch, where a row's pieces of 16 bytes are exchanged as above, and out in rows.
    const bool full = m0 + FM * 32 <= p.m && n0 + kWide <= p.n;
    const int own = afresh(lane), row = own % 32, high = own / 32;
    auto exchange = [&](int bytes) { return bytes == 128 ? (row >> 1) & 7 : (row >> 2) & 3; };
    auto flush = [&](auto type, int i, auto bytes_, int from, auto *to, int64_t ld, bool wide) {
        // rows of bytes_ bytes from the scratch to memory
        asm volatile("" ::: "memory");
        using U = decltype(type);
        constexpr int bytes = bytes_.value, pieces = bytes / 16, per = 16 / sizeof(U);
#pragma unroll
        for (int c = 0; c < 32 * pieces / 64; c++) {
            const int r = c * (64 / pieces) + own / pieces, piece = own % pieces;
            const int turned = piece ^ (bytes == 128 ? (r >> 1) & 7 : (r >> 2) & 3);
            const Pack<U, per> v = *(const Pack<U, per> *)(scratch + r * bytes + turned * 16);
            U *at_row = to + (m0 + i * 32 + r) * ld + n0 + from + piece * per;
            if (full && wide) {
                put(at_row, v);
            } else if (m0 + i * 32 + r < p.m) {
                const int64_t left = p.n - n0 - from - piece * per;
                if (wide && left >= per) {
                    put(at_row, v);
                } else {
#pragma unroll
                    for (int e = 0; e < per; e++)
                        if (e < left) at_row[e] = v.v[e];
                }
            }
        }
        asm volatile("" ::: "memory");
    };
    if constexpr (KIND == kInput)
        if (split) {
            float *const sums = p.partial + share * p.m * p.partial_ld;
#pragma unroll
            for (int i = 0; i < FM; i++)
#pragma unroll
                for (int j = 0; j < FN; j++) {
#pragma unroll
                    for (int g = 0; g < 4; g++) {
                        Pack<float, 4> v;
#pragma unroll
                        for (int e = 0; e < 4; e++) v.v[e] = acc[i][j][g * 4 + e];
                        *(Pack<float, 4> *)(scratch + row * 128 + ((g * 2 + high) ^ exchange(128)) * 16) = v;
                    }
                    flush(0.0f, i, std::integral_constant<int, 128>{}, j * 32, sums, p.partial_ld, true);
                }
            return;
        }
    constexpr std::integral_constant<int, kWide * 2> out_bytes{};
    with_act(KIND == kForward ? p.act : BYZ_ACT_NONE, [&](auto act) {
#pragma unroll
        for (int i = 0; i < FM; i++) {
#pragma unroll
            for (int j = 0; j < FN; j += KIND == kForward ? 2 : 1)
#pragma unroll
                for (int g = 0; g < 4; g++) {
                    Pack<T, 4> v;
#pragma unroll
                    for (int e = 0; e < 4; e++) {
                        const float x = acc[i][j][g * 4 + e];
                        if constexpr (KIND == kForward)
                            v.v[e] = round_to<T>(act_value<act.value>(x) * acc[i][j + 1][g * 4 + e]);
                        else
                            v.v[e] = round_to<T>(x);
                    }
                    const int piece = (KIND == kForward ? j / 2 : j) * 4 + g;
                    *(Pack<T, 4> *)(scratch + row * out_bytes.value + (piece ^ exchange(out_bytes.value)) * 16 + high * 8) = v;
                }
            flush(T{}, i, out_bytes, 0, out, p.out_ld, p.out_wide);
            if constexpr (KIND == kForward)
                if (p.gate) {
#pragma unroll
                    for (int j = 0; j < FN; j++) {
#pragma unroll
                        for (int g = 0; g < 4; g++) {
                            Pack<float, 4> v;
#pragma unroll
                            for (int e = 0; e < 4; e++) v.v[e] = acc[i][j][g * 4 + e];
                            *(Pack<float, 4> *)(scratch + row * 128 + ((g * 2 + high) ^ exchange(128)) * 16) = v;
                        }
                        flush(0.0f, i, std::integral_constant<int, 128>{}, j / 2 * 32, j % 2 ? p.up : p.gate, p.gate_ld, p.gate_wide);
                    }
                }
        }
    });
}

// Up to 16 tokens.  A block has 8 outputs: a matrix instruction's 16 columns are their gate rows and their up rows.  Its waves
// share k, 64 values (a cache line of a row) at a time.  Blocks of 16 outputs, with an instruction for each weight, are half as
// many: 344 of them on 256 compute units took 11.3 us for a token of 2048 -> 5504.
constexpr int kSkinnyWaves = 8, kSkinnyOut = 8;
template <typename T>
__global__ __launch_bounds__(kSkinnyWaves * 64) void skinny_kernel(Product p) {
    using frag = typename Frag<T>::type;
    __shared__ f32x4 part[kSkinnyWaves][64];
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, col = lane % 16;
    const int64_t n0 = (int64_t)blockIdx.x * kSkinnyOut, n = std::min<int64_t>(n0 + col % 8, p.n - 1);
    const T *w = (const T *)(col < 8 ? p.b : p.b2) + n * p.b_ld;
    const bool token = col < p.m;
    const T *x = (const T *)p.a + (token ? col : 0) * p.a_ld;
    f32x4 acc = {};
    constexpr int kAhead = 4, kApart = kSkinnyWaves * 64;
    int64_t k0 = wave * 64;
    if (p.direct)
        for (; k0 + (kAhead - 1) * kApart + 64 <= p.k; k0 += kAhead * kApart) {
            frag a[2 * kAhead], b[2 * kAhead];
#pragma unroll
            for (int u = 0; u < 2 * kAhead; u++) {
                const int64_t k = k0 + u / 2 * kApart + u % 2 * 32 + lane / 16 * 8;
                b[u] = *(const frag *)(w + k);
                a[u] = frag{};
                if (token) a[u] = *(const frag *)(x + k);
            }
#pragma unroll
            for (int u = 0; u < 2 * kAhead; u++) acc = mma16(a[u], b[u], acc);
        }
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
    for (; k0 < p.k; k0 += kApart)
        for (int half = 0; half < 2; half++) {
            const int64_t k = k0 + half * 32 + lane / 16 * 8;
            frag a = piece(x, k), b = piece(w, k);
            if (!token) a = frag{};
            acc = mma16(a, b, acc);
        }
    part[wave][lane] = acc;
    __syncthreads();
    if (wave == 0) {
        for (int v = 1; v < kSkinnyWaves; v++) acc += part[v][lane];
        with_act(p.act, [&](auto act) {
#pragma unroll
            for (int r = 0; r < 4; r++) {
                const float up = __shfl_xor(acc[r], 8);  // of lanes with a gate
                const int64_t row = lane / 16 * 4 + r, at = n0 + col;
                if (col >= 8 || row >= p.m || at >= p.n) continue;
                ((T *)p.out)[row * p.out_ld + at] = round_to<T>(act_value<act.value>(acc[r]) * up);
                if (p.gate) {
                    p.gate[row * p.gate_ld + at] = acc[r];
                    p.up[row * p.gate_ld + at] = up;
                }
            }
        });
    }
}

// dgate | dup from dh, gate and up: `d` is [m][2 np] (dgate, then dup), zeros in the padding.  They are rounded to the type,
// which is what the matrix instructions of both products behind take: in bf16 gradients are 2.3e-3 off their 64-bit values so, for
// 1.7e-3 of their own rounding alone; two 16-bit parts of each would double the products.
struct Slopes {
    const void *dh;
    const float *gate, *up;
    int64_t dh_ld, gate_ld, m, n, np;
    void *d;
    int act;
};

// Four values a thread, rows of np / 4 threads.  Bound by memory: 258 us for 8192 x 10944 (1256 MB, 4.9 TB/s); eight values a
// thread, whose loads are 32 bytes apart: 315.
template <typename T, bool WIDE>
__global__ __launch_bounds__(256) void slopes_kernel(Slopes s) {
    const int64_t across = s.np / 4, all = s.m * across;
    const bool small = all <= UINT32_MAX;
    with_act(s.act, [&](auto act) {
        for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < all; at += (int64_t)gridDim.x * 256) {
            const int64_t i = small ? (uint32_t)at / (uint32_t)across : at / across, j = (at - i * across) * 4;
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

// Adds the sums of the blocks that share a tile, in their order, four values a thread.
template <typename T>
__global__ __launch_bounds__(256) void join_kernel(const float *partial, int splits, int64_t m, int64_t n, int64_t ld, T *out, int64_t out_ld) {
    const int64_t across = ld / 4, all = m * across, apart = m * ld;
    const bool wide = ((uintptr_t)out & 7) == 0 && out_ld % 4 == 0;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < all; at += (int64_t)gridDim.x * 256) {
        const int64_t i = at / across, j = (at - i * across) * 4;
        const float *from = partial + i * ld + j;
        Pack<float, 4> sum = *(const Pack<float, 4> *)from;
        for (int k = 1; k < splits; k++) {
            const Pack<float, 4> v = *(const Pack<float, 4> *)(from + k * apart);
#pragma unroll
            for (int e = 0; e < 4; e++) sum.v[e] += v.v[e];
        }
        Pack<T, 4> r;
#pragma unroll
        for (int e = 0; e < 4; e++) r.v[e] = round_to<T>(sum.v[e]);
        T *to = out + i * out_ld + j;
        if (wide && j + 4 <= n) {
            put(to, r);
        } else {
#pragma unroll
            for (int e = 0; e < 4; e++)
                if (j + e < n) to[e] = r.v[e];
        }
    }
}

unsigned grid_of(int64_t threads) { return (unsigned)std::min<int64_t>((threads + 255) / 256, 8192); }

template <typename T, int BM, int BN, int WM, int WN, Kind KIND, int STAGES>
int launch_tile(Product p, hipStream_t s) {
    constexpr int kOut = KIND == kForward ? BN / 2 : BN, kThreads = WM * WN * 64, kLds = STAGES * (BM + BN) * 128;
    const int64_t tm = (p.m + BM - 1) / BM, tn = (p.n + kOut - 1) / kOut, tiles = tm * tn * (KIND == kWeight ? 2 : KIND == kInput ? p.splits : 1);
    if (tiles > INT32_MAX / kThreads) return BYZ_EUNSUPPORTED;
    p.tiles_m = (int)tm, p.tiles_n = (int)tn;
    // a lane's place in a tile's side is a 32-bit offset
    const int64_t most = INT32_MAX / (int64_t)sizeof(T);
    p.direct = (KIND == kWeight ? kStep : BM) * p.a_ld + BM < most && (KIND == kForward ? BN : kStep) * p.b_ld + BN < most;
    p.out_wide = aligned(p.out, 16) && p.out_ld % 8 == 0 && (!p.out2 || aligned(p.out2, 16));
    p.gate_wide = p.gate && aligned(p.gate, 16) && aligned(p.up, 16) && p.gate_ld % 4 == 0;
    auto *kernel = &product_kernel<T, BM, BN, WM, WN, KIND, STAGES>;
    BYZ_HIP(hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, kLds));
    kernel<<<(unsigned)tiles, kThreads, kLds, s>>>(p);
    BYZ_HIP(hipGetLastError());
    return BYZ_OK;
}

// The tiles that a product can be cut into: how many blocks of them a compute unit holds, and what a step takes of
// its time (us, measured on products that fill the card).  Fewer than two blocks leave room for more stages.
struct Shape {
    int bm, bn, stages, resident;
    double step;
};
constexpr Shape kShapes[] = {{256, 256, 2, 1, 1.85}, {128, 128, 2, 2, 0.6}, {128, 128, 4, 1, 0.6}, {64, 128, 3, 2, 0.35},
                             {64, 128, 6, 1, 0.35},  {64, 64, 4, 2, 0.22},  {64, 64, 8, 1, 0.22}};

struct Choice {
    int shape, splits;
};

// The shape of the shortest estimated time: rounds of blocks, each so many steps and 3 us for its first loads and its stores; a step
// takes the blocks' products on a compute unit or, where those are shorter, the way from memory (1 us) over the stages ahead.
// dx of few tokens has few tiles and a long sum, which up to 16 blocks of a tile share, 8 steps each at least; the kernel that
// adds their sums takes 4 us and its bytes at 4 TB/s.
Choice best_shape(int64_t m, int64_t across, int64_t k, Kind kind) {
    Choice best{};
    double best_time = 0.0;
    const int64_t steps = (k + kStep - 1) / kStep;
    for (int splits = 1; splits <= (kind == kInput ? 16 : 1) && (splits == 1 || steps >= 8 * splits); splits *= 2)
        for (int i = 0; i < (kind != kForward ? 7 : 5); i++) {
            const Shape &c = kShapes[i];
            const int64_t tiles = ((m + c.bm - 1) / c.bm) * ((across + c.bn - 1) / c.bn) * (kind == kWeight ? 2 : splits);
            const int64_t rounds = (tiles + 256 * c.resident - 1) / (256 * c.resident), together = std::min<int64_t>(c.resident, (tiles + 255) / 256);
            const double step = std::max(together * c.step, 1.0 / (c.stages - 1));
            double time = rounds * ((steps + splits - 1) / splits * step + 3.0);
            if (splits > 1) time += 4.0 + (double)m * (double)across * (8 * splits + 2) / 4e6;
            if (best_time == 0.0 || time < best_time) best = {i, splits}, best_time = time;
        }
    return best;
}

// Operands' rows start at 16-byte boundaries and have whole 16-byte pieces.
template <typename T, Kind KIND>
int launch_shape(int shape, const Product &p, hipStream_t s) {
    switch (shape) {
        case 0: return launch_tile<T, 256, 256, 2, 4, KIND, 2>(p, s);
        case 1: return launch_tile<T, 128, 128, 2, 2, KIND, 2>(p, s);
        case 2: return launch_tile<T, 128, 128, 2, 2, KIND, 4>(p, s);
        case 3: return launch_tile<T, 64, 128, 2, 2, KIND, 3>(p, s);
        case 4: return launch_tile<T, 64, 128, 2, 2, KIND, 6>(p, s);
        default: break;
    }
    if constexpr (KIND != kForward)
        return shape == 5 ? launch_tile<T, 64, 64, 2, 2, KIND, 4>(p, s) : launch_tile<T, 64, 64, 2, 2, KIND, 8>(p, s);
    return BYZ_EINTERNAL;
}

// kInput: `partial` has room for the sums of the blocks that share a tile.
template <typename T, Kind KIND>
int launch_product(Product p, float *partial, hipStream_t s) {
    const Choice c = best_shape(p.m, KIND == kForward ? 2 * p.n : p.n, p.k, KIND);
    p.splits = c.splits;
    if (c.splits > 1) {
        const int64_t steps = (p.k + kStep - 1) / kStep;
        p.split_steps = (int)((steps + c.splits - 1) / c.splits);
        p.partial = partial, p.partial_ld = (p.n + 3) / 4 * 4;
    }
    int rc = launch_shape<T, KIND>(c.shape, p, s);
    if (rc == BYZ_OK && c.splits > 1) {
        join_kernel<T><<<grid_of(p.m * (p.partial_ld / 4)), 256, 0, s>>>(partial, c.splits, p.m, p.n, p.partial_ld, (T *)p.out, p.out_ld);
        BYZ_HIP(hipGetLastError());
    }
    return rc;
}

int64_t padded(int64_t v) { return (v + 63) / 64 * 64; }

bool sizes_ok(int64_t m, int64_t k, int64_t n) {
    const int64_t most = (int64_t)1 << 31;
    return m >= 0 && k >= 0 && n >= 0 && m < most && k < most && n < most;
}

// Whether the tile kernel reads a matrix as it lies: pieces of 16 bytes, none of them beyond the columns.
bool pieces(const void *at, int64_t cols, int64_t ld) { return aligned(at, 16) && cols % 8 == 0 && ld % 8 == 0; }

// Workspace, in elements: for the backward pass dgate | dup and the sums of blocks that share a tile of dx; behind them
// matrices that have to be copied, `aligned` without them.
struct Layout {
    int64_t np, kp;
    int64_t d, partial, x, w, aligned, all;
    Layout(int64_t m, int64_t k, int64_t n, bool backward) : np(padded(n)), kp((k + 7) / 8 * 8) {
        d = 0;
        partial = aligned = d + (backward ? m * 2 * np : 0);
        if (backward && m > 0 && k > 0) {
            const int splits = best_shape(m, k, np + n, kInput).splits;
            if (splits > 1) aligned += 2 * splits * m * ((k + 3) / 4 * 4);
        }
        x = aligned;
        w = x + m * kp;
        all = w + 2 * n * kp;
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

// Whether the tile kernel reads x and the weights, where a call has use for them, as they lie.
bool good_x(const Call &c, bool used) { return !used || c.m == 0 || c.k == 0 || pieces(c.x, c.k, c.x_ld); }
bool good_w(const Call &c, bool used) {
    return !used || c.n == 0 || c.k == 0 || (pieces(c.w_gate, c.k, c.w_ld) && pieces(c.w_up, c.k, c.w_ld));
}

// Copies those that it does not: rows of whole pieces, zeros behind k.
template <typename T>
int align_operands(Call &c, const Layout &lay, bool x, bool w, hipStream_t s) {
    T *ws = (T *)c.ws;
    int rc = BYZ_OK;
    if (!good_x(c, x)) rc = align<T>(&c.x, &c.x_ld, c.m, c.k, ws + lay.x, lay.kp, s);
    if (rc == BYZ_OK && !good_w(c, w)) {
        int64_t ld = c.w_ld;
        rc = align<T>(&c.w_gate, &ld, c.n, c.k, ws + lay.w, lay.kp, s);
        if (rc == BYZ_OK) rc = align<T>(&c.w_up, &c.w_ld, c.n, c.k, ws + lay.w + c.n * lay.kp, lay.kp, s);
    }
    return rc;
}

size_t forward_bytes(const Call &c) {
    return c.m <= kSkinny || (good_x(c, true) && good_w(c, true)) ? 0 : (size_t)Layout(c.m, c.k, c.n, false).all * 2;
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
        return launch_product<T, kForward>(p, nullptr, s);
    }
    p.direct = pieces(c.x, 8, c.x_ld) && pieces(c.w_gate, 8, c.w_ld) && pieces(c.w_up, 8, c.w_ld);
    skinny_kernel<T><<<(unsigned)((p.n + kSkinnyOut - 1) / kSkinnyOut), kSkinnyWaves * 64, 0, s>>>(p);
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
        rc = launch_product<T, kInput>(p, (float *)((T *)c.ws + lay.partial), s);
    }
    if (rc == BYZ_OK && dw) {
        Product p{};
        p.a = d, p.a_ld = 2 * lay.np, p.turn = lay.np, p.b = c.x, p.b_ld = c.x_ld;
        p.m = c.n, p.n = cols, p.k = c.m, p.out = g.dw_gate, p.out2 = g.dw_up, p.out_ld = g.dw_ld;
        p.a_outer = lay.np, p.b_outer = lay.kp;
        rc = launch_product<T, kWeight>(p, nullptr, s);
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

extern "C" size_t byz_gated_ffn_backward_aligned_workspace_bytes(int64_t m, int64_t k, int64_t n, int dtype) {
    if (!sizes_ok(m, k, n) || (dtype != BYZ_BF16 && dtype != BYZ_F16)) return 0;
    return (size_t)Layout(m, k, n, true).aligned * 2;
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
    const Call c{x, w_gate, w_up, x_ld, w_ld, m, k, n, act, workspace};
    const Layout lay(m, k, n, true);
    const size_t need = (size_t)(good_x(c, dw_gate) && good_w(c, dx) ? lay.aligned : lay.all) * 2;
    if (workspace_bytes < need || (need && (!workspace || !aligned(workspace, 16)))) return BYZ_ENOMEM;
    const Gradients g{dh, gate, up, dh_ld, gate_ld, dx, dw_gate, dw_up, dx_ld, dw_ld};
    return dtype == BYZ_BF16 ? backward<bf16>(c, g, (hipStream_t)stream) : backward<f16>(c, g, (hipStream_t)stream);
}

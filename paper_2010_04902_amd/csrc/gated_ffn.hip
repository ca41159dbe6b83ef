// Gated feed-forward block: both projections, activation and product in one kernel, and its gradients
// (gfx950, bf16 and fp16 with fp32 sums on the matrix cores).
//
// One tile kernel does all products as C[i, j] = sum_k A[i, k] B[j, k], both operands with the summed index
// contiguous in memory.  Forward, the rows of B in a tile are half gate and half up weights of the same outputs, laid out so
// that a wave holds both sums of an output in the same lane and register: the epilogue needs no exchange.
// Backward, one kernel makes dgate and dup (and both transposed), X and the weights are transposed, and
//     dx = [dgate | dup] [w_gate ; w_up]   sums over 2n,     [dw_gate ; dw_up] = [dgate | dup]^T x   over m.
// The workspace's copies are padded with zeros to whole steps of the sum.  The saved sums are fp32: rounded to bf16
// they would be a third rounding on the way to a weight's gradient (2.9e-3 off its 64-bit value instead of 2.35e-3;
// dgate's and the result's own are the others).
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

constexpr int kStep = 64;    // values of the summed index in a tile: 128 bytes, eight 16-byte pieces, a row
constexpr int kPieces = 8;

struct Product {
    const void *a, *b, *b2;  // b2: second half of a tile's rows (forward: w_up)
    int64_t a_ld, b_ld;
    int64_t m, n, k;         // forward: n outputs, of 2n rows in all
    void *out, *out2;        // backward weights: rows from `split` on go to out2
    int64_t out_ld, split;
    float *gate, *up;        // forward: saved sums
    int64_t gate_ld;
    int act;
    int tiles_m, tiles_n;
    bool pieces;             // operands' rows start at 16-byte boundaries
};

// LDS place of piece p of a tile's row: rows are 128 bytes, two rows span the banks; without the exchange
// of pieces, 16 lanes that read one piece of 16 rows would meet in 4 banks.
__device__ __forceinline__ int place(int row, int p) { return row * 128 + ((p ^ ((row >> 1) & 7)) * 16); }

template <typename T, int BM, int BN, int WM, int WN, bool DUAL>
struct Tile {
    static constexpr int kWaves = WM * WN, kThreads = kWaves * 64;
    static constexpr int kBytes = (BM + BN) * 128;  // one step of both operands
    static constexpr int FM = BM / WM / 32, FN = BN / WN / 32;

    // global row of a tile's row, clamped: rows past the end are computed and not stored
    static __device__ __forceinline__ const T *row_at(const Product &p, int64_t m0, int64_t n0, int row) {
        if (row < BM) return (const T *)p.a + std::min<int64_t>(m0 + row, p.m - 1) * p.a_ld;
        row -= BM;
        if constexpr (DUAL) {
            const T *base = (const T *)(row < BN / 2 ? p.b : p.b2);
            return base + std::min<int64_t>(n0 + row % (BN / 2), p.n - 1) * p.b_ld;
        }
        return (const T *)p.b + std::min<int64_t>(n0 + row, p.n - 1) * p.b_ld;
    }

    // A whole step, memory to LDS without registers: a wave instruction fills eight rows.
    static __device__ __forceinline__ void load_step(const T *const (&rows)[(BM + BN) / 8 / kWaves], int64_t k0, char *lds) {
        const int wave = threadIdx.x / 64;
#pragma unroll
        for (int i = 0; i < (BM + BN) / 8 / kWaves; i++)
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(rows[i] + k0),
                                             (__attribute__((address_space(3))) void *)(lds + (i * kWaves + wave) * 1024), 16, 0, 0);
    }

    // The last, shorter step, or any step of operands off the 16-byte boundaries: through registers, zeros behind k.
    static __device__ void load_part(const Product &p, int64_t m0, int64_t n0, int64_t k0, char *lds) {
        for (int at = threadIdx.x; at < (BM + BN) * kPieces; at += kThreads) {
            const int row = at / kPieces, piece = at % kPieces;
            const T *src = row_at(p, m0, n0, row);
            const int64_t k = k0 + piece * 8;
            typename Frag<T>::type v;
            if (p.pieces && k + 8 <= p.k) {
                v = *(const typename Frag<T>::type *)(src + k);
            } else {
#pragma unroll
                for (int e = 0; e < 8; e++) v[e] = k + e < p.k ? src[k + e] : (T)0.0f;
            }
            *(typename Frag<T>::type *)(lds + place(row, piece)) = v;
        }
    }
};

template <typename T, int BM, int BN, int WM, int WN, bool DUAL>
__global__ __launch_bounds__(WM * WN * 64) void product_kernel(Product p) {
    using Tl = Tile<T, BM, BN, WM, WN, DUAL>;
    using frag = typename Frag<T>::type;
    constexpr int FM = Tl::FM, FN = Tl::FN, kLoads = (BM + BN) / 8 / Tl::kWaves;
    extern __shared__ char lds[];
    const int wave = threadIdx.x / 64, lane = threadIdx.x % 64, wm = wave / WN, wn = wave % WN;
    constexpr int kOut = DUAL ? BN / 2 : BN;  // outputs across a tile
    const int64_t m0 = (int64_t)(blockIdx.x % p.tiles_m) * BM, n0 = (int64_t)(blockIdx.x / p.tiles_m) * kOut;

    const T *rows[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; i++) {
        const int row = (i * Tl::kWaves + wave) * 8 + lane / 8;
        rows[i] = Tl::row_at(p, m0, n0, row) + ((lane % 8) ^ ((row >> 1) & 7)) * 8;
    }
    // fragment rows in the tile
    int arow[FM], brow[FN];
#pragma unroll
    for (int i = 0; i < FM; i++) arow[i] = wm * FM * 32 + i * 32 + lane % 32;
#pragma unroll
    for (int j = 0; j < FN; j++)
        brow[j] = BM + (DUAL ? (j % 2) * (BN / 2) + (wn * (FN / 2) + j / 2) * 32 : (wn * FN + j) * 32) + lane % 32;

    f32x16 acc[FM][FN] = {};
    const int64_t whole = p.pieces ? p.k / kStep : 0, steps = (p.k + kStep - 1) / kStep;
    auto load = [&](int64_t t) {
        char *to = lds + (t & 1) * Tl::kBytes;
        if (t < whole)
            Tl::load_step(rows, t * kStep, to);
        else
            Tl::load_part(p, m0, n0, t * kStep, to);
    };
    if (steps > 0) load(0);
    for (int64_t t = 0; t < steps; t++) {
        __builtin_amdgcn_s_waitcnt(0x0F70);  // this wave's loads to LDS are done
        __syncthreads();                     // everybody's are, and the other half has been read
        if (t + 1 < steps) load(t + 1);
        const char *at = lds + (t & 1) * Tl::kBytes;
#pragma unroll
        for (int kk = 0; kk < kStep / 16; kk++) {
            frag a[FM], b[FN];
#pragma unroll
            for (int i = 0; i < FM; i++) a[i] = *(const frag *)(at + place(arow[i], kk * 2 + lane / 32));
#pragma unroll
            for (int j = 0; j < FN; j++) b[j] = *(const frag *)(at + place(brow[j], kk * 2 + lane / 32));
#pragma unroll
            for (int i = 0; i < FM; i++)
#pragma unroll
                for (int j = 0; j < FN; j++) acc[i][j] = mma32(a[i], b[j], acc[i][j]);
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
    if constexpr (DUAL) {
        with_act(p.act, [&](auto act) {
            each([&](int i, int r, int64_t row) {
#pragma unroll
                for (int j = 0; j < FN; j += 2) {
                    const int64_t col = n0 + (wn * (FN / 2) + j / 2) * 32 + lane % 32;
                    if (col >= p.n) continue;
                    const float g = acc[i][j][r], u = acc[i][j + 1][r];
                    ((T *)p.out)[row * p.out_ld + col] = round_to<T>(act_value<act.value>(g) * u);
                    if (p.gate) {
                        p.gate[row * p.gate_ld + col] = g;
                        p.up[row * p.gate_ld + col] = u;
                    }
                }
            });
        });
    } else {
        each([&](int i, int r, int64_t row) {
            T *out = row < p.split ? (T *)p.out + row * p.out_ld : (T *)p.out2 + (row - p.split) * p.out_ld;
#pragma unroll
            for (int j = 0; j < FN; j++) {
                const int64_t col = n0 + (wn * FN + j) * 32 + lane % 32;
                if (col < p.n) out[col] = round_to<T>(acc[i][j][r]);
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
        if (p.pieces && k + 8 <= p.k) {
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

// dgate | dup from dh, gate and up: `d` is [m][2 np] (dgate, then dup), `dt` its transposed [2 np][mp]; zeros in the padding.
// A block a 64 x 64 piece of the padded m x n.
struct Slopes {
    const void *dh;
    const float *gate, *up;
    int64_t dh_ld, gate_ld, m, n, np, mp;
    void *d, *dt;
    int act, across;
};

template <typename T>
__global__ __launch_bounds__(256) void slopes_kernel(Slopes s) {
    __shared__ T tile[2][64][66];
    const int64_t m0 = (int64_t)(blockIdx.x / s.across) * 64, n0 = (int64_t)(blockIdx.x % s.across) * 64;
    const int col = threadIdx.x % 64;
    with_act(s.act, [&](auto act) {
        for (int r = threadIdx.x / 64; r < 64; r += 4) {
            const int64_t i = m0 + r, j = n0 + col;
            T dg = (T)0.0f, du = (T)0.0f;
            if (i < s.m && j < s.n) {
                const float dh = (float)((const T *)s.dh)[i * s.dh_ld + j];
                const float g = s.gate[i * s.gate_ld + j], u = s.up[i * s.gate_ld + j];
                dg = round_to<T>(dh * u * act_slope<act.value>(g));
                du = round_to<T>(dh * act_value<act.value>(g));
            }
            if (i < s.m) {
                ((T *)s.d)[i * 2 * s.np + j] = dg;
                ((T *)s.d)[i * 2 * s.np + s.np + j] = du;
            }
            tile[0][r][col] = dg, tile[1][r][col] = du;
        }
    });
    __syncthreads();
    for (int half = 0; half < 2; half++)
        for (int r = threadIdx.x / 64; r < 64; r += 4)
            ((T *)s.dt)[(half * s.np + n0 + r) * s.mp + m0 + col] = tile[half][col][r];
}

// out[c][r] = in[r][c] of a rows x cols matrix; rows from `rows` up to the next multiple of 64 give zeros.
template <typename T>
__global__ __launch_bounds__(256) void transpose_kernel(const T *in, int64_t in_ld, int64_t rows, int64_t cols, T *out,
                                                        int64_t out_ld, int across) {
    __shared__ T tile[64][66];
    const int64_t r0 = (int64_t)(blockIdx.x / across) * 64, c0 = (int64_t)(blockIdx.x % across) * 64;
    const int lane = threadIdx.x % 64;
    for (int r = threadIdx.x / 64; r < 64; r += 4)
        tile[r][lane] = r0 + r < rows && c0 + lane < cols ? in[(r0 + r) * in_ld + c0 + lane] : (T)0.0f;
    __syncthreads();
    for (int r = threadIdx.x / 64; r < 64; r += 4)
        if (c0 + r < cols) out[(c0 + r) * out_ld + r0 + lane] = tile[lane][r];
}

template <typename T, int BM, int BN, int WM, int WN, bool DUAL>
int launch_tile(Product p, hipStream_t s) {
    using Tl = Tile<T, BM, BN, WM, WN, DUAL>;
    constexpr int kOut = DUAL ? BN / 2 : BN;
    const int64_t tm = (p.m + BM - 1) / BM, tn = (p.n + kOut - 1) / kOut;
    if (tm * tn > INT32_MAX / Tl::kThreads) return BYZ_EUNSUPPORTED;
    p.tiles_m = (int)tm, p.tiles_n = (int)tn;
    auto *kernel = &product_kernel<T, BM, BN, WM, WN, DUAL>;
    BYZ_HIP(hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, 2 * Tl::kBytes));
    kernel<<<(unsigned)(tm * tn), Tl::kThreads, 2 * Tl::kBytes, s>>>(p);
    BYZ_HIP(hipGetLastError());
    return BYZ_OK;
}

template <typename T, bool DUAL>
int launch_product(const Product &p, hipStream_t s) {
    const int64_t across = DUAL ? 2 * p.n : p.n;
    auto tiles = [&](int bm, int bn) { return ((p.m + bm - 1) / bm) * ((across + bn - 1) / bn); };
    if (tiles(256, 256) >= 192) return launch_tile<T, 256, 256, 2, 4, DUAL>(p, s);
    if (tiles(128, 128) >= 192) return launch_tile<T, 128, 128, 2, 2, DUAL>(p, s);
    return launch_tile<T, 64, 128, 2, 2, DUAL>(p, s);
}

int64_t padded(int64_t v) { return (v + 63) / 64 * 64; }

bool sizes_ok(int64_t m, int64_t k, int64_t n) {
    const int64_t most = (int64_t)1 << 31;
    return m >= 0 && k >= 0 && n >= 0 && m < most && k < most && n < most;
}

// Workspace of the backward pass, in elements.
struct Layout {
    int64_t np, mp;
    int64_t d, dt, wt, xt, all;
    Layout(int64_t m, int64_t k, int64_t n) : np(padded(n)), mp(padded(m)) {
        d = 0;
        dt = d + m * 2 * np;      // m rows of 2 np
        wt = dt + 2 * np * mp;    // 2 np rows of mp
        xt = wt + k * 2 * np;     // k rows of 2 np: w_gate's and w_up's columns
        all = xt + k * mp;        // k rows of mp
    }
};

template <typename T>
int forward(const Product &p, hipStream_t s) {
    if (p.m <= 16) {
        skinny_kernel<T><<<(unsigned)((p.n + 15) / 16), kSkinnyWaves * 64, 0, s>>>(p);
        BYZ_HIP(hipGetLastError());
        return BYZ_OK;
    }
    return launch_product<T, true>(p, s);
}

struct Backward {
    const void *dh, *x, *w_gate, *w_up;
    const float *gate, *up;
    int64_t dh_ld, x_ld, w_ld, gate_ld, m, k, n;
    int act;
    void *dx, *dw_gate, *dw_up, *ws;
    int64_t dx_ld, dw_ld;
};

template <typename T>
int transpose(const void *in, int64_t in_ld, int64_t rows, int64_t cols, T *out, int64_t out_ld, hipStream_t s) {
    const int64_t across = (cols + 63) / 64, blocks = (rows + 63) / 64 * across;
    if (blocks == 0) return BYZ_OK;
    if (blocks > INT32_MAX / 256) return BYZ_EUNSUPPORTED;
    transpose_kernel<T><<<(unsigned)blocks, 256, 0, s>>>((const T *)in, in_ld, rows, cols, out, out_ld, (int)across);
    BYZ_HIP(hipGetLastError());
    return BYZ_OK;
}

template <typename T>
int backward(const Backward &b, hipStream_t s) {
    const Layout lay(b.m, b.k, b.n);
    T *ws = (T *)b.ws;
    if (b.m > 0 && b.n > 0) {
        const int64_t across = lay.np / 64, blocks = lay.mp / 64 * across;
        if (blocks > INT32_MAX / 256) return BYZ_EUNSUPPORTED;
        const Slopes v{b.dh, b.gate, b.up, b.dh_ld, b.gate_ld, b.m, b.n, lay.np, lay.mp, ws + lay.d, ws + lay.dt, b.act, (int)across};
        slopes_kernel<T><<<(unsigned)blocks, 256, 0, s>>>(v);
        BYZ_HIP(hipGetLastError());
    }
    int rc = BYZ_OK;
    if (b.dx && b.m > 0 && b.k > 0) {
        rc = transpose<T>(b.w_gate, b.w_ld, b.n, b.k, ws + lay.wt, 2 * lay.np, s);
        if (rc == BYZ_OK) rc = transpose<T>(b.w_up, b.w_ld, b.n, b.k, ws + lay.wt + lay.np, 2 * lay.np, s);
        if (rc != BYZ_OK) return rc;
        Product p{};
        p.a = ws + lay.d, p.a_ld = 2 * lay.np, p.b = ws + lay.wt, p.b_ld = 2 * lay.np;
        p.m = b.m, p.n = b.k, p.k = 2 * lay.np, p.out = b.dx, p.out_ld = b.dx_ld, p.split = b.m, p.pieces = true;
        rc = launch_product<T, false>(p, s);
    }
    if (rc == BYZ_OK && b.dw_gate && b.n > 0 && b.k > 0) {
        rc = transpose<T>(b.x, b.x_ld, b.m, b.k, ws + lay.xt, lay.mp, s);
        if (rc != BYZ_OK) return rc;
        // dgate's rows and dup's, a product each: neither writes over the padding between them
        for (int half = 0; half < 2 && rc == BYZ_OK; half++) {
            Product p{};
            p.a = ws + lay.dt + half * lay.np * lay.mp, p.a_ld = lay.mp, p.b = ws + lay.xt, p.b_ld = lay.mp;
            p.m = b.n, p.n = b.k, p.k = lay.mp, p.out = half ? b.dw_up : b.dw_gate, p.out_ld = b.dw_ld, p.split = b.n;
            p.pieces = true;
            rc = launch_product<T, false>(p, s);
        }
    }
    return rc;
}

bool matrix_ok(const void *at, int64_t rows, int64_t cols, int64_t ld, int elem = 2) {
    return rows == 0 || cols == 0 || (at && aligned(at, elem) && ld >= cols && extent_ok(rows, ld, cols));
}

}  // namespace

extern "C" int byz_gated_ffn(const void *x, int64_t x_ld, const void *w_gate, const void *w_up, int64_t w_ld,
                             int64_t m, int64_t k, int64_t n, int dtype, int act, void *h, int64_t h_ld,
                             float *gate_out, float *up_out, int64_t gate_ld, void *stream) {
    if (!sizes_ok(m, k, n) || !dtype_known(dtype) || !act_known(act) || !gate_out != !up_out) return BYZ_EINVAL;
    if (dtype == BYZ_F32) return BYZ_EUNSUPPORTED;
    if (!matrix_ok(x, m, k, x_ld) || !matrix_ok(w_gate, n, k, w_ld) || !matrix_ok(w_up, n, k, w_ld) || !matrix_ok(h, m, n, h_ld) ||
        (gate_out && (!matrix_ok(gate_out, m, n, gate_ld, 4) || !matrix_ok(up_out, m, n, gate_ld, 4))))
        return BYZ_EINVAL;
    if (m == 0 || n == 0) return BYZ_OK;
    Product p{};
    p.a = x, p.a_ld = x_ld, p.b = w_gate, p.b2 = w_up, p.b_ld = w_ld, p.m = m, p.n = n, p.k = k;
    p.out = h, p.out_ld = h_ld, p.gate = gate_out, p.up = up_out, p.gate_ld = gate_ld, p.act = act;
    p.pieces = aligned(x, 16) && aligned(w_gate, 16) && aligned(w_up, 16) && x_ld % 8 == 0 && w_ld % 8 == 0;
    return dtype == BYZ_BF16 ? forward<bf16>(p, (hipStream_t)stream) : forward<f16>(p, (hipStream_t)stream);
}

extern "C" size_t byz_gated_ffn_backward_workspace_bytes(int64_t m, int64_t k, int64_t n, int dtype) {
    if (!sizes_ok(m, k, n) || (dtype != BYZ_BF16 && dtype != BYZ_F16)) return 0;
    return (size_t)Layout(m, k, n).all * 2;
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
    if (workspace_bytes < (size_t)Layout(m, k, n).all * 2) return BYZ_ENOMEM;
    if (workspace_bytes && (!workspace || !aligned(workspace, 16))) return BYZ_ENOMEM;
    const Backward b{dh, x, w_gate, w_up, gate, up, dh_ld, x_ld, w_ld, gate_ld, m, k, n, act, dx, dw_gate, dw_up, workspace, dx_ld, dw_ld};
    return dtype == BYZ_BF16 ? backward<bf16>(b, (hipStream_t)stream) : backward<f16>(b, (hipStream_t)stream);
}

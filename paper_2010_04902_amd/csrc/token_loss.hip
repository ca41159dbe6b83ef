// Losses of tokens' log-probabilities, from logits (gfx950): the log-probabilities themselves, the clipped policy loss with its KL
// term, and the preference loss of pairs of sequences.
//
// All are functions of logp = (z_label - m) / T - log sum exp((z - m) / T), with m the row's largest logit, and all their gradients
// are w (onehot(label) - softmax(z / T)) with one weight w = (d loss / d logp) / T a row.  So there are three steps: a row's
// maximum and sum (one read), what the loss makes of logp (a few values a row, in fp64 from an fp32 sum), and the dense
// gradient (another read, and the write), which needs a row's m, log-sum, w and label and nothing else.
#include <algorithm>

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

// exp(g) - 1 - g: near 0 its series
__device__ __forceinline__ double exp_rest(double g) {
    if (!(fabs(g) < 0.5)) return exp_of(g) - 1.0 - g;
    double s = 1.0 / 479001600;  // 1 / 12!, and down to 1 / 2!
    double f = 479001600;
#pragma unroll
    for (int n = 12; n > 2; n--) f /= n, s = s * g + 1.0 / f;
    return s * g * g;
}

// The policy loss of a row and its derivative by logp.
__device__ __forceinline__ void policy(const Args &a, int64_t row, double logp, double &loss, double &slope) {
    const double advantage = a.advantage[row], r = exp_of(logp - (double)a.old[row]);
    const bool above = advantage >= 0.0 && r > (double)a.high, below = !(advantage >= 0.0) && r < (double)a.low;
    loss = -advantage * (above ? (double)a.high : below ? (double)a.low : r);
    slope = above || below ? 0.0 * advantage : -advantage * r;
    if (a.kl != 0.0f) {
        const double g = (double)a.ref[row] - logp, rest = exp_rest(g);
        loss += (double)a.kl * rest;
        slope -= (double)a.kl * (rest + g);
    }
}

// A row's results from its maximum and sum, by one thread; z is the label's logit.
__device__ __forceinline__ Terms finish(const Args &a, int64_t row, int32_t label, float m, float sum, float z) {
    const bool empty = label < 0;
    if (empty || m == -INFINITY) m = 0.0f;  // no token, or nothing but banned logits (or NaN, which is in the sum)
    const double log_sum = empty ? 0.0 : log_of(sum);
    double logp = empty ? 0.0 : label >= a.vocab ? NAN : ((double)z - (double)m) / (double)a.temperature - log_sum;
    Terms t{m, (float)log_sum, 0.0f, label};
    if (a.stats) a.stats[row * 2] = m, a.stats[row * 2 + 1] = (float)log_sum;
    if (a.logp) a.logp[row] = (float)logp;
    if (a.kind == kPolicy) {
        double loss = 0.0, slope = 0.0;
        if (!empty) policy(a, row, logp, loss, slope);
        if (a.loss) a.loss[row] = (float)loss;
        if (a.dloss && !empty) t.w = (float)((double)a.dloss[row] * slope / (double)a.temperature);
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
            policy(a, row, (z - (double)t.m) / (double)a.temperature - (double)t.log_sum, loss, slope);
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
        t.w = (float)(slope / (double)a.temperature);
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
            const double w = (double)a.beta * slope * (double)a.dloss[pair] / (double)a.temperature;
            for (int64_t i = b0 + (int64_t)threadIdx.x; i < b2; i += 256)
                if (a.terms[i].label >= 0) a.terms[i].w = (float)(i < b1 ? w : -w);
        }
    }
}

// The dense gradient: `parts` blocks a row.  Rows without a token or weight are not read.
template <typename T>
__global__ __launch_bounds__(256) void gradient_kernel(Args a, int64_t parts, int64_t each) {
    constexpr int V = 16 / sizeof(T);
    const int64_t total = a.rows * parts;
    for (int64_t block = blockIdx.x; block < total; block += gridDim.x) {
        const int64_t row = block / parts, part = block - row * parts;
        const Terms t = a.terms[row];
        const Row<T> r(a.logits, row, a.ld, a.vocab);
        T *out = (T *)a.dlogits + row * a.dlogits_ld;
        const int64_t from = part * each, to = std::min(r.vectors, from + each);
        const bool last = part == parts - 1 && (int)threadIdx.x < r.tail;
        const int64_t edge = r.edge(threadIdx.x);
        if (t.w == 0.0f) {
            for (int64_t i = from + threadIdx.x; i < to; i += 256) put_words(out + i * V, Words<T, V>::of([](int) { return 0.0f; }));
            if (last) out[edge] = (T)0.0f;
            continue;
        }
        const Softmax<T> q((double)t.m, (double)t.log_sum, (double)a.temperature, -t.w);
        auto write = [&](auto odd) {
            for (int64_t i = from + threadIdx.x; i < to; i += 256) {
                const Words<T, V> v = r.template vector_of<odd.value>(i);
                put_words(out + i * V, Words<T, V>::of([&](int e) { return q.weighted(v[e]); }));
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

// ------------------------------------------------------------------ launches

size_t terms_bytes(int64_t rows) { return (size_t)rows * sizeof(Terms); }
size_t workspace_of(int64_t rows) { return terms_bytes(rows) + (size_t)rows * sizeof(double); }

template <typename T>
int launch_rows(const Args &a, hipStream_t s) {
    rows_kernel<T, 256><<<(unsigned)std::min(a.rows, kMaxGrid), 256, 0, s>>>(a);
    BYZ_HIP(hipGetLastError());
    return BYZ_OK;
}

template <typename T>
int launch_gradient(const Args &a, hipStream_t s) {
    const int64_t vectors = a.vocab * (int64_t)sizeof(T) / 16, each = 1024;
    const int64_t parts = std::max<int64_t>(1, (vectors + each - 1) / each);
    gradient_kernel<T><<<(unsigned)std::min(a.rows * parts, kMaxGrid), 256, 0, s>>>(a, parts, each);
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
    return a;
}

// The checks that all calls share, and the workspace's parts.
int check(Args &a, int dtype, bool gradient, void *workspace, size_t bytes) {
    if (!sizes_ok(a.rows, a.vocab, dtype) || !(a.temperature > 0.0f) || !real(a.temperature)) return BYZ_EINVAL;
    if (a.rows == 0) return BYZ_OK;
    if (!a.logits || !a.label || !aligned(a.logits, dtype_size(dtype)) || !aligned(a.label, 4) || a.ld < a.vocab ||
        !extent_ok(a.rows, a.ld, a.vocab) || !floats_ok(a.stats) || !floats_ok(a.given_stats))
        return BYZ_EINVAL;
    if (gradient && (!a.dlogits || !a.dloss || !floats_ok(a.dloss) || !aligned(a.dlogits, dtype_size(dtype)) || a.dlogits_ld < a.vocab ||
                     !extent_ok(a.rows, a.dlogits_ld, a.vocab)))
        return BYZ_EINVAL;
    if (!workspace || !aligned(workspace, 16) || bytes < workspace_of(a.rows)) return BYZ_ENOMEM;
    a.terms = (Terms *)workspace;
    a.logp64 = (double *)((char *)workspace + terms_bytes(a.rows));
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
    return sizes_ok(rows, vocab, dtype) ? workspace_of(rows) : 0;
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

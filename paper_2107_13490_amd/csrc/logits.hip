// Log probabilities of given classes with entropy and the largest logits, and softmax cross entropy with its gradient as
// fixed-point codes.
#include <algorithm>

#include "common.hpp"
#include "context.hpp"

namespace adapt {

constexpr int kRowThreads = 256;
constexpr int kMaxTop = 32;

struct LogitArgs {
    const void *logits;
    uint64_t rows, classes, ld;
    int fl;
    const int64_t *labels;
    float *logp, *lse, *entropy;
    int topk;
    int32_t *top_index;
    float *top_logp;
    // cross entropy
    const float *weights;
    void *grad;
    uint64_t ldg;
    int wl_g, fl_g, mode;
    uint64_t seed, stream;
};

template <typename T>
__device__ __forceinline__ double value_of(T l, int fl) { return ldexp((double)l, -fl); }

// a logit's place among those of its row: larger first, then the lower index
template <typename T>
__device__ __forceinline__ uint64_t key_of(T l, uint32_t j) { return ((uint64_t)((uint32_t)(int32_t)l ^ 0x80000000u) << 32) | (0x7fffffffu - j); }
template <>
__device__ __forceinline__ uint64_t key_of<float>(float l, uint32_t j)
{
    const float v = l != l ? -INFINITY : l == 0.0f ? 0.0f : l;
    const uint32_t b = __float_as_uint(v);
    return ((uint64_t)((b & 0x80000000u) ? ~b : b | 0x80000000u) << 32) | (0x7fffffffu - j);
}

template <typename V, typename Op>
__device__ __forceinline__ V block_reduce(V v, Op op)
{
    __shared__ V part[kRowThreads / kWave];
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v = op(v, __shfl_xor(v, off, 64));
    if ((threadIdx.x & (kWave - 1)) == 0) part[threadIdx.x / kWave] = v;
    __syncthreads();
    v = part[0];
    for (int w = 1; w < kRowThreads / kWave; ++w) v = op(v, part[w]);
    __syncthreads();
    return v;
}

// largest value of a row (-inf: no class possible; NaN: a NaN or +inf among the logits) and the sums of exp(x - m) and (x - m) exp(x - m)
struct RowStats { double m, s, e; };

template <typename T>
__device__ __forceinline__ RowStats row_stats(const T *row, uint64_t classes, int fl)
{
    RowStats r;
    double m = -INFINITY;
    int bad = 0;
    for (uint64_t j = threadIdx.x; j < classes; j += kRowThreads) {
        const double x = value_of(row[j], fl);
        bad |= !(x < INFINITY);
        m = fmax(m, x);
    }
    r.m = block_reduce(m, [](double a, double b) { return fmax(a, b); });
    if (block_reduce(bad, [](int a, int b) { return a | b; })) r.m = NAN;
    r.s = r.e = 0.0;
    for (uint64_t j = threadIdx.x; j < classes; j += kRowThreads) {
        const double d = value_of(row[j], fl) - r.m;
        if (!(d > -INFINITY)) continue;
        const double t = exp(d);
        r.s += t;
        r.e += t * d;
    }
    const auto add = [](double a, double b) { return a + b; };
    r.s = block_reduce(r.s, add);
    r.e = block_reduce(r.e, add);
    return r;
}

__device__ __forceinline__ float log_prob(double x, const RowStats &r)
{
    return r.m == -INFINITY ? -INFINITY : (float)(x - r.m - log(r.s));
}

template <typename T>
__device__ __forceinline__ float label_log_prob(const T *row, int64_t label, uint64_t classes, int fl, const RowStats &r)
{
    if (label < 0) return 0.0f;
    if ((uint64_t)label >= classes || r.m != r.m) return NAN;
    return log_prob(value_of(row[label], fl), r);
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads) log_probs_kernel(const LogitArgs a)
{
    for (uint64_t i = blockIdx.x; i < a.rows; i += gridDim.x) {
        const T *row = static_cast<const T *>(a.logits) + i * a.ld;
        const RowStats r = row_stats(row, a.classes, a.fl);
        if (threadIdx.x == 0) {
            const bool none = r.m == -INFINITY;
            if (a.lse) a.lse[i] = none ? -INFINITY : (float)(r.m + log(r.s));
            if (a.entropy) a.entropy[i] = r.m != r.m ? NAN : none ? 0.0f : (float)(log(r.s) - r.e / r.s);
            if (a.logp) a.logp[i] = label_log_prob(row, a.labels[i], a.classes, a.fl, r);
        }
        uint64_t last = ~0ull;
        for (int k = 0; k < a.topk; ++k) {
            uint64_t best = 0;
            for (uint64_t j = threadIdx.x; j < a.classes; j += kRowThreads) {
                const uint64_t key = key_of(row[j], (uint32_t)j);
                if (key < last && key > best) best = key;
            }
            last = block_reduce(best, [](uint64_t x, uint64_t y) { return x > y ? x : y; });
            if (threadIdx.x == 0) {
                const uint32_t j = 0x7fffffffu - (uint32_t)last;
                a.top_index[i * a.topk + k] = (int32_t)j;
                a.top_logp[i * a.topk + k] = r.m != r.m ? NAN : log_prob(value_of(row[j], a.fl), r);
            }
        }
    }
}

template <typename T, typename G>
__global__ void __launch_bounds__(kRowThreads) cross_entropy_kernel(const LogitArgs a)
{
    const double qmin = -ldexp(1.0, a.wl_g - 1), qmax = ldexp(1.0, a.wl_g - 1) - 1.0;
    for (uint64_t i = blockIdx.x; i < a.rows; i += gridDim.x) {
        const T *row = static_cast<const T *>(a.logits) + i * a.ld;
        G *grad = static_cast<G *>(a.grad) + i * a.ldg;
        const RowStats r = row_stats(row, a.classes, a.fl);
        const int64_t label = a.labels[i];
        if (threadIdx.x == 0 && a.logp) a.logp[i] = label_log_prob(row, label, a.classes, a.fl, r);
        const bool counts = label >= 0 && (uint64_t)label < a.classes && r.m > -INFINITY;
        const double scale = counts ? (a.weights ? (double)a.weights[i] : 1.0) * ldexp(1.0, a.fl_g) / r.s : 0.0;
        for (uint64_t j = threadIdx.x; j < a.classes; j += kRowThreads) {
            long long q = 0;
            if (counts) {
                double t = exp(value_of(row[j], a.fl) - r.m);
                if (j == (uint64_t)label) t -= r.s;
                const double y = fmin(fmax(t * scale, qmin), qmax);
                q = ((long long)floor(y * 65536.0) + (long long)rounding_bits_of(a.seed, a.stream, i * a.classes + j, a.mode)) >> 16;
                q = q > (long long)qmax ? (long long)qmax : q;
            }
            grad[j] = (G)q;
        }
    }
}

size_t ws_need_log_probs(int, uint64_t, uint64_t, int, adapt_fmt) { return 16; }
size_t ws_need_cross_entropy(int, uint64_t, uint64_t, adapt_fmt, adapt_fmt) { return 16; }

bool logits_ok(uint64_t rows, uint64_t classes, uint64_t ld)
{
    return classes >= 1 && classes <= (1ull << 30) && ld >= classes && rows < (1ull << 31) && ld <= (1ull << 40) &&
           (rows == 0 || ld <= (1ull << 40) / rows);
}

}  // namespace adapt

using namespace adapt;

static int logit_bytes(adapt_fmt f) { return f.wl == ADAPT_WL_FP32 ? 4 : storage_bytes(f); }

extern "C" int adapt_log_probs(adapt_ctx *ctx, const void *logits, adapt_fmt f, size_t rows, size_t classes, size_t ld, const int64_t *labels,
                               float *logp, float *lse, float *entropy, int topk, int32_t *top_index, float *top_logp)
{
    if (!ctx || !(f.wl == ADAPT_WL_FP32 || fmt_ok_wide(f)) || !logits_ok(rows, classes, ld)) return ADAPT_EINVAL;
    if (topk < 0 || topk > kMaxTop || (size_t)topk > classes || (topk > 0 && rows > 0 && (!top_index || !top_logp))) return ADAPT_EINVAL;
    if (!on_current_device(ctx)) return ADAPT_EINVAL;
    if (rows == 0) return ADAPT_OK;
    if (!logits || !aligned_to(logits, logit_bytes(f)) || (logp && !labels) || !aligned_to(labels, 8) || !aligned_to(logp, 4) ||
        !aligned_to(lse, 4) || !aligned_to(entropy, 4) || !aligned_to(top_index, 4) || !aligned_to(top_logp, 4))
        return ADAPT_EINVAL;
    LogitArgs a = {};
    a.logits = logits;
    a.rows = rows; a.classes = classes; a.ld = ld;
    a.fl = f.wl == ADAPT_WL_FP32 ? 0 : f.fl;
    a.labels = labels; a.logp = logp; a.lse = lse; a.entropy = entropy;
    a.topk = topk; a.top_index = top_index; a.top_logp = top_logp;
    const dim3 grid((unsigned)std::min<size_t>(rows, 1u << 20)), block(kRowThreads);
    if (f.wl == ADAPT_WL_FP32) hipLaunchKernelGGL(log_probs_kernel<float>, grid, block, 0, ctx->stream, a);
    else if (f.wl <= 8) hipLaunchKernelGGL(log_probs_kernel<int8_t>, grid, block, 0, ctx->stream, a);
    else if (f.wl <= 16) hipLaunchKernelGGL(log_probs_kernel<int16_t>, grid, block, 0, ctx->stream, a);
    else hipLaunchKernelGGL(log_probs_kernel<int32_t>, grid, block, 0, ctx->stream, a);
    return hip_status(ctx, hipGetLastError());
}

template <typename T>
static void launch_cross_entropy(adapt_ctx *ctx, const LogitArgs &a)
{
    const dim3 grid((unsigned)std::min<uint64_t>(a.rows, 1u << 20)), block(kRowThreads);
    if (a.wl_g <= 8) hipLaunchKernelGGL((cross_entropy_kernel<T, int8_t>), grid, block, 0, ctx->stream, a);
    else if (a.wl_g <= 16) hipLaunchKernelGGL((cross_entropy_kernel<T, int16_t>), grid, block, 0, ctx->stream, a);
    else hipLaunchKernelGGL((cross_entropy_kernel<T, int32_t>), grid, block, 0, ctx->stream, a);
}

extern "C" int adapt_cross_entropy(adapt_ctx *ctx, const void *logits, adapt_fmt f, size_t rows, size_t classes, size_t ld, const int64_t *labels,
                                   const float *weights, adapt_fmt fg, adapt_rng rng, void *dlogits, size_t ldg, float *logp)
{
    if (!ctx || !(f.wl == ADAPT_WL_FP32 || fmt_ok_wide(f)) || !fmt_ok_wide(fg) || !logits_ok(rows, classes, ld) || !logits_ok(rows, classes, ldg))
        return ADAPT_EINVAL;
    if (rng.mode != ADAPT_SR && rng.mode != ADAPT_RN_HALF_UP) return ADAPT_EINVAL;
    if (!on_current_device(ctx)) return ADAPT_EINVAL;
    if (rows == 0) return ADAPT_OK;
    if (!logits || !labels || !dlogits || !aligned_to(logits, logit_bytes(f)) || !aligned_to(labels, 8) || !aligned_to(weights, 4) ||
        !aligned_to(dlogits, storage_bytes(fg)) || !aligned_to(logp, 4))
        return ADAPT_EINVAL;
    LogitArgs a = {};
    a.logits = logits;
    a.rows = rows; a.classes = classes; a.ld = ld;
    a.fl = f.wl == ADAPT_WL_FP32 ? 0 : f.fl;
    a.labels = labels; a.logp = logp; a.weights = weights;
    a.grad = dlogits; a.ldg = ldg;
    a.wl_g = fg.wl; a.fl_g = fg.fl; a.mode = rng.mode; a.seed = rng.seed; a.stream = rng.stream;
    if (f.wl == ADAPT_WL_FP32) launch_cross_entropy<float>(ctx, a);
    else if (f.wl <= 8) launch_cross_entropy<int8_t>(ctx, a);
    else if (f.wl <= 16) launch_cross_entropy<int16_t>(ctx, a);
    else launch_cross_entropy<int32_t>(ctx, a);
    return hip_status(ctx, hipGetLastError());
}

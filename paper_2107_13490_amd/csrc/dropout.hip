// Dropout of fixed-point codes: one draw of the generator decides whether an element stays and how its scaled value is
// rounded, and no mask is stored (the gradient draws the same bits again).
//
// With R = 16 random bits, T of the 65536 draws dropped and K = 65536 - T kept, the scaled value is X/K, X = x 2^(16+s).
// Given R >= T the number u = R - T is uniform on 0..K-1, so floor((X + u)/K) is X/K rounded up with probability
// (X mod K)/K: its expectation over all draws is K/65536 X/K = x 2^s, exactly.
#include <cmath>

#include <algorithm>

#include "common.hpp"
#include "context.hpp"

namespace adapt {

constexpr int kDropThreads = 256;

struct DropArgs {
    const void *x, *res;
    void *out;
    uint64_t n;
    int up;                  // X = floor(x 2^up)
    int res_up;              // fractional bits that the residual gains
    int drop, keep;          // T, K
    int es_x, es_res, es_o, wl, mode;
    uint64_t seed, stream;
};

__device__ __forceinline__ long long code_at(const void *q, int es, uint64_t i)
{
    return es == 1 ? static_cast<const int8_t *>(q)[i] : es == 2 ? static_cast<const int16_t *>(q)[i] : static_cast<const int32_t *>(q)[i];
}

// |X| <= 2^62 (x has 32 bits, up <= 31) and |res 2^res_up| <= 2^62, the positive ends left out: the sum fits 64 bits
__device__ __forceinline__ long long drop_one(long long x, int up, int drop, int keep, uint32_t r16, int mode)
{
    if ((int)r16 < drop) return 0;
    const long long X = up >= 0 ? (long long)((unsigned long long)x << up) : x >> -up;
    const long long t = X + (mode == ADAPT_SR ? (int)r16 - drop : keep >> 1);
    const long long q = t / keep;
    return q - (q * keep > t);                             // towards minus infinity
}

__global__ void __launch_bounds__(kDropThreads) dropout_kernel(const DropArgs a)
{
    const long long hi = (1ll << (a.wl - 1)) - 1, lo = -hi - 1;
    for (uint64_t i = (uint64_t)blockIdx.x * kDropThreads + threadIdx.x; i < a.n; i += (uint64_t)gridDim.x * kDropThreads) {
        const uint32_t r = rounding_bits_of(a.seed, a.stream, i, ADAPT_SR);
        long long y = drop_one(code_at(a.x, a.es_x, i), a.up, a.drop, a.keep, r, a.mode);
        if (a.res) y += (long long)((unsigned long long)code_at(a.res, a.es_res, i) << a.res_up);
        y = min(max(y, lo), hi);
        if (a.es_o == 1) static_cast<int8_t *>(a.out)[i] = (int8_t)y;
        else if (a.es_o == 2) static_cast<int16_t *>(a.out)[i] = (int16_t)y;
        else static_cast<int32_t *>(a.out)[i] = (int32_t)y;
    }
}

}  // namespace adapt

using namespace adapt;

extern "C" int adapt_dropout(adapt_ctx *ctx, const void *x, adapt_fmt fx, size_t n, double p, adapt_fmt fo, adapt_rng rng,
                             const void *res, adapt_fmt fres, void *out)
{
    if (!ctx || !fmt_ok_wide(fx) || !fmt_ok_wide(fo) || (rng.mode != ADAPT_SR && rng.mode != ADAPT_RN_HALF_UP)) return ADAPT_EINVAL;
    if (!(p >= 0.0 && p < 1.0) || n > ((uint64_t)1 << 40) || (res && !fmt_ok_wide(fres))) return ADAPT_EINVAL;
    const int drop = (int)std::floor(p * 65536.0 + 0.5);
    if (drop > 65535) return ADAPT_EINVAL;
    if (fo.fl - fx.fl > 15 || (res && fo.fl < fres.fl)) return ADAPT_EUNSUPPORTED;
    if (!on_current_device(ctx)) return ADAPT_EINVAL;
    if (n == 0) return ADAPT_OK;
    const int es_x = storage_bytes(fx), es_o = storage_bytes(fo), es_r = res ? storage_bytes(fres) : 1;
    if (!x || !out || !aligned_to(x, es_x) || !aligned_to(out, es_o) || !aligned_to(res, es_r)) return ADAPT_EINVAL;
    DropArgs a = {x, res, out, n, 16 + fo.fl - fx.fl, res ? fo.fl - fres.fl : 0, drop, 65536 - drop, es_x, es_r, es_o, fo.wl, rng.mode, rng.seed, rng.stream};
    const int grid = (int)std::min<uint64_t>((n + kDropThreads - 1) / kDropThreads, (uint64_t)ctx->num_cu * 8);
    hipLaunchKernelGGL(dropout_kernel, dim3(grid), dim3(kDropThreads), 0, ctx->stream, a);
    return hip_status(ctx, hipGetLastError());
}

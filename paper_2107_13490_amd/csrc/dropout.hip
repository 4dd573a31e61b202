// Dropout of fixed-point codes: one draw of the generator decides whether an element stays and how its scaled value is
// rounded, and no mask is stored (the gradient draws the same bits again).
//
// With R = 16 random bits, T of the 65536 draws dropped and K = 65536 - T kept, the scaled value is X/K, X = x 2^(16+s).
// Given R >= T the number u = R - T is uniform on 0..K-1, so floor((X + u)/K) is X/K rounded up with probability
// (X mod K)/K: its expectation over all draws is K/65536 X/K = x 2^s, exactly.
#include <cmath>

#include <algorithm>

#include "code_vec.hpp"
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

// |X| <= 2^62 (x has 32 bits, 0 <= up <= 31) and |res 2^res_up| <= 2^62, the positive ends left out: the sum fits 64 bits
__device__ __forceinline__ long long drop_one(long long x, int up, int drop, int keep, uint32_t r16, int mode)
{
    if ((int)r16 < drop) return 0;
    const long long X = (long long)((unsigned long long)x << up);
    const long long t = X + (mode == ADAPT_SR ? (int)r16 - drop : keep >> 1);
    const long long q = t / keep;
    return q - (q * keep > t);                             // towards minus infinity
}

// What bounds it: the issue of vector instructions at 8 bits (about 11 per element, 5 of them the generator's 19 products and 20 three-way
// xors per block of eight; 4 more with a residual), memory above.  33.5 M codes, us: 8 -> 8 bits 15.8 (4.2 TB/s), with an 8-bit residual
// 22 to 25 (4.0 to 4.5), 16 -> 16 bits 27 (4.95; a copy on this card runs at 5.0).
//
// How floor((X + u)/K) is found; all of them exactly.  33.5 M codes of 8 bits, us: BY_TABLE 15.8, BY_F64 28; of 16 bits:
// BY_I32 27, BY_F64 34.  The faster form is taken wherever it is exact; 64-bit integers (8.4 M codes of 32 bits 50, BY_F64 12) where none is.
//   BY_TABLE  8-bit x: the quotient and the rest of X/K for each of its 256 values, in LDS.  An entry is q 2^16 + r with r + R
//             carrying into the quotient where R is among the r largest draws, so that adding R to it rounds.
//   BY_I32    |X + u| < 2^31, K >= 2^11: an fp32 quotient is off by less than one, and the rest says by what.
//   BY_F64    |X + u| < 2^51: with a half added the sum is still exact, and its product with 1/K off by less than
//             2^51 2^-52 / K, half of what separates it from a whole number.
enum { BY_TABLE, BY_I32, BY_F64 };

struct DropConst {
    double d_up, d_inv, d_add;       // 2^up, 1/K, 1/2 and what makes R (nearest: 0) the u of the rule
    int down;                        // BY_F64: bits that x loses first (its fractional bits beyond 16 more than the output's)
    float f_inv;
    int drop, keep, up;
};

// RES: whether a residual is added, where that costs much (BY_F64 finds out by itself)
template <typename TX, typename TO, int HOW, bool RES>
__global__ void __launch_bounds__(kDropThreads) dropout_kernel(const DropArgs a, const DropConst k)
{
    const TX *x = static_cast<const TX *>(a.x);
    TO *out = static_cast<TO *>(a.out);
    const double lo = -ldexp(1.0, a.wl - 1), hi = ldexp(1.0, a.wl - 1) - 1.0;
    const int ilo = (int)lo, ihi = (int)hi;
    const double res_scale = ldexp(1.0, a.res_up);
    const bool has_res = HOW == BY_F64 ? a.res != nullptr : RES, nearest = HOW == BY_F64 && a.mode != ADAPT_SR;
    __shared__ uint32_t table[HOW == BY_TABLE ? 256 : 1];
    if constexpr (HOW == BY_TABLE) {
        static_assert(kDropThreads == 256, "an entry per thread");
        const double X = (double)(int8_t)threadIdx.x * k.d_up;
        int q = (int)floor((X + 0.5) * k.d_inv);
        int r = (int)(X - (double)q * (double)k.keep);
        if (!RES && (q < ilo || q >= ihi)) { q = q < ilo ? ilo : ihi; r = 0; }        // saturated here where nothing is added
        table[threadIdx.x] = ((uint32_t)q << 16) | (uint32_t)r;
        __syncthreads();
    }
    auto one = [&](int c, int res, uint32_t r16) -> int {
        const bool stays = (int)r16 >= k.drop;
        int q;
        if constexpr (HOW == BY_TABLE) {
            q = (int)(table[c & 255] + r16) >> 16;
        } else if constexpr (HOW == BY_I32) {
            const int n = (int)(((uint32_t)c << k.up) + r16) - k.drop;
            q = (int)floorf((float)n * k.f_inv);
            const int rest = n - __mul24(q, k.keep);
            q += (rest >= k.keep) - (rest < 0);
        } else {
            double y = floor(fma((double)(c >> k.down), k.d_up, (nearest ? 0.0 : (double)r16) + k.d_add) * k.d_inv);
            y = stays ? y : 0.0;
            if (has_res) y += (double)res * res_scale;                   // beyond 2^53 it saturates, rounded or not
            return (int)fmin(fmax(y, lo), hi);
        }
        q = stays ? q : 0;
        if (RES) q += (int)((uint32_t)res << a.res_up);
        return HOW == BY_TABLE && !RES ? q : min(max(q, ilo), ihi);
    };
    auto residual = [&](uint64_t g, int (&r)[8]) {
        if (a.es_res == 1) load8(static_cast<const int8_t *>(a.res) + 8 * g, r);
        else if (a.es_res == 2) load8(static_cast<const int16_t *>(a.res) + 8 * g, r);
        else load8(static_cast<const int32_t *>(a.res) + 8 * g, r);
    };
    auto group = [&](uint64_t g, const int (&c)[8], const int (&r)[8]) {
        const u32x4 blk = rounding_block(a.seed, a.stream, g);
        if constexpr (HOW == BY_TABLE && !RES && sizeof(TO) < 4) {
            uint32_t sum[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const uint32_t r16 = lane16(blk, e);
                sum[e] = (int)r16 >= k.drop ? table[c[e] & 255] + r16 : 0;
            }
            store_upper<false>(out + 8 * g, sum);
            return;
        }
        int v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = one(c[e], r[e], lane16(blk, e));
        store8(out + 8 * g, v);
    };
    const uint64_t full = a.n >> 3, stride = (uint64_t)gridDim.x * kDropThreads;
    uint64_t g = (uint64_t)blockIdx.x * kDropThreads + threadIdx.x;
    for (; g + stride < full; g += 2 * stride) {
        int c0[8], c1[8], r0[8] = {}, r1[8] = {};
        load8(x + 8 * g, c0);
        load8(x + 8 * (g + stride), c1);
        if (has_res) { residual(g, r0); residual(g + stride, r1); }
        group(g, c0, r0);
        group(g + stride, c1, r1);
    }
    if (g < full) {
        int c[8], r[8] = {};
        load8(x + 8 * g, c);
        if (has_res) residual(g, r);
        group(g, c, r);
        g += stride;
    }
    if (g == full)                                         // the last, incomplete group has an owner too
        for (uint64_t i = full << 3; i < a.n; ++i)
            out[i] = (TO)one(x[i], has_res ? (int)code_at(a.res, a.es_res, i) : 0, rounding_bits_of(a.seed, a.stream, i, ADAPT_SR));
}

// X beyond 2^50: 64-bit integers, an element per thread
__global__ void __launch_bounds__(kDropThreads) dropout_i64_kernel(const DropArgs a)
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

template <typename TX, int HOW, bool RES>
static void launch(adapt_ctx *ctx, dim3 grid, const DropArgs &a, const DropConst &k)
{
    const dim3 block(kDropThreads);
    if (a.es_o == 1) hipLaunchKernelGGL((dropout_kernel<TX, int8_t, HOW, RES>), grid, block, 0, ctx->stream, a, k);
    else if (a.es_o == 2) hipLaunchKernelGGL((dropout_kernel<TX, int16_t, HOW, RES>), grid, block, 0, ctx->stream, a, k);
    else hipLaunchKernelGGL((dropout_kernel<TX, int32_t, HOW, RES>), grid, block, 0, ctx->stream, a, k);
}

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
    // a code may take the place of the one that it is made of, and of no other
    const auto in_the_way = [&](const void *in, int es) { return !(in == out && es == es_o) && rows_overlap(in, n * es, 0, out, n * es_o, 0, 1); };
    if (in_the_way(x, es_x) || (res && in_the_way(res, es_r))) return ADAPT_EINVAL;
    const int up = 16 + fo.fl - fx.fl, keep = 65536 - drop;
    const DropArgs a = {x, res, out, n, up, res ? fo.fl - fres.fl : 0, drop, keep, es_x, es_r, es_o, fo.wl, rng.mode, rng.seed, rng.stream};
    const bool nearest = rng.mode != ADAPT_SR;
    const DropConst k = {std::ldexp(1.0, std::max(up, 0)), 1.0 / keep, 0.5 + (nearest ? keep >> 1 : -drop), std::max(-up, 0), 1.0f / (float)keep, drop, keep, up};
    const uint64_t groups = (n + 7) >> 3;
    const dim3 grid((unsigned)std::min<uint64_t>((groups + kDropThreads - 1) / kDropThreads, (uint64_t)ctx->num_cu * 8)), block(kDropThreads);
    const bool in_32 = !nearest && (!res || fres.wl - 1 + a.res_up <= 29);      // the residual and its sum with a quotient
    const bool table = in_32 && fx.wl <= 8 && up >= 0 && std::ldexp(1.0, fx.wl - 1 + up) < 32767.0 * keep;
    const bool i32 = in_32 && fx.wl <= 16 && up >= 0 && fx.wl - 1 + up <= 30 && keep >= 2048;
    if (fx.wl - 1 + up > 50) hipLaunchKernelGGL(dropout_i64_kernel, grid, block, 0, ctx->stream, a);
    else if (fx.wl > 16) launch<int32_t, BY_F64, true>(ctx, grid, a, k);
    else if (fx.wl > 8) {
        if (!i32) launch<int16_t, BY_F64, true>(ctx, grid, a, k);
        else if (res) launch<int16_t, BY_I32, true>(ctx, grid, a, k);
        else launch<int16_t, BY_I32, false>(ctx, grid, a, k);
    } else {
        if (!table) launch<int8_t, BY_F64, true>(ctx, grid, a, k);
        else if (res) launch<int8_t, BY_TABLE, true>(ctx, grid, a, k);
        else launch<int8_t, BY_TABLE, false>(ctx, grid, a, k);
    }
    return hip_status(ctx, hipGetLastError());
}

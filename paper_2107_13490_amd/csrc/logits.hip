// Log probabilities of given classes with entropy and the largest logits, and softmax cross entropy with its gradient as
// fixed-point codes.
#include <algorithm>

#include "code_vec.hpp"
#include "common.hpp"
#include "context.hpp"

namespace adapt {

constexpr int kMaxTop = 32;

struct LogitArgs {
    const void *logits;
    uint64_t row0;               // first row of the launch
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

// The order of logits as that of 32-bit numbers: a NaN counts as -inf, -0 as 0
__device__ __forceinline__ uint32_t order_of(int v) { return (uint32_t)v ^ 0x80000000u; }
__device__ __forceinline__ uint32_t order_of(float v)
{
    v = v != v ? -INFINITY : v == 0.0f ? 0.0f : v;
    const uint32_t b = __float_as_uint(v);
    return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
// larger first, then the lower index; never 0 (indices are below 2^30)
__device__ __forceinline__ uint64_t key_of(uint32_t order, uint32_t index) { return ((uint64_t)order << 32) | (0x7fffffffu - index); }

// The logarithm of a sum of exponentials.  log_of_sum is good to 2^-48 of itself: with q = (m - 1)/(m + 1) for the mantissa m, taken between
// the roots of 1/2 and 2, log m is 2 atanh q = 2 (q + q^3/3 + .. + q^17/17), the next term 2^-50 of it; the quotient comes from the
// device's reciprocal (23 bits) by two Newton steps.  The cross entropy's sums have 64 bits, and its loss keeps them (256 x 100 3.8 us;
// 4.2 with the general logarithm, 3.7 with fp32).  Sums of fp32 exponentials take the fp32 logarithm of a mantissa between 1 and 2, which is
// good to 2^-23 (absolutely, where the result is below 1) and exact for 1 (128 x 10 log probabilities 3.4 us, in fp64 3.6).
__device__ __forceinline__ double log_of_fp32_sum(double s)
{
    int k;
    const float m = (float)frexp(s, &k);
    return fma((double)(k - 1), 0.69314718055994530942, (double)logf(m + m));
}
__device__ __forceinline__ double log_of_sum(double s)
{
    int k;
    double m = frexp(s, &k);
    if (m < 0.70710678118654752) { m += m; --k; }
    const double f = m - 1.0, d = m + 1.0;
    double c = __builtin_amdgcn_rcp(d);
    c = fma(c, fma(-d, c, 1.0), c);
    double q = f * c;
    q = fma(c, fma(-d, q, f), q);
    const double z = q * q, z2 = z * z, z4 = z2 * z2;
    const double lo = fma(fma(z, 1.0 / 9, 1.0 / 7), z2, fma(z, 1.0 / 5, 1.0 / 3));
    const double hi = fma(fma(z, 1.0 / 17, 1.0 / 15), z2, fma(z, 1.0 / 13, 1.0 / 11));
    const double p = fma(hi, z4, lo);
    q += q;
    return fma((double)k, 0.69314718055994530942, fma(q * z, p, q));
}

// ---------------------------------------------------------------------------------------------
// Cross entropy.  A block takes a row, or one chunk of a long one: the sum of the exponentials (with the largest logit before it
// where the format's whole range does not do as a reference), then the codes, both in 64 bits, since a code is a floor.  Elements
// come in units that start where the generator's blocks of eight start, so that a unit takes whole blocks whatever the number of
// classes; in a dense tensor units are aligned vectors, too.  What a row has before its first and behind its last whole unit are
// its edges, one element per thread.
// What bounds it: the two sweeps and the codes in memory, and at 8 bits as much the issue of 13 instructions per element, 5 of them the
// generator's.  The rows in flight exceed an XCD's L2, so the second sweep comes from memory as well; rows kept in LDS or registers
// leave too few wavefronts (8192 x 32000 of 8 bits 126 -> 131 us, 2047 x 65531 of 16 bits 143 -> 162).  us (TB/s of both sweeps and the
// codes): 8192 x 32000, 8 -> 8 bits 123 (6.4), 1535 x 65531, 16 -> 16 bits 118 (5.7), 922 of 1024 x 50001, fp32 -> 8 bits 87 (4.8); a copy runs at 5.0.
// ---------------------------------------------------------------------------------------------
template <typename T> constexpr int kUnit = sizeof(T) == 1 ? 16 : 8;      // elements
template <typename T> constexpr int kWords = kUnit<T> * (int)sizeof(T) / 4;
constexpr int kMostThreads = 1024;

template <typename T>
__device__ __forceinline__ T unit_get(const uint32_t (&w)[kWords<T>], int e)
{
    if constexpr (sizeof(T) == 1) return (T)(w[e >> 2] >> (8 * (e & 3)));
    else if constexpr (sizeof(T) == 2) return (T)(w[e >> 1] >> (16 * (e & 1)));
    else return __builtin_bit_cast(T, w[e]);
}

// exp in fp64 of a number of at most 700: 2^(n/256) e^r, |r| <= ln 2 / 512, with a table of the 256 roots and four terms (the
// next is 4e-17).  It ends as fp64 does: subnormal below -708, 0 below -745.2 and for -inf (a class of p = 0 has a gradient of 0, and
// not of a little below 0 under a negative weight).
__device__ __forceinline__ double exp_by_roots(double d, const double *roots)
{
    d = fmax(d, -800.0);
    const double shifted = fma(d, 369.32993046757462711, 6755399441055744.0);      // 256 / ln 2; 1.5 2^52 leaves n in the low word
    const int n = __double2loint(shifted);
    const double r = fma(shifted - 6755399441055744.0, -0.0027076061740622863, d); // ln 2 / 256
    double p = fma(r, 1.0 / 24.0, 1.0 / 6.0);
    p = fma(p, r, 0.5);
    p = fma(p, r, 1.0);
    p = fma(p, r, 1.0);
    return ldexp(p * roots[n & 255], n >> 8);
}

// The exponentials of one type of logits relative to a reference, as each block sets them up in LDS.
//   int8     e^x for each code; the reference is 0 (|x| <= 128)
//   int16    e^-d = hi[d >> 8] lo[d & 255] for the distance d of a code to the reference
//   others   exp_by_roots of the distance
// The reference of int16 and int32 is the largest code of the format where the whole range of distances is below 700, so that
// no exponential vanishes; otherwise, the largest of the row.
template <typename T>
struct Exponentials {
    static constexpr int kTable = sizeof(T) == 1 ? 256 : sizeof(T) == 2 ? 512 : 256;
    const double *table;
    int fl;
    double step;      // 2^-fl
    double ref;       // int32: the reference's value

    __device__ __forceinline__ static void build(double *table, int fl)
    {
        const double step = ldexp(1.0, -fl);
        for (int j = threadIdx.x; j < kTable; j += blockDim.x) {
            if constexpr (sizeof(T) == 1) table[j] = exp((double)(int8_t)j * step);
            else if constexpr (sizeof(T) == 2) table[j] = exp(-(double)(j < 256 ? j << 8 : j - 256) * step);
            else table[j] = exp2((double)j / 256.0);
        }
    }
    __device__ __forceinline__ double at(T l, T m) const
    {
        if constexpr (sizeof(T) == 1) return table[(uint8_t)l];
        else if constexpr (sizeof(T) == 2) {
            const uint32_t d = (uint32_t)((int)m - (int)l);
            return table[d >> 8] * table[256 + (d & 255)];
        } else if constexpr (__is_same(T, float)) return exp_by_roots((double)l - (double)m, table);
        else return exp_by_roots(fma((double)l, step, -ref), table);
    }
};

template <typename T> __device__ __forceinline__ T lowest() { return (T)(sizeof(T) == 1 ? -128 : sizeof(T) == 2 ? -32768 : INT32_MIN); }
template <> __device__ __forceinline__ float lowest<float>() { return -INFINITY; }
template <typename T> __device__ __forceinline__ T larger(T a, T b) { return a > b ? a : b; }
template <> __device__ __forceinline__ float larger<float>(float a, float b) { return fmaxf(a, b); }

// the value of the lane N places on in its row of 16
template <int N, typename V>
__device__ __forceinline__ V from_row(V v)
{
    constexpr int kWordsOf = (sizeof(V) + 3) / 4;
    uint32_t w[kWordsOf] = {};
    __builtin_memcpy(w, &v, sizeof(V));
#pragma unroll
    for (int k = 0; k < kWordsOf; ++k) w[k] = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w[k], 0x120 + N, 0xf, 0xf, false);
    __builtin_memcpy(&v, w, sizeof(V));
    return v;
}

// reduction over a wavefront, all of whose lanes take part: in lane 0
template <typename V, typename Op>
__device__ __forceinline__ V over_wave(V v, Op op)
{
    v = op(v, from_row<8>(v));
    v = op(v, from_row<4>(v));
    v = op(v, from_row<2>(v));
    v = op(v, from_row<1>(v));
    v = op(v, (V)__shfl_xor(v, 16, 64));
    return op(v, (V)__shfl_xor(v, 32, 64));
}

// reduction over the block, in every thread; `part` is used once
template <typename V, typename Op>
__device__ __forceinline__ V over_block(V v, V *part, Op op)
{
    v = over_wave(v, op);
    if ((threadIdx.x & (kWave - 1)) == 0) part[threadIdx.x / kWave] = v;
    __syncthreads();
    v = part[0];
    for (int w = 1; w < (int)(blockDim.x / kWave); ++w) v = op(v, part[w]);
    return v;
}

struct Pair { double a, b; };
__device__ __forceinline__ Pair sums_over_block(Pair v, Pair *part)
{
    const auto add = [](double x, double y) { return x + y; };
    v.a = over_wave(v.a, add);
    v.b = over_wave(v.b, add);
    if ((threadIdx.x & (kWave - 1)) == 0) part[threadIdx.x / kWave] = v;
    __syncthreads();
    v = part[0];
    for (int w = 1; w < (int)(blockDim.x / kWave); ++w) { v.a += part[w].a; v.b += part[w].b; }
    return v;
}

// a 64-bit value of one lane, in all
__device__ __forceinline__ uint64_t of_lane(uint64_t v, int lane)
{
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
}

struct RowPart { double m, s; };      // largest value (0: not needed) and sum of a chunk

enum { WHOLE_ROW, CHUNK_SUMS, CHUNK_CODES };
struct ChunkArgs {
    uint32_t splits, units;           // chunks of a row, units of a chunk
    RowPart *part;                    // [row][chunk]
    bool fixed;                       // the reference is the code `top`
    int top;
    bool past;                        // codes are stored past the caches
};

template <typename T>
__device__ __forceinline__ void load_unit(const T *p, uint32_t (&w)[kWords<T>]) { __builtin_memcpy(w, p, kUnit<T> * sizeof(T)); }

template <typename T, typename G, int MODE>
__global__ void __launch_bounds__(kMostThreads, 8) cross_entropy_kernel(const LogitArgs a, const ChunkArgs c)
{
    constexpr int U = kUnit<T>, W = kWords<T>;
    constexpr bool kByte = sizeof(T) == 1, kFloat = __is_same(T, float);
    using X = Exponentials<T>;
    __shared__ double table[X::kTable];
    __shared__ double part_s[kMostThreads / kWave];
    __shared__ T part_m[kMostThreads / kWave];
    __shared__ int64_t codes64[kByte && sizeof(G) == 4 ? 256 : 1];
    __shared__ int32_t codes32[kByte && sizeof(G) < 4 ? 256 : 1];
    const uint32_t in_launch = blockIdx.x / c.splits, chunk = blockIdx.x - in_launch * c.splits;
    const uint64_t i = a.row0 + in_launch;
    const T *row = static_cast<const T *>(a.logits) + i * a.ld;
    const uint64_t base = i * a.classes;
    const uint32_t head = (uint32_t)min((uint64_t)(-base & (U - 1)), a.classes);
    const uint64_t whole = (a.classes - head) / U, first = min((uint64_t)chunk * c.units, whole);
    const uint32_t units = (uint32_t)min(whole - first, (uint64_t)c.units), tail = (uint32_t)(a.classes - head - whole * U);
    const T *body = row + head + first * U;
    // the edges belong to the first chunk
    const bool on_edge = chunk == 0 && threadIdx.x < head + tail;
    const uint64_t edge_col = threadIdx.x < head ? threadIdx.x : a.classes - (head + tail) + threadIdx.x;
    const T edge = on_edge ? row[edge_col] : lowest<T>();
    G *grad = static_cast<G *>(a.grad) + i * a.ldg;
    const int64_t label = a.labels[i];
    const bool there = label >= 0 && (uint64_t)label < a.classes;
    const bool tells = threadIdx.x == 0 && chunk == 0 && a.logp;
    const auto no_gradient = [&] {
        G zero[U] = {};
        for (uint32_t u = threadIdx.x; u < units; u += blockDim.x) __builtin_memcpy(grad + head + (first + u) * U, zero, sizeof(zero));
        if (on_edge) grad[edge_col] = 0;
    };
    if (!there) {                                             // such a row is not read
        if (MODE == CHUNK_SUMS) return;
        no_gradient();
        if (tells) a.logp[i] = label < 0 ? 0.0f : NAN;
        return;
    }

    X::build(table, a.fl);
    X ex = {table, a.fl, ldexp(1.0, -a.fl), 0.0};
    T m = (T)c.top;
    if (!kByte && !kFloat && !c.fixed && MODE != CHUNK_CODES) {
        m = edge;
        for (uint32_t u = threadIdx.x; u < units; u += blockDim.x) {
            uint32_t w[W];
            load_unit(body + (uint64_t)u * U, w);
#pragma unroll
            for (int e = 0; e < U; ++e) m = larger(m, unit_get<T>(w, e));
        }
        m = over_block(m, part_m, [](T x, T y) { return larger(x, y); });
    } else {
        __syncthreads();
    }

    ex.ref = (double)m * ex.step;
    double ref, sum;
    const auto add = [](double x, double y) { return x + y; };
    if constexpr (MODE != CHUNK_CODES) {
        double s = 0.0;
        if constexpr (kFloat) {
            // every thread has a reference of its own, which follows the logits only where they get 600 ahead of it (the difference
            // is exact to half a step of its own; r + 600 may lie hundreds further on, where exponentials end)
            float r = -INFINITY;
            int bad = 0;
            const auto take = [&](float largest) -> bool {
                if (!(largest < INFINITY)) { bad = 1; return false; }
                if (largest - r > 600.0f) { s = r > -INFINITY ? s * exp((double)r - (double)largest) : 0.0; r = largest; }
                return largest > -INFINITY;
            };
            if (on_edge && take(edge)) s += ex.at(edge, r);
            for (uint32_t u = threadIdx.x; u < units; u += blockDim.x) {
                uint32_t w[W];
                load_unit(body + (uint64_t)u * U, w);
                float largest = unit_get<T>(w, 0);
#pragma unroll
                for (int e = 1; e < U; ++e) largest = __builtin_elementwise_maximum(largest, unit_get<T>(w, e));
                if (!take(largest)) continue;
#pragma unroll
                for (int e = 0; e < U; ++e) s += ex.at(unit_get<T>(w, e), r);
            }
            m = over_block(r, part_m, [](T x, T y) { return larger(x, y); });
            s = r > -INFINITY ? s * exp((double)r - (double)m) : 0.0;
            if (__syncthreads_or(bad)) s = NAN;
        } else {
            if (on_edge) s = ex.at(edge, m);
            for (uint32_t u = threadIdx.x; u < units; u += blockDim.x) {
                uint32_t w[W];
                load_unit(body + (uint64_t)u * U, w);
#pragma unroll
                for (int e = 0; e < U; ++e) s += ex.at(unit_get<T>(w, e), m);
            }
        }
        sum = over_block(s, part_s, add);
        ref = kByte ? 0.0 : value_of(m, a.fl);
        if constexpr (MODE == CHUNK_SUMS) {
            if (threadIdx.x == 0) c.part[blockIdx.x] = {ref, sum};
            return;
        }
    } else {
        __shared__ double part_r[kMostThreads / kWave];
        const RowPart *p = c.part + i * c.splits;
        double s = 0.0;
        ref = -INFINITY;
        for (uint32_t j = threadIdx.x; j < c.splits; j += blockDim.x) ref = fmax(ref, p[j].m);
        ref = over_block(ref, part_r, [](double x, double y) { return fmax(x, y); });
        for (uint32_t j = threadIdx.x; j < c.splits; j += blockDim.x) s += p[j].m > -INFINITY ? p[j].s * exp(p[j].m - ref) : p[j].s;
        sum = over_block(s, part_s, add);
        if constexpr (!kByte) m = kFloat ? (T)ref : (T)ldexp(ref, a.fl);
        ex.ref = ref;
    }

    const bool bad = sum != sum, none = ref == -INFINITY;
    if (tells) a.logp[i] = bad ? NAN : none ? -INFINITY : (float)fmin(value_of(row[label], a.fl) - ref - log_of_sum(sum), 0.0);
    const double weight = a.weights ? (double)a.weights[i] : 1.0;
    if (bad || none || !(fabs(weight) < INFINITY)) {
        no_gradient();
        return;
    }
    // floor of the clamped value in units of 2^-16 of a code, and the code for a draw
    const double tmin = -ldexp(1.0, a.wl_g + 15), tmax = ldexp(1.0, a.wl_g + 15) - 65536.0;
    const double scale = weight * ldexp(1.0, a.fl_g + 16) / sum;
    const auto grid_of = [&](double t) { return floor(fmin(fmax(t * scale, tmin), tmax)); };
    const auto code_of = [](double z, uint32_t r16) -> int {
        if constexpr (sizeof(G) == 4) return (int)(((long long)z + r16) >> 16);
        else return ((int)z + (int)r16) >> 16;
    };
    if constexpr (kByte) {
        for (int j = threadIdx.x; j < 256; j += blockDim.x) {
            if constexpr (sizeof(G) == 4) codes64[j] = (int64_t)grid_of(table[j]);
            else codes32[j] = (int32_t)grid_of(table[j]);
        }
        __syncthreads();
    }
    const auto code_at = [&](T l, uint32_t r16) -> G {
        if constexpr (kByte && sizeof(G) == 4) return (G)((codes64[(uint8_t)l] + (int)r16) >> 16);
        else if constexpr (kByte) return (G)((codes32[(uint8_t)l] + (int)r16) >> 16);
        else return (G)code_of(grid_of(ex.at(l, m)), r16);
    };
    const uint64_t group0 = (base + head) / 8 + first * (U / 8);
    for (uint32_t u = threadIdx.x; u < units; u += blockDim.x) {
        uint32_t w[W];
        load_unit(body + (uint64_t)u * U, w);
        uint32_t q[U];      // codes; of at most 16 bits: in the upper halves
#pragma unroll
        for (int h = 0; h < U / 8; ++h) {
            u32x4 blk = {0x80008000u, 0x80008000u, 0x80008000u, 0x80008000u};
            if (a.mode == ADAPT_SR) blk = rounding_block(a.seed, a.stream, group0 + (uint64_t)u * (U / 8) + h);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const T l = unit_get<T>(w, 8 * h + e);
                if constexpr (sizeof(G) == 4) q[8 * h + e] = (uint32_t)code_at(l, lane16(blk, e));
                else q[8 * h + e] = (uint32_t)(kByte ? codes32[(uint8_t)l] : (int)grid_of(ex.at(l, m))) + lane16(blk, e);
            }
        }
        G *to = grad + head + (first + u) * U;
        if constexpr (sizeof(G) == 4) __builtin_memcpy(to, q, sizeof(q));
        else if (c.past) store_upper<true>(to, q);
        else store_upper<false>(to, q);
    }
    if (on_edge) grad[edge_col] = code_at(edge, rounding_bits_of(a.seed, a.stream, base + edge_col, a.mode));
    // the label's own element, by the thread that has just stored it among others
    const int64_t at = label - (int64_t)head - (int64_t)(first * U);
    const bool mine = at >= 0 && at < (int64_t)units * U ? (uint32_t)(at / U) % blockDim.x == threadIdx.x : on_edge && edge_col == (uint64_t)label;
    if (mine) grad[label] = (G)code_of(grid_of(ex.at(row[label], m) - sum), rounding_bits_of(a.seed, a.stream, base + (uint64_t)label, a.mode));
}

// ---------------------------------------------------------------------------------------------
// Log probabilities.  One sweep over the row (or a chunk of it): sums of e^(x - r) and (x - r) e^(x - r) in fp32 over a unit and in
// fp64 from there on, and each thread's largest unit.  For 8-bit codes within +-16 r = 0 (8192 x 32000: 63 instead of 78 us); otherwise
// every thread has a reference of its own that follows the logits where they get 8 ahead of it.
// The k largest: the threads fall into 64 groups (their lanes), and the k-th largest of the groups' maxima is a bound below
// which none of them lies.  Few threads have anything above it; their units are spread over all threads, which put what they find
// into a list, whose members count how many are ahead of them.  Should the list overflow (the largest logits in few places,
// many of them), the row is swept once for each of the k.
// What bounds it: memory from 16 bits on (4096 x 32000 53 us, 4.9 TB/s; 1000 x 50001 fp32 with 5 alternatives 39 us, 5.1), the exponentials'
// and additions' issue at 8 bits (8192 x 32000 63 us, 4.2), with 8 alternatives 83.
// ---------------------------------------------------------------------------------------------
struct LogPart { double r, s, e; };      // reference (fp64 values; NaN: not a distribution), sums of a chunk

struct LogChunkArgs {
    uint32_t splits, units;
    LogPart *part;                       // [row][chunk]
    uint64_t *keys;                      // [row][chunk][topk]
    int listed;                          // entries of the list
};

template <typename T> struct RowValue { typedef float type; };      // 8- and 16-bit codes are exact in fp32
template <> struct RowValue<int32_t> { typedef int type; };

// scratch of the selection, in LDS
struct TopScratch {
    uint64_t bound;
    uint32_t count, reaching;
    uint32_t ahead[kWave];      // groups ahead of this one, and (16 bits up) those not behind it
    uint64_t group[kWave];
    uint64_t best[kMaxTop];
    uint64_t part[kMostThreads / kWave];
    uint16_t reach[kMostThreads];
};

// The bound for the k largest from one key per thread (0: none); the scratch's counts are 0 afterwards
__device__ __forceinline__ uint64_t bound_of(uint64_t key, int k, TopScratch &s, uint64_t *list)
{
    const int lane = threadIdx.x & (kWave - 1), wave = threadIdx.x / kWave, waves = blockDim.x / kWave;
    list[threadIdx.x] = key;
    if (threadIdx.x < kWave) s.ahead[lane] = 0;
    if (threadIdx.x == 0) { s.bound = 0; s.count = s.reaching = 0; }
    __syncthreads();
    if (wave == 0) {
        for (int w = 1; w < waves; ++w) { const uint64_t o = list[w * kWave + lane]; key = o > key ? o : key; }
        s.group[lane] = key;
    }
    __syncthreads();
    key = s.group[lane];
    uint32_t ahead = 0;
    for (int j = wave; j < kWave; j += waves) {
        const uint64_t other = of_lane(key, __builtin_amdgcn_readfirstlane(j));
        ahead += other > key ? 0x10001u : other == key ? 0x10000u : 0u;
    }
    atomicAdd(&s.ahead[lane], ahead);
    __syncthreads();
    ahead = s.ahead[lane];
    if (wave == 0 && (int)(ahead & 0xffff) < k && (int)(ahead >> 16) >= k) s.bound = key;      // the same from every such lane
    __syncthreads();
    return s.bound;
}

__device__ __forceinline__ void put(uint64_t key, TopScratch &s, uint64_t *list, int listed)
{
    const uint32_t at = atomicAdd(&s.count, 1u);
    if (at < (uint32_t)listed) list[at] = key;
}

// The k largest of the list's `count` entries, in order, to s.best
__device__ __forceinline__ void best_of_list(const uint32_t found, int k, TopScratch &s, const uint64_t *list)
{
    const uint32_t count = __builtin_amdgcn_readfirstlane(found);      // the same in every thread
    if (count <= (uint32_t)kWave) {
        if (threadIdx.x < kWave) {
            const uint64_t key = threadIdx.x < count ? list[threadIdx.x] : 0;
            int ahead = 0;
            for (uint32_t j = 0; j < count; ++j) ahead += of_lane(key, (int)j) > key;
            if (threadIdx.x < count && ahead < k) s.best[ahead] = key;
        }
    } else {
        for (uint32_t i = threadIdx.x; i < count; i += blockDim.x) {
            const uint64_t key = list[i];
            uint32_t ahead = 0;
#pragma unroll 8
            for (uint32_t j = 0; j < count; ++j) ahead += list[j] > key;
            if (ahead < (uint32_t)k) s.best[ahead] = key;
        }
    }
    __syncthreads();
}

// The same from what `every(look)` shows of the thread's keys, one sweep for each
template <typename Every>
__device__ __forceinline__ void one_by_one(int k, TopScratch &s, const Every &every)
{
    uint64_t last = ~0ull;
    for (int n = 0; n < k; ++n) {
        uint64_t best = 0;
        every([&](uint64_t key) { if (key < last && key > best) best = key; });
        last = over_block(best, s.part, [](uint64_t x, uint64_t y) { return x > y ? x : y; });
        if (threadIdx.x == 0) s.best[n] = last;
        __syncthreads();
    }
}

// a row's label and its logit, each loaded before it is needed
template <typename T>
struct LabelOf {
    int64_t label;
    T logit = 0;
    __device__ __forceinline__ LabelOf(const LogitArgs &a, uint64_t i) : label(a.logp ? a.labels[i] : -1) {}
    __device__ __forceinline__ void look_up(const LogitArgs &a, const T *row)
    {
        if (label >= 0 && (uint64_t)label < a.classes) logit = row[label];
    }
};

template <typename T>
__device__ __forceinline__ double value_of_order(uint32_t order, int fl)
{
    if constexpr (__is_same(T, float)) return (double)__uint_as_float((order & 0x80000000u) ? order & 0x7fffffffu : ~order);
    else if constexpr (sizeof(T) == 4) return value_of((int32_t)(order ^ 0x80000000u), fl);
    else return ldexp((double)__uint_as_float((order & 0x80000000u) ? order & 0x7fffffffu : ~order), -fl);
}

// what becomes of a row once its sums are known, for threads 0.. of a row; `best`: the thread's share of its largest logits
template <typename T>
__device__ __forceinline__ void finish_row(const LogitArgs &a, uint64_t i, const LabelOf<T> &l, const LogPart &p, int thread, uint64_t best)
{
    const bool bad = p.r != p.r, none = p.r == -INFINITY;
    const double log_s = log_of_fp32_sum(p.s);
    // at most 0, as the entropy is at least 0: exponents of up to 23 are rounded to fp32 (8-bit codes with the reference 0), so that a sum
    // can be smaller than its largest term by 8e-7 of itself
    const auto log_prob = [&](double x) { return bad ? NAN : none ? -INFINITY : (float)fmin(x - p.r - log_s, 0.0); };
    if (thread == 0) {
        if (a.lse) a.lse[i] = bad ? NAN : none ? -INFINITY : (float)(p.r + log_s);
        if (a.entropy) a.entropy[i] = bad ? NAN : none ? 0.0f : (float)fmax(log_s - p.e / p.s, 0.0);
        if (a.logp) a.logp[i] = l.label < 0 ? 0.0f : (uint64_t)l.label >= a.classes ? NAN : log_prob(value_of(l.logit, a.fl));
    }
    if (thread < a.topk) {
        a.top_index[i * a.topk + thread] = (int32_t)(0x7fffffffu - (uint32_t)best);
        a.top_logp[i * a.topk + thread] = log_prob(value_of_order<T>((uint32_t)(best >> 32), a.fl));
    }
}

// moves the sums of a thread or chunk to another reference
__device__ __forceinline__ void rebase(LogPart &p, double r)
{
    if (p.r == -INFINITY) { p.s = p.e = 0.0; }
    else {
        const double k = exp(p.r - r);
        p.e = k * (p.e + (p.r - r) * p.s);
        p.s *= k;
    }
    p.r = r;
}

template <typename T, bool TOP, bool FIXED>
__global__ void __launch_bounds__(kMostThreads, 8) log_probs_kernel(const LogitArgs a, const LogChunkArgs c)
{
    constexpr int U = kUnit<T>, W = kWords<T>;
    constexpr bool kFloat = __is_same(T, float);
    typedef typename RowValue<T>::type V;
    extern __shared__ uint64_t list[];
    __shared__ TopScratch top;
    __shared__ double part_r[kMostThreads / kWave];
    __shared__ Pair part_s[kMostThreads / kWave];
    const uint32_t in_launch = blockIdx.x / c.splits, chunk = blockIdx.x - in_launch * c.splits;
    const uint64_t i = a.row0 + in_launch;
    const T *row = static_cast<const T *>(a.logits) + i * a.ld;
    // units start at 16-byte addresses
    const uint32_t head = (uint32_t)min((uint64_t)((-(uintptr_t)row & 15) / sizeof(T)), a.classes);
    const uint64_t whole = (a.classes - head) / U, first = min((uint64_t)chunk * c.units, whole);
    const uint32_t units = (uint32_t)min(whole - first, (uint64_t)c.units), tail = (uint32_t)(a.classes - head - whole * U);
    const T *body = row + head + first * U;
    const bool on_edge = chunk == 0 && threadIdx.x < head + tail;
    const uint32_t edge_col = threadIdx.x < head ? threadIdx.x : (uint32_t)a.classes - (head + tail) + threadIdx.x;

    LabelOf<T> wanted(a, i);
    const float to_log2 = 1.44269504f * ldexpf(1.0f, -a.fl);
    V r = 0;
    bool begun = FIXED;
    double s = 0.0, e = 0.0;
    int bad = 0;
    // a reference for values up to `largest`; false: nothing to add
    const auto refer = [&](V largest) -> bool {
        if (kFloat && !((float)largest < INFINITY)) { bad = 1; return false; }
        if (FIXED) return true;
        const float ahead = begun ? (float)((double)largest - (double)r) * to_log2 : INFINITY;
        if (ahead > 11.5f && (!kFloat || (float)largest > -INFINITY)) {
            const double d = ((double)r - (double)largest) * (double)to_log2, k = begun ? exp2(d) : 0.0;
            e = begun ? k * (e + d * s) : 0.0;
            s *= k;
            r = largest;
            begun = true;
        }
        return begun;
    };
    const auto log2_of = [&](V x) -> float {
        if constexpr (FIXED) return (float)x * to_log2;
        else if constexpr (__is_same(T, int32_t)) return (float)((double)x - (double)r) * to_log2;
        else if constexpr (kFloat) return fmaxf((x - r) * to_log2, -200.0f);
        else return (x - r) * to_log2;
    };
    // the thread's largest unit, of equal ones the first: number 0 are the head's elements, the tail's come last
    V largest = 0;
    uint32_t where = ~0u;
    const uint32_t edge_unit = threadIdx.x < head ? 0 : 0x7ffffff0u;
    const auto clean = [](V v) -> V {
        if constexpr (kFloat) return v != v ? -INFINITY : v;
        else return v;
    };
    V edge = 0;
    if (on_edge) {
        edge = (V)row[edge_col];
        if (refer(edge)) { const float g = log2_of(edge), t = __builtin_amdgcn_exp2f(g); s += t; e += (double)(t * g); }
        if (kFloat) edge = clean(edge);
    }
    for (uint32_t u = threadIdx.x; u < units; u += blockDim.x) {
        uint32_t w[W];
        load_unit(body + (uint64_t)u * U, w);
        V v[U], m;
#pragma unroll
        for (int j = 0; j < U; ++j) v[j] = (V)unit_get<T>(w, j);
        if (TOP || !FIXED) {
            m = v[0];
#pragma unroll
            for (int j = 1; j < U; ++j) {
                if constexpr (kFloat) m = __builtin_elementwise_maximum(m, v[j]);
                else if constexpr (sizeof(T) < 4) m = __builtin_elementwise_maximum(m, v[j]);
                else m = max(m, v[j]);
            }
        }
        if (FIXED || refer(m)) {
            float us = 0.0f, ue = 0.0f;
#pragma unroll
            for (int j = 0; j < U; ++j) {
                const float g = log2_of(v[j]), t = __builtin_amdgcn_exp2f(g);
                us += t;
                ue = fmaf(t, g, ue);
            }
            s += us;
            e += ue;
        }
        if constexpr (TOP) {
            if (kFloat && m != m) {
                m = clean(v[0]);
#pragma unroll
                for (int j = 1; j < U; ++j) m = larger(m, clean(v[j]));
            }
            if (where == ~0u || m > largest) { largest = m; where = (uint32_t)first + u + 1; }
        }
    }
    if (TOP && on_edge && (where == ~0u || (edge_unit == 0 ? edge >= largest : edge > largest))) { largest = edge; where = edge_unit; }
    if (c.splits == 1) wanted.look_up(a, row);
    // one reference for the block
    const auto maximum = [](double x, double y) { return fmax(x, y); };
    const double ln2 = 0.69314718055994530942;
    LogPart p = {begun ? (double)r * ldexp(1.0, -a.fl) : -INFINITY, s, e * ln2};
    if (!FIXED) {
        const double ref = over_block(p.r, part_r, maximum);
        rebase(p, ref);
    }
    const Pair sums = sums_over_block({p.s, p.e}, part_s);
    p.s = sums.a;
    p.e = sums.b;
    if (kFloat && __syncthreads_or(bad)) p.r = NAN;

    if constexpr (TOP) {
        const uint64_t mine = where == ~0u ? 0 : key_of(order_of(largest), where);
        const uint64_t bound = bound_of(mine, a.topk, top, list);
        // the threads that reach it, then their units, spread over all threads
        if (mine >= bound && mine) top.reach[atomicAdd(&top.reaching, 1u)] = (uint16_t)threadIdx.x;
        if (on_edge && key_of(order_of(edge), edge_unit) >= bound) put(key_of(order_of(edge), edge_col), top, list, c.listed);
        __syncthreads();
        const uint32_t each = (units + blockDim.x - 1) / blockDim.x, pairs = top.reaching * each;
        for (uint32_t n = threadIdx.x; n < pairs; n += blockDim.x) {
            const uint32_t thread = n / each, u = top.reach[thread] + (n - thread * each) * blockDim.x;
            if (u >= units) continue;
            uint32_t w[W];
            load_unit(body + (uint64_t)u * U, w);
#pragma unroll
            for (int j = 0; j < U; ++j) {
                const uint32_t order = order_of((V)unit_get<T>(w, j));
                if (key_of(order, (uint32_t)first + u + 1) >= bound) put(key_of(order, head + ((uint32_t)first + u) * U + j), top, list, c.listed);
            }
        }
        __syncthreads();
        const uint32_t found = top.count;
        if (found <= (uint32_t)c.listed) {
            if ((int)threadIdx.x < a.topk) top.best[threadIdx.x] = 0;      // a chunk may have fewer
            __syncthreads();
            best_of_list(found, a.topk, top, list);
        } else {
            one_by_one(a.topk, top, [&](auto &&look) {
                if (on_edge) look(key_of(order_of((V)row[edge_col]), edge_col));
                for (uint32_t u = threadIdx.x; u < units; u += blockDim.x)
                    for (int j = 0; j < U; ++j) look(key_of(order_of((V)body[(uint64_t)u * U + j]), head + ((uint32_t)first + u) * U + j));
            });
        }
    }
    if (c.splits == 1) {
        finish_row(a, i, wanted, p, threadIdx.x, (int)threadIdx.x < a.topk ? top.best[threadIdx.x] : 0);
        return;
    }
    if (threadIdx.x == 0) c.part[blockIdx.x] = p;
    if (TOP && (int)threadIdx.x < a.topk) c.keys[(uint64_t)blockIdx.x * a.topk + threadIdx.x] = top.best[threadIdx.x];
}

// Rows of up to kSmall classes: a wavefront each, whose lanes hold their logits.  us in a captured graph, this / a block per row:
// 256 x 100 log probabilities of 8 bits 3.1 / 3.2, with 5 alternatives 4.8 / 9.3, cross entropy 3.8 / 5.0; 8192 x 100 5.4 / 6.4, 10.0 / 27,
// 7.7 / 12.3.  At 256 classes (8192 rows) they meet without alternatives, 6.1 / 6.3 and 11.1 / 11.3; with 5 of them (10.9 / 26) a wavefront
// would be faster for longer rows, too.
constexpr int kSmall = 256, kSmallThreads = 256;

template <typename T>
struct SmallRow {
    static constexpr int N = kSmall / kWave;
    T l[N];
    double m;          // largest; -inf: no class possible; NaN: not a distribution
    __device__ __forceinline__ SmallRow(const T *row, int classes, int fl)
    {
        const int lane = threadIdx.x & (kWave - 1);
        int bad = 0;
        m = -INFINITY;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            l[k] = lane + k * kWave < classes ? row[lane + k * kWave] : lowest<T>();
            if (lane + k * kWave < classes) {
                if (__is_same(T, float)) bad |= !(l[k] < (T)INFINITY);
                m = fmax(m, value_of(l[k], fl));
            }
        }
        m = over_wave(m, [](double x, double y) { return fmax(x, y); });
        if (__is_same(T, float) && __ballot(bad)) m = NAN;
    }
};
__device__ __forceinline__ double wave_sum(double v)
{
    v = over_wave(v, [](double x, double y) { return x + y; });
    return __longlong_as_double((long long)of_lane((uint64_t)__double_as_longlong(v), 0));      // the lanes add in different orders
}

template <typename T>
__global__ void __launch_bounds__(kSmallThreads) log_probs_small_kernel(const LogitArgs a)
{
    typedef typename RowValue<T>::type V;
    constexpr int N = SmallRow<T>::N;
    const uint64_t i = a.row0 + (uint64_t)blockIdx.x * (kSmallThreads / kWave) + threadIdx.x / kWave;
    if (i >= a.rows) return;
    const int lane = threadIdx.x & (kWave - 1), classes = (int)a.classes;
    const T *row = static_cast<const T *>(a.logits) + i * a.ld;
    LabelOf<T> wanted(a, i);
    const SmallRow<T> x(row, classes, a.fl);
    wanted.look_up(a, row);
    LogPart p = {x.m, 0.0, 0.0};
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const double d = value_of(x.l[k], a.fl) - x.m;
        if (k * kWave < classes && lane + k * kWave < classes && d > -700.0) {
            const float t = expf((float)d);
            p.s += t;
            p.e += t * d;
        }
    }
    p.s = wave_sum(p.s);
    p.e = wave_sum(p.e);
    uint64_t best = 0, last = ~0ull;
    for (int n = 0; n < a.topk; ++n) {
        uint64_t key = 0;
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const uint64_t o = lane + k * kWave < classes ? key_of(order_of((V)x.l[k]), lane + k * kWave) : 0;
            if (o < last && o > key) key = o;
        }
        last = over_wave(key, [](uint64_t u, uint64_t v) { return u > v ? u : v; });
        if (lane == n) best = last;
    }
    finish_row(a, i, wanted, p, lane, best);
}

template <typename T, typename G>
__global__ void __launch_bounds__(kSmallThreads) cross_entropy_small_kernel(const LogitArgs a)
{
    constexpr int N = SmallRow<T>::N;
    const uint64_t i = a.row0 + (uint64_t)blockIdx.x * (kSmallThreads / kWave) + threadIdx.x / kWave;
    if (i >= a.rows) return;
    const int lane = threadIdx.x & (kWave - 1), classes = (int)a.classes;
    const T *row = static_cast<const T *>(a.logits) + i * a.ld;
    const int64_t label = a.labels[i];
    const bool there = label >= 0 && (uint64_t)label < a.classes;
    const double at_label = there ? value_of(row[label], a.fl) : 0.0, weight = a.weights ? (double)a.weights[i] : 1.0;
    const SmallRow<T> x(row, classes, a.fl);
    double e[N], s = 0.0;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        e[k] = 0.0;
        if (k * kWave < classes && lane + k * kWave < classes) e[k] = exp(value_of(x.l[k], a.fl) - x.m);
        s += e[k];
    }
    s = wave_sum(s);
    const bool counts = there && x.m > -INFINITY && fabs(weight) < INFINITY;
    if (lane == 0 && a.logp)
        a.logp[i] = label < 0 ? 0.0f : !there || x.m != x.m ? NAN : x.m == -INFINITY ? -INFINITY : (float)fmin(at_label - x.m - log_of_sum(s), 0.0);
    const double tmin = -ldexp(1.0, a.wl_g + 15), tmax = ldexp(1.0, a.wl_g + 15) - 65536.0, scale = weight * ldexp(1.0, a.fl_g + 16) / s;
    G *grad = static_cast<G *>(a.grad) + i * a.ldg;
#pragma unroll
    for (int k = 0; k < N; ++k) {
        const int j = lane + k * kWave;
        if (j >= classes) break;
        const double t = floor(fmin(fmax((j == label ? e[k] - s : e[k]) * scale, tmin), tmax));
        const long long q = ((long long)t + rounding_bits_of(a.seed, a.stream, i * a.classes + j, a.mode)) >> 16;
        grad[j] = counts ? (G)q : (G)0;
    }
}

constexpr int kJoinThreads = 256;
template <typename T>
__global__ void __launch_bounds__(kJoinThreads) join_log_probs_kernel(const LogitArgs a, const LogChunkArgs c)
{
    extern __shared__ uint64_t list[];
    __shared__ TopScratch top;
    __shared__ double part_r[kMostThreads / kWave];
    __shared__ Pair part_s[kMostThreads / kWave];
    const uint64_t i = blockIdx.x;
    LabelOf<T> wanted(a, i);
    const LogPart *parts = c.part + i * c.splits;
    // a chunk's keys are in order: it is taken in `slices` of every so many, so that there are 64 largest ones to compare
    const uint64_t *keys = c.keys + i * c.splits * a.topk;
    const uint32_t slices = min((uint32_t)a.topk, (kWave + c.splits - 1) / c.splits), heads = c.splits * slices;
    const auto head_of = [&](uint32_t j) { return keys + (uint64_t)(j / slices) * a.topk + j % slices; };
    // everything that has to come from memory first
    const LogPart none = {-INFINITY, 0.0, 0.0}, own = threadIdx.x < c.splits ? parts[threadIdx.x] : none;
    uint64_t mine = 0;
    for (uint32_t j = threadIdx.x; j < heads; j += kJoinThreads) mine = max(mine, *head_of(j));
    wanted.look_up(a, static_cast<const T *>(a.logits) + i * a.ld);
    double ref = own.r;
    int bad = own.r != own.r;
    for (uint32_t j = threadIdx.x + kJoinThreads; j < c.splits; j += kJoinThreads) {
        ref = fmax(ref, parts[j].r);
        bad |= parts[j].r != parts[j].r;
    }
    ref = over_block(ref, part_r, [](double x, double y) { return fmax(x, y); });
    LogPart p = own;
    rebase(p, ref);
    for (uint32_t j = threadIdx.x + kJoinThreads; j < c.splits; j += kJoinThreads) {
        LogPart q = parts[j];
        rebase(q, ref);
        p.s += q.s;
        p.e += q.e;
    }
    const Pair sums = sums_over_block({p.s, p.e}, part_s);
    p.s = sums.a;
    p.e = sums.b;
    if (__syncthreads_or(bad)) p.r = NAN;
    if (a.topk > 0) {
        const uint64_t bound = bound_of(mine, a.topk, top, list);
        if (mine >= bound)
            for (uint32_t j = threadIdx.x; j < heads; j += kJoinThreads) {
                const uint64_t *key = head_of(j);
                for (uint32_t n = j % slices; n < (uint32_t)a.topk && *key >= bound && *key != 0; n += slices, key += slices) put(*key, top, list, c.listed);
            }
        __syncthreads();
        if (top.count <= (uint32_t)c.listed) {
            best_of_list(top.count, a.topk, top, list);
        } else {
            one_by_one(a.topk, top, [&](auto &&look) { for (uint32_t j = threadIdx.x; j < c.splits * a.topk; j += kJoinThreads) look(keys[j]); });
        }
    }
    finish_row(a, i, wanted, p, threadIdx.x, (int)threadIdx.x < a.topk ? top.best[threadIdx.x] : 0);
}

struct LogProbsPlan {
    uint32_t splits, units, threads;
    size_t part_bytes, ws_bytes;
};

// Threads: a thread takes two units where blocks are few (eight where they fill the card), rows of 4096 units 1024 threads where each has a
// compute unit of its own.  Chunks: a second launch and its join pay only for few, long rows.  us in a captured graph, chunks / a
// block per row, 8 bits without alternatives, 16 bits with 8, fp32 with 32: 1 x 100000 (6250 or 12500 units) 6.0 / 7.9, 12.4 / 14.7,
// 16.7 / 17.6; 1 x 200000 6.1 / 12.6, 12.6 / 21.7, 16.4 / 24.6; 64 x 100000 8.2 / 8.4, 18.0 / 15.3, 22.3 / 18.2; 64 x 200000 10.0 / 13.1,
// 20.2 / 22.3, 26.4 / 28.5; 200 x 200000 17.3 / 15.5, 29.3 / 21.6, 49.5 / 33.9.  The threshold is one for all: 32 to 64 rows with alternatives
// lose up to 22 % by it as far as some 150,000 classes of 16 bits or fp32.
static LogProbsPlan plan_log_probs(int num_cu, uint64_t rows, uint64_t classes, int topk, adapt_fmt f)
{
    const int U = f.wl != ADAPT_WL_FP32 && f.wl <= 8 ? 16 : 8;
    LogProbsPlan p = {};
    const uint64_t all = std::max<uint64_t>(classes / U, 1), wanted = 4 * (uint64_t)num_cu /* blocks */;
    uint64_t splits = 1;
    if (rows > 0 && rows * 4 <= (uint64_t)num_cu && all >= 12288) splits = std::min<uint64_t>((wanted + rows - 1) / rows, all / 256);
    p.units = (uint32_t)((all + splits - 1) / splits);
    p.splits = (uint32_t)((all + p.units - 1) / p.units);
    const uint64_t per = rows * splits >= wanted && splits == 1 ? 8 : 2, threads = (p.units + per - 1) / per;
    const uint64_t most = splits == 1 && rows <= (uint64_t)num_cu && all >= 4096 ? 1024 : 512;
    p.threads = (uint32_t)std::min<uint64_t>((threads + kWave - 1) / kWave * kWave, most);
    if (p.splits > 1) {
        p.part_bytes = (rows * p.splits * sizeof(LogPart) + 255) & ~(size_t)255;
        p.ws_bytes = p.part_bytes + rows * p.splits * topk * sizeof(uint64_t);
    }
    return p;
}

size_t ws_need_log_probs(int num_cu, uint64_t rows, uint64_t classes, int topk, adapt_fmt f)
{
    return plan_log_probs(num_cu, rows, classes, topk, f).ws_bytes + 16;
}

// How the rows of a cross entropy are cut.  Chunks of a row, whose sums are a launch of their own, for few and long rows: us in a captured
// graph, chunks / a block per row, 8 bits, 16 bits, fp32: one row of 2500 units 8.3 / 7.8, 8.9 / 8.4, 10.1 / 12.2, of 3200 8.5 / 8.9, 8.7 / 9.7,
// 9.9 / 14.3, of 5000 8.2 / 11.7, 8.6 / 12.8, 9.8 / 19.1; 64 rows of 2500 units 9.9 / 8.6, 10.6 / 9.2, 12.3 / 12.9, of 3200 10.2 / 9.9, 10.8 / 10.4,
// 12.5 / 15.2, of 5000 10.5 / 12.9, 11.4 / 13.9, 12.6 / 20.0; 128 rows of 3200 units 11.4 / 10.2, 12.5 / 11.1, 14.3 / 15.3, of 5000 13.3 / 13.4,
// 14.6 / 14.8, 17.4 / 20.3; 200 x 100000 classes 19.9 / 16.9, 32.3 / 30.9, 47.1 / 46.9.  The threshold is where 8 and 16 bits meet at up to 64 rows;
// 65 to 128 rows of them lose up to 16 % between it and 5000 units, and one row of fp32 would gain from 1800 on.
// Threads: one unit each where every row has a compute unit of its own (1 x 5000, 1, 2, 4 units: 4.4, 5.0, 5.5), two where blocks are few
// (400 x 5000 of 16 bits, 1, 2, 4: 8.2, 7.5, 8.4), otherwise eight and at most 512 threads: 256, 512, 1024 threads take 8192 x 32000 of
// 8 bits 140, 151, 190; 1536 x 65531 of 16 bits 186, 157, 163; 1024 x 50001 fp32 129, 125, 126.
struct CrossEntropyPlan {
    uint32_t splits, units, threads;
    size_t ws_bytes;
};

static CrossEntropyPlan plan_cross_entropy(int num_cu, uint64_t rows, uint64_t classes, adapt_fmt f)
{
    const int U = f.wl != ADAPT_WL_FP32 && f.wl <= 8 ? 16 : 8;
    CrossEntropyPlan p = {};
    const uint64_t all = std::max<uint64_t>(classes / U, 1), wanted = 4 * (uint64_t)num_cu /* blocks */;
    uint64_t splits = 1;
    if (rows > 0 && rows * 2 <= (uint64_t)num_cu && all >= 3200) splits = std::min<uint64_t>((wanted + rows - 1) / rows, all / 256);
    p.splits = (uint32_t)splits;
    p.units = (uint32_t)((all + splits - 1) / splits);
    const bool alone = rows <= (uint64_t)num_cu;
    const uint64_t per = splits > 1 ? 4 : alone ? 1 : rows < wanted ? 2 : 8, threads = (p.units + per - 1) / per;
    p.threads = (uint32_t)std::min<uint64_t>((threads + kWave - 1) / kWave * kWave, splits == 1 && alone ? 1024 : 512);
    p.ws_bytes = p.splits > 1 ? rows * p.splits * sizeof(RowPart) : 0;
    return p;
}

size_t ws_need_cross_entropy(int num_cu, uint64_t rows, uint64_t classes, adapt_fmt f, adapt_fmt)
{
    return plan_cross_entropy(num_cu, rows, classes, f).ws_bytes + 16;
}

bool logits_ok(uint64_t rows, uint64_t classes, uint64_t ld)
{
    return classes >= 1 && classes <= (1ull << 30) && ld >= classes && rows < (1ull << 31) && ld <= (1ull << 40) &&
           (rows == 0 || ld <= (1ull << 40) / rows);
}

}  // namespace adapt

using namespace adapt;

static int logit_bytes(adapt_fmt f) { return f.wl == ADAPT_WL_FP32 ? 4 : storage_bytes(f); }

// A launch takes fewer than 2^32 threads: rows in slabs of 2^21 blocks (rows in chunks are fewer)
template <typename Launch>
static void for_slabs(LogitArgs a, uint64_t rows_per_block, const Launch &launch)
{
    const uint64_t most = rows_per_block << 21;
    for (a.row0 = 0; a.row0 < a.rows; a.row0 += most) {
        const uint64_t rows = std::min(a.rows - a.row0, most);
        launch(a, (unsigned)((rows + rows_per_block - 1) / rows_per_block));
    }
}

template <typename T>
static void launch_log_probs(adapt_ctx *ctx, const LogitArgs &a, const LogProbsPlan &p)
{
    const bool fixed = sizeof(T) == 1 && a.fl >= 3;
    LogChunkArgs c = {p.splits, p.units, reinterpret_cast<LogPart *>(scratch(ctx)), reinterpret_cast<uint64_t *>(scratch(ctx) + p.part_bytes),
                      (int)(4 * p.threads)};
    const dim3 block(p.threads);
    const size_t lds = a.topk > 0 ? c.listed * sizeof(uint64_t) : 0;
    for_slabs(a, 1, [&](const LogitArgs &s, unsigned rows) {
        const dim3 grid(rows * p.splits);
        if constexpr (sizeof(T) == 1) {
            if (fixed && a.topk > 0) hipLaunchKernelGGL((log_probs_kernel<T, true, true>), grid, block, lds, ctx->stream, s, c);
            else if (fixed) hipLaunchKernelGGL((log_probs_kernel<T, false, true>), grid, block, lds, ctx->stream, s, c);
        }
        if (!fixed && a.topk > 0) hipLaunchKernelGGL((log_probs_kernel<T, true, false>), grid, block, lds, ctx->stream, s, c);
        else if (!fixed) hipLaunchKernelGGL((log_probs_kernel<T, false, false>), grid, block, lds, ctx->stream, s, c);
    });
    if (p.splits > 1) {
        c.listed = 1024;
        hipLaunchKernelGGL(join_log_probs_kernel<T>, dim3((unsigned)a.rows), dim3(kJoinThreads), a.topk ? c.listed * sizeof(uint64_t) : 0, ctx->stream, a, c);
    }
}

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
    if (classes <= (size_t)kSmall) {
        const dim3 block(kSmallThreads);
        for_slabs(a, kSmallThreads / kWave, [&](const LogitArgs &s, unsigned blocks) {
            const dim3 grid(blocks);
            if (f.wl == ADAPT_WL_FP32) hipLaunchKernelGGL(log_probs_small_kernel<float>, grid, block, 0, ctx->stream, s);
            else if (f.wl <= 8) hipLaunchKernelGGL(log_probs_small_kernel<int8_t>, grid, block, 0, ctx->stream, s);
            else if (f.wl <= 16) hipLaunchKernelGGL(log_probs_small_kernel<int16_t>, grid, block, 0, ctx->stream, s);
            else hipLaunchKernelGGL(log_probs_small_kernel<int32_t>, grid, block, 0, ctx->stream, s);
        });
        return hip_status(ctx, hipGetLastError());
    }
    const LogProbsPlan p = plan_log_probs(ctx->num_cu, rows, classes, topk, f);
    if (p.ws_bytes > scratch_bytes(ctx)) return ADAPT_EWORKSPACE;
    if (f.wl == ADAPT_WL_FP32) launch_log_probs<float>(ctx, a, p);
    else if (f.wl <= 8) launch_log_probs<int8_t>(ctx, a, p);
    else if (f.wl <= 16) launch_log_probs<int16_t>(ctx, a, p);
    else launch_log_probs<int32_t>(ctx, a, p);
    return hip_status(ctx, hipGetLastError());
}

// The reference of integer logits where it is the largest code: of the storage for int16 (distances to it index tables), of the format for
// int32.  (8-bit codes take 0, fp32 logits what the rows hold.)
struct FixedReference { bool fixed; int top; };
template <typename T>
static FixedReference fixed_reference(int wl, int fl)
{
    if (sizeof(T) == 1 || __is_same(T, float)) return {false, 0};
    const int span = sizeof(T) == 2 ? 16 : wl;
    return {span - fl <= 9, (int)((1ll << (span - 1)) - 1)};
}

template <typename T, typename G>
static void launch_cross_entropy(adapt_ctx *ctx, const LogitArgs &a, const CrossEntropyPlan &p, int wl)
{
    // Codes of 8 and 16 bits that take 96 MiB or more leave the caches before the next call reads them, and take the room that the sweeps
    // need (wider ones always go through them: not measured past them).  us, in the
    // caches / past them, alone and with a copy of the codes behind: 62 MiB (2048 x 32000, 8 bits) 33.5 / 33.4, 51 / 57; 125 MiB (4096)
    // 74 / 60, 127 / 123; 128 MiB (1024 x 65531, 16 bits) 83 / 66, 133 / 126; 250 MiB (8192 x 32000, 8 bits) 134 / 127, 231 / 229
    const bool past = a.rows * a.classes * sizeof(G) >= ((uint64_t)96 << 20);
    if (a.classes <= (uint64_t)kSmall) {
        for_slabs(a, kSmallThreads / kWave, [&](const LogitArgs &s, unsigned blocks) {
            hipLaunchKernelGGL((cross_entropy_small_kernel<T, G>), dim3(blocks), dim3(kSmallThreads), 0, ctx->stream, s);
        });
        return;
    }
    const FixedReference ref = fixed_reference<T>(wl, a.fl);
    const ChunkArgs c = {p.splits, p.units, reinterpret_cast<RowPart *>(scratch(ctx)), ref.fixed, ref.top, past};
    const dim3 block(p.threads);
    for_slabs(a, 1, [&](const LogitArgs &s, unsigned rows) {
        const dim3 grid(rows * p.splits);
        if (p.splits == 1) {
            hipLaunchKernelGGL((cross_entropy_kernel<T, G, WHOLE_ROW>), grid, block, 0, ctx->stream, s, c);
        } else {
            hipLaunchKernelGGL((cross_entropy_kernel<T, G, CHUNK_SUMS>), grid, block, 0, ctx->stream, s, c);
            hipLaunchKernelGGL((cross_entropy_kernel<T, G, CHUNK_CODES>), grid, block, 0, ctx->stream, s, c);
        }
    });
}
template <typename T>
static void launch_cross_entropy_to(adapt_ctx *ctx, const LogitArgs &a, const CrossEntropyPlan &p, int wl)
{
    if (a.wl_g <= 8) launch_cross_entropy<T, int8_t>(ctx, a, p, wl);
    else if (a.wl_g <= 16) launch_cross_entropy<T, int16_t>(ctx, a, p, wl);
    else launch_cross_entropy<T, int32_t>(ctx, a, p, wl);
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
    // the codes are written while the row is still read
    const uint64_t es = logit_bytes(f), es_g = storage_bytes(fg);
    if (rows_overlap(logits, classes * es, ld * es, dlogits, classes * es_g, ldg * es_g, rows)) return ADAPT_EINVAL;
    LogitArgs a = {};
    a.logits = logits;
    a.rows = rows; a.classes = classes; a.ld = ld;
    a.fl = f.wl == ADAPT_WL_FP32 ? 0 : f.fl;
    a.labels = labels; a.logp = logp; a.weights = weights;
    a.grad = dlogits; a.ldg = ldg;
    a.wl_g = fg.wl; a.fl_g = fg.fl; a.mode = rng.mode; a.seed = rng.seed; a.stream = rng.stream;
    const CrossEntropyPlan p = plan_cross_entropy(ctx->num_cu, rows, classes, f);
    if (p.ws_bytes > scratch_bytes(ctx)) return ADAPT_EWORKSPACE;
    if (f.wl == ADAPT_WL_FP32) launch_cross_entropy_to<float>(ctx, a, p, 0);
    else if (f.wl <= 8) launch_cross_entropy_to<int8_t>(ctx, a, p, f.wl);
    else if (f.wl <= 16) launch_cross_entropy_to<int16_t>(ctx, a, p, f.wl);
    else launch_cross_entropy_to<int32_t>(ctx, a, p, f.wl);
    return hip_status(ctx, hipGetLastError());
}

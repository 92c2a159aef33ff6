// What the routing kernels share: arguments, scores, the choice in 64 bits, lists of the largest keys.
#pragma once

#include <cfloat>
#include <cmath>

#include "layer_common.cuh"

namespace route {

using namespace layer;

constexpr int kMaxE = 1024;
constexpr int kMaxK = 64;
constexpr int kMaxGroups = 64;
constexpr unsigned kAll = 0xffffffffu;

struct RouteArgs {
    const void* logits;
    const float* bias;
    const uint8_t* mask;
    int32_t* topk;
    float* weights;
    int64_t N, T, ld;
    float scale;
    int32_t E, k, score, groups, kept, top, renormalise, dtype;
    int32_t chunk_bits;               // the number of chunks of four experts is below 1 << chunk_bits
};

template <typename T> struct Type;
template <> struct Type<float> { static constexpr int32_t code = TAOT_F32; static constexpr float big = FLT_MAX; };
template <> struct Type<__nv_bfloat16> { static constexpr int32_t code = TAOT_BF16; static constexpr float big = 3.38953139e38f; };
template <> struct Type<__half> { static constexpr int32_t code = TAOT_F16; static constexpr float big = 65504.0f; };

// A logit as every kernel here sees it: -infinity if the expert is closed, an infinite one as the largest finite value of the type
__device__ __forceinline__ float seen(float v, float big) { return v > -big ? fminf(v, big) : -INFINITY; }     // (false for a NaN)
__device__ __forceinline__ float logit_at(const void* p, int64_t i, int32_t dtype)
{
    if (dtype == TAOT_F32) return seen(static_cast<const float*>(p)[i], Type<float>::big);
    if (dtype == TAOT_BF16) return seen(to_f32(static_cast<const __nv_bfloat16*>(p)[i]), Type<__nv_bfloat16>::big);
    return seen(to_f32(static_cast<const __half*>(p)[i]), Type<__half>::big);
}

// 1 / (1 + exp(-x)) down to the smallest values: the exponential is that of a number that is not positive.  A weight, which
// decides nothing: the quick division, to two ulps
__device__ __forceinline__ float sigmoid(float x)
{
    const float e = expf(-fabsf(x));
    return __fdividef(x < 0.0f ? e : 1.0f, 1.0f + e);
}

// A chosen expert's part of a renormalised weight, before the division by the sum: its score relative to the largest chosen logit
// `most`, so that it is a normal number wherever the weight is one.  Of a sigmoid, which is exp(min(x, 0)) / (1 + exp(-|x|)), what is
// taken out is exp(min(most, 0)).
__device__ __forceinline__ float part_of(int32_t score, float x, float most)
{
    if (score == TAOT_SOFTMAX) return expf(x - most);
    return __fdividef(expf(fminf(x, 0.0f) - fminf(most, 0.0f)), 1.0f + expf(-fabsf(x)));
}

__device__ __forceinline__ float warp_max(float v)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(kAll, v, o));
    return v;
}

// e^x in 64 bits, to about an ulp: x = n ln 2 + r with ln 2 in two parts (Cody and Waite), the Taylor series of e^r (|r| <= ln 2 / 2: its 14th term is
// below 5e-18), and 2^n in two factors, so that results below 2^-1022 are rounded once.  No branches: several run side by side.
__device__ __forceinline__ double exp_of(double x)
{
    x = fmin(fmax(x, -750.0), 750.0);                              // 0 and infinity beyond
    const double whole = 6755399441055744.0;                       // 1.5 * 2^52: what is added to it is rounded to whole numbers
    const double t = fma(x, 1.4426950408889634, whole);
    const int n = __double2loint(t);
    const double nd = t - whole;
    double r = fma(nd, -6.93147180369123816490e-01, x);            // (the upper 33 bits of ln 2: the product is exact)
    r = fma(nd, -1.90821492927058770002e-10, r);
    double p = 1.0 / 6227020800.0;                                 // 1 / 13!
    p = fma(p, r, 1.0 / 479001600.0);
    p = fma(p, r, 1.0 / 39916800.0);
    p = fma(p, r, 1.0 / 3628800.0);
    p = fma(p, r, 1.0 / 362880.0);
    p = fma(p, r, 1.0 / 40320.0);
    p = fma(p, r, 1.0 / 5040.0);
    p = fma(p, r, 1.0 / 720.0);
    p = fma(p, r, 1.0 / 120.0);
    p = fma(p, r, 1.0 / 24.0);
    p = fma(p, r, 1.0 / 6.0);
    p = fma(p, r, 0.5);
    p = fma(p, r, 1.0);
    p = fma(p, r, 1.0);
    const int half = n >> 1;
    return p * __hiloint2double((half + 1023) << 20, 0) * __hiloint2double((n - half + 1023) << 20, 0);
}

// the order-preserving image of a number in 64 bits; closed experts (-infinity) have 0
__device__ __forceinline__ uint64_t ordered(double v)
{
    const long long b = __double_as_longlong(v + 0.0);             // (one zero)
    return v > -INFINITY ? (uint64_t)(b ^ ((b >> 63) | (long long)0x8000000000000000ull)) : 0ull;
}
__device__ __forceinline__ double number_of(uint64_t u)
{
    const long long b = (long long)u;
    return u ? __longlong_as_double(b ^ (~(b >> 63) | (long long)0x8000000000000000ull)) : -INFINITY;
}

// the lowest index among the lanes' that has the largest key (kMaxE if that is 0)
__device__ __forceinline__ int warp_argmax(uint64_t u, int i)
{
    const uint32_t hi = (uint32_t)(u >> 32), most_hi = __reduce_max_sync(kAll, hi);
    const uint32_t lo = hi == most_hi ? (uint32_t)u : 0u, most_lo = __reduce_max_sync(kAll, lo);
    return (int)__reduce_min_sync(kAll, hi == most_hi && (uint32_t)u == most_lo && u != 0 ? (unsigned)i : (unsigned)kMaxE);
}

// eight experts of a lane, 32 apart
template <typename T>
__device__ __forceinline__ void read_eight(const RouteArgs& a, int64_t row, int e0, float (&x)[8])
{
    const T* p = static_cast<const T*>(a.logits) + row * a.ld;
#pragma unroll
    for (int u = 0; u < 8; ++u) x[u] = e0 + 32 * u < a.E ? to_f32(p[e0 + 32 * u]) : -INFINITY;
#pragma unroll
    for (int u = 0; u < 8; ++u) x[u] = seen(x[u], Type<T>::big);
}
__device__ __forceinline__ void read_eight(const RouteArgs& a, int64_t row, int e0, float (&x)[8])
{
    if (a.dtype == TAOT_F32) read_eight<float>(a, row, e0, x);
    else if (a.dtype == TAOT_BF16) read_eight<__nv_bfloat16>(a, row, e0, x);
    else read_eight<__half>(a, row, e0, x);
}

// a lane's largest key and the first expert that has it
__device__ __forceinline__ void own_largest(const uint64_t* key, int E, uint64_t& u, int& i)
{
    u = 0;
    i = kMaxE;
    for (int e0 = threadIdx.x & 31; e0 < E; e0 += 256) {
        uint64_t v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = e0 + 32 * q < E ? key[e0 + 32 * q] : 0ull;
#pragma unroll
        for (int q = 0; q < 8; ++q)
            if (v[q] > u) { u = v[q]; i = e0 + 32 * q; }
    }
}

// The chosen experts of one row, by arithmetic in 64 bits, by a whole warp: lane j % 32 holds place j in at0 (j < 32) or at1, -1
// where no expert is left.  key [E] is shared memory of the warp.  top and total: the largest open logit and the sum of
// exp(logit - top).  Few rows come here, but a warp that has one is the last to end: loads and exponentials go eight at a time, and
// a lane keeps its largest key at hand.
static __device__ __noinline__ void choose_exactly(const RouteArgs& a, int64_t row, uint64_t* key, int& at0, int& at1, float& top_out, float& total_out)
{
    const int lane = threadIdx.x & 31;
    const float* bias = a.bias ? a.bias + row / a.T * a.E : nullptr;
    const bool scored = bias || a.groups > 1;                      // keys are scores
    float top = -INFINITY;
    for (int e0 = lane; e0 < a.E; e0 += 256) {
        float x[8];
        read_eight(a, row, e0, x);
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            top = fmaxf(top, x[u]);
            if (e0 + 32 * u < a.E) key[e0 + 32 * u] = ordered((double)x[u]);
        }
    }
    top = warp_max(top);
    double total = 0.0;
    if (a.score == TAOT_SOFTMAX && top > -INFINITY) {
        for (int e0 = lane; e0 < a.E; e0 += 256) {
            float x[8];
            read_eight(a, row, e0, x);
#pragma unroll
            for (int u = 0; u < 8; ++u) total += exp_of((double)x[u] - (double)top);
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(kAll, total, o);
    }
    top_out = top;
    total_out = (float)total;
    if (scored) {
        const double inv = 1.0 / total;
        for (int e0 = lane; e0 < a.E; e0 += 256) {
            float x[8], b[8];
            read_eight(a, row, e0, x);
#pragma unroll
            for (int u = 0; u < 8; ++u) b[u] = bias && e0 + 32 * u < a.E ? bias[e0 + 32 * u] : 0.0f;
            double s[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) s[u] = exp_of(a.score == TAOT_SOFTMAX ? (double)x[u] - (double)top : -(double)x[u]);
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                s[u] = a.score == TAOT_SOFTMAX ? s[u] * inv : __drcp_rn(1.0 + s[u]);
                if (e0 + 32 * u < a.E) key[e0 + 32 * u] = x[u] > -INFINITY && isfinite(b[u]) ? ordered(s[u] + (double)b[u]) : 0ull;
            }
        }
    }
    __syncwarp();
    if (a.groups > 1) {
        const int size = a.E / a.groups;
        uint64_t score0 = 0, score1 = 0;                           // of groups lane and lane + 32
        for (int g = lane; g < a.groups; g += 32) {
            uint64_t m1 = 0, m2 = 0;
            int e = lane % size;                                   // (each lane from another place on: other banks)
#pragma unroll 8
            for (int i = 0; i < size; ++i) {
                const uint64_t v = key[g * size + e];
                e = e + 1 == size ? 0 : e + 1;
                m2 = max(m2, min(m1, v));
                m1 = max(m1, v);
            }
            const uint64_t s = a.top == 2 && m2 ? ordered(number_of(m1) + number_of(m2)) : m1;
            if (g < 32) score0 = s; else score1 = s;
        }
        uint64_t kept = 0, left = a.groups == 64 ? ~0ull : (1ull << a.groups) - 1;
        for (int i = 0; i < a.kept; ++i) {
            const uint64_t v0 = left >> lane & 1 ? score0 : 0ull, v1 = left >> (lane + 32) & 1 ? score1 : 0ull;
            const bool second = v1 > v0;
            int g = warp_argmax(second ? v1 : v0, second ? lane + 32 : lane);
            if (g == kMaxE) g = __ffsll((long long)left) - 1;      // groups without open experts come last, in order
            kept |= 1ull << g;
            left &= ~(1ull << g);
        }
        for (int e0 = lane; e0 < a.E; e0 += 256) {
            float x[8];
            if (!bias) read_eight(a, row, e0, x);
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int e = e0 + 32 * u;
                if (e >= a.E) continue;
                if (!((kept >> (e / size)) & 1)) key[e] = 0ull;
                else if (!bias) key[e] = ordered((double)x[u]);
            }
        }
    }
    uint64_t v;
    int i;
    own_largest(key, a.E, v, i);
    at0 = at1 = -1;
    for (int j = 0; j < a.k; ++j) {
        const int e = warp_argmax(v, i);
        if (e == kMaxE) break;                                     // (the same for all lanes)
        if ((j & 31) == lane) {
            if (j < 32) at0 = e; else at1 = e;
        }
        if (e == i) {
            key[e] = 0ull;
            own_largest(key, a.E, v, i);
        }
    }
    __syncwarp();
}

// Writes a row's table entries and weights, by a whole warp: lane j % 32 holds place j in at0 (j < 32) or at1.
static __device__ __noinline__ void write_row(const RouteArgs& a, int64_t row, int at0, int at1, float top, float total)
{
    const int lane = threadIdx.x & 31;
    const int at[2] = {at0, at1};
    float x[2], w[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) x[h] = at[h] >= 0 ? logit_at(a.logits, row * a.ld + at[h], a.dtype) : -INFINITY;
    if (a.renormalise) {
        const float most = warp_max(fmaxf(x[0], x[1]));
#pragma unroll
        for (int h = 0; h < 2; ++h) w[h] = at[h] < 0 ? 0.0f : part_of(a.score, x[h], most);
        const float sum = warp_sum(w[0] + w[1]);
#pragma unroll
        for (int h = 0; h < 2; ++h) w[h] = at[h] < 0 ? 0.0f : w[h] / sum;
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) w[h] = at[h] < 0 ? 0.0f : a.score == TAOT_SOFTMAX ? expf(x[h] - top) / total : sigmoid(x[h]);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int j = lane + 32 * h;
        if (j < a.k) {
            a.topk[row * a.k + j] = at[h];
            if (a.weights) a.weights[row * a.k + j] = a.scale * w[h];
        }
    }
}

// ---------------------------------------------------------------------------------------------------------------------
// Lists of the K = 8 or 16 largest keys.
//
// The K largest of a row are found by lists of 32-bit keys in descending order: the row is cut into chunks of four experts, whose
// largest keys (with the chunk's number in the low bits, so that ties go to the lower one) are sorted and merged until the K
// best chunks are left; they hold the K best experts, whose keys are sorted and merged the same way, with the expert's place
// among the chosen chunks in the low bits.  Every comparison is a minimum and a maximum of 32-bit words: no branches, and no
// index travels beside a value.
//
// A key is the order-preserving image of an fp32 number v (the logit, or score + bias) without its lowest bits, so that
//  - experts whose v differ in those bits alone may stand in the wrong order: the chosen ones are put right by their full v;
//  - it may be open which of two experts is the last chosen one: then the row is done again by choose_exactly, as it is where
//    two scores are closer than the error of their fp32 arithmetic.
// Keys of 16-bit logits lose nothing, nor do fp32 logits that hold 16-bit numbers.

__device__ __forceinline__ uint32_t ordered(float v)              // larger numbers have larger images
{
    const int32_t i = __float_as_int(v);
    return (uint32_t)(i ^ ((i >> 31) | (int32_t)0x80000000));
}
__device__ __forceinline__ float number_of(uint32_t u)
{
    const int32_t i = (int32_t)u;
    return __int_as_float(i ^ (~(i >> 31) | (int32_t)0x80000000));
}

__device__ __forceinline__ void order(uint32_t& a, uint32_t& b)
{
    const uint32_t x = max(a, b), y = min(a, b);
    a = x; b = y;
}

// sorts N of the list that first rise and then fall, or the other way round, largest first
template <int K, int N>
__device__ __forceinline__ void sort_slope(uint32_t (&v)[K], int at)
{
#pragma unroll
    for (int q = N / 2; q >= 1; q /= 2)
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (!(i & q)) order(v[at + i], v[at + i + q]);
}

// 19 comparisons for eight (Batcher's odd-even merge sort), 70 for sixteen
template <int K>
__device__ __forceinline__ void sort_list(uint32_t (&v)[K])
{
#pragma unroll
    for (int b = 0; b < K; b += 8) {
#pragma unroll
        for (int i = 0; i < 8; i += 2) order(v[b + i], v[b + i + 1]);
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
            order(v[b + i], v[b + i + 2]); order(v[b + i + 1], v[b + i + 3]); order(v[b + i + 1], v[b + i + 2]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) order(v[b + i], v[b + i + 4]);
        order(v[b + 2], v[b + 4]); order(v[b + 3], v[b + 5]);
        order(v[b + 1], v[b + 2]); order(v[b + 3], v[b + 4]); order(v[b + 5], v[b + 6]);
    }
    if constexpr (K == 16) {
#pragma unroll
        for (int i = 0; i < 8; ++i) order(v[i], v[15 - i]);
        sort_slope<K, 8>(v, 0);
        sort_slope<K, 8>(v, 8);
    }
}

// the K largest of two sorted lists in v, sorted; the largest of the others in lost
template <bool LOST, int K>
__device__ __forceinline__ void merge_list(uint32_t (&v)[K], const uint32_t (&w)[K], uint32_t& lost)
{
#pragma unroll
    for (int i = 0; i < K; ++i) {
        const uint32_t a = v[i], b = w[K - 1 - i];
        v[i] = max(a, b);
        if (LOST) lost = max(lost, min(a, b));
    }
    sort_slope<K, K>(v, 0);
}

__device__ __forceinline__ float fast_exp2(float v)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));        // relative error at most 2^-22
    return r;
}
__device__ __forceinline__ float fast_reciprocal(float v)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));        // relative error at most 2^-23
    return r;
}

// The score of an open logit in fp32, which decides where 64 bits are not needed, and how far it may be off.  (Weights have their own
// exponentials, by expf; one that is not renormalised takes the softmax's sum from these, whose error is 2^-22 of the largest terms.)  The exponent t is rounded twice, by |t| 2^-24 each.
//   sigmoid: the exponential is off by 2 |t| 2^-24 ln 2 + 2^-22 of itself, the score by that times s (1 - s) (|t| s (1 - s) stays
//            below 0.33, s (1 - s) below 1 / 4), and by 2^-23 and 2^-24 of itself: 2.8e-8 + 6e-8 + 1.8e-7 < 3e-7 in all;
//   softmax: the same of the exponential, with p |t| below 0.54 p_max; and the sum, in which `terms` terms follow one another.
struct Scores {
    float top, inv;               // largest logit, reciprocal of the sum of exponentials (softmax)
};
constexpr float kLog2e = 1.44269504f;
__device__ __forceinline__ float score_of(int32_t score, const Scores& s, float x)
{
    return score == TAOT_SIGMOID ? fast_reciprocal(1.0f + fast_exp2(-x * kLog2e)) : fast_exp2((x - s.top) * kLog2e) * s.inv;
}
__device__ __forceinline__ float score_error(int32_t score, const Scores& s, int terms)
{
    return score == TAOT_SIGMOID ? 3e-7f : s.inv * ((float)(terms + 16) * 1.2e-7f);
}

// ---------------------------------------------------------------------------------------------------------------------
// What fp32 leaves open, settled in 64 bits for the few experts that it is open for.  A warp works on one row.  Few rows come here,
// but a warp that has one is the last to end, and its code is not in the instruction cache: it is kept short.

// the key of a chosen form in 64 bits: the score (+ bias), or the logit
__device__ __forceinline__ uint64_t exact_key(const RouteArgs& a, const float* bias, bool scored, int64_t row, int e, float top, double inv)
{
    const float x = logit_at(a.logits, row * a.ld + e, a.dtype);
    if (!scored) return ordered((double)x);
    const float b = bias ? bias[e] : 0.0f;
    double s = exp_of(a.score == TAOT_SOFTMAX ? (double)x - (double)top : -(double)x);
    s = a.score == TAOT_SOFTMAX ? s * inv : __drcp_rn(1.0 + s);
    return x > -INFINITY && isfinite(b) ? ordered(s + (double)b) : 0ull;
}

// the reciprocal of the sum of exp(logit - top) over a row
__device__ __forceinline__ double exact_inverse(const RouteArgs& a, int64_t row, float top)
{
    double total = 0.0;
    for (int e = threadIdx.x & 31; e < a.E; e += 32) total += exp_of((double)logit_at(a.logits, row * a.ld + e, a.dtype) - (double)top);
#pragma unroll
    for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(kAll, total, o);
    return 1.0 / total;
}

// The experts of a row that may matter: those of the groups in `kept` whose key in fp32 is at least `least` of their group (held by
// lane at + group * step).  Up to 32 of them go to `found`; returns how many there are.
__device__ __forceinline__ int gather(const RouteArgs& a, const float* bias, bool scored, int64_t row, const Scores& sc, uint32_t kept, float least,
                                      int at, int step, int32_t* found)
{
    const int lane = threadIdx.x & 31, size = a.E / a.groups;
    int count = 0;
    for (int e0 = lane; e0 < a.E + lane; e0 += 256) {              // eight at a time, so that their latencies overlap
        float v[8], b[8];
        read_eight(a, row, e0, v);
#pragma unroll
        for (int u = 0; u < 8; ++u) b[u] = scored && bias && e0 + 32 * u < a.E ? bias[e0 + 32 * u] : 0.0f;
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            if (e0 - lane + 32 * u >= a.E) break;                  // (the same for all lanes)
            const int e = e0 + 32 * u, g = min(e, a.E - 1) / size;
            if (scored && bias && v[u] > -INFINITY) v[u] = isfinite(b[u]) ? score_of(a.score, sc, v[u]) + b[u] : -INFINITY;
            const float limit = __shfl_sync(kAll, least, at + g * step);
            const bool hit = v[u] > -INFINITY && v[u] >= limit && (kept >> g & 1);
            const unsigned all = __ballot_sync(kAll, hit);
            const int place = count + __popc(all & ((1u << lane) - 1));
            if (hit && place < 32) found[place] = e;
            count += __popc(all);
        }
    }
    __syncwarp();
    return count;
}

// Which groups are kept (of at most 8), where their scores in fp32 are too close: from the experts whose keys are at least `least`, a
// lower bound of the last key that counts in a group.  Returns false where there are too many of them.
static __device__ __noinline__ bool settle_groups(const RouteArgs& a, int64_t row, const Scores sc, float least, int at, int step, int32_t* found, uint32_t& kept)
{
    const int lane = threadIdx.x & 31, size = a.E / a.groups;
    const float* bias = a.bias ? a.bias + row / a.T * a.E : nullptr;
    const int count = gather(a, bias, true, row, sc, 0xffffffffu, least, at, step, found);
    if (count > 32) return false;
    const double inv = a.score == TAOT_SOFTMAX ? exact_inverse(a, row, sc.top) : 1.0;
    const int e = lane < count ? found[lane] : 0;
    const uint64_t mine = lane < count ? exact_key(a, bias, true, row, e, sc.top, inv) : 0ull;
    uint64_t score = 0;                                            // of group `lane`
    for (int g = 0; g < a.groups; ++g) {
        uint64_t u = lane < count && e / size == g ? mine : 0ull, m[2] = {0, 0};
        for (int i = 0; i < a.top; ++i) {
            const int who = warp_argmax(u, lane);
            if (who == kMaxE) break;
            m[i] = __shfl_sync(kAll, u, who);
            if (lane == who) u = 0;
        }
        if (lane == g) score = m[1] ? ordered(number_of(m[0]) + number_of(m[1])) : m[0];
    }
    int rank = 0;
    for (int g = 0; g < a.groups; ++g) {
        const uint64_t u = __shfl_sync(kAll, score, g);
        if (u > score || (u == score && g < lane)) ++rank;
    }
    kept = __ballot_sync(kAll, lane < a.groups && rank < a.kept);
    __syncwarp();
    return true;
}

// The chosen experts of a row (at most 16; -1 where there is none) go to `found`, from those whose key in fp32 is at least `least`, a lower
// bound of the last chosen one's.  Returns false where there are too many of them.
static __device__ __noinline__ bool settle_choice(const RouteArgs& a, int64_t row, const Scores sc, uint32_t kept, float least, int32_t* found)
{
    const int lane = threadIdx.x & 31;
    const float* bias = a.bias ? a.bias + row / a.T * a.E : nullptr;
    const int count = gather(a, bias, bias != nullptr, row, sc, kept, least, 0, 0, found);
    if (count > 32) return false;
    const double inv = bias && a.score == TAOT_SOFTMAX ? exact_inverse(a, row, sc.top) : 1.0;
    const int e = lane < count ? found[lane] : kMaxE;
    const uint64_t mine = lane < count ? exact_key(a, bias, bias != nullptr, row, e, sc.top, inv) : 0ull;
    int rank = 0;
    for (int i = 0; i < count; ++i) {
        const uint64_t u = __shfl_sync(kAll, mine, i);
        const int f = __shfl_sync(kAll, e, i);
        if (u > mine || (u == mine && f < e)) ++rank;
    }
    __syncwarp();
    found[lane] = -1;
    __syncwarp();
    if (lane < count) found[rank] = e;
    __syncwarp();
    return true;
}

// four consecutive logits as numbers
__device__ __forceinline__ void four(const float* p, float (&x)[4])
{
    const float4 v = *reinterpret_cast<const float4*>(p);
    x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
}
__device__ __forceinline__ void four(const __nv_bfloat16* p, float (&x)[4])
{
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    x[0] = __uint_as_float(v.x << 16); x[1] = __uint_as_float(v.x & 0xffff0000u);
    x[2] = __uint_as_float(v.y << 16); x[3] = __uint_as_float(v.y & 0xffff0000u);
}
__device__ __forceinline__ void four(const __half* p, float (&x)[4])
{
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    const float2 lo = __half22float2(*reinterpret_cast<const __half2*>(&v.x)), hi = __half22float2(*reinterpret_cast<const __half2*>(&v.y));
    x[0] = lo.x; x[1] = lo.y; x[2] = hi.x; x[3] = hi.y;
}

// launches the kernels of rows that a warp's lanes share (route_lanes.cu)
cudaError_t launch_lanes(const RouteArgs& a, bool wide, cudaStream_t st);

// the kernels of rows that a lane has to itself (route_stream.cu), and whether they take a call
bool streams(const RouteArgs& a, bool wide);
cudaError_t launch_stream(const RouteArgs& a, cudaStream_t st);

}  // namespace route

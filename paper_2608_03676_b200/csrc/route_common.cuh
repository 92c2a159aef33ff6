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

// 1 / (1 + exp(-x)) down to the smallest values: the exponential is that of a number that is not positive
__device__ __forceinline__ float sigmoid(float x)
{
    const float e = expf(-fabsf(x));
    return __fdividef(x < 0.0f ? e : 1.0f, 1.0f + e);
}

__device__ __forceinline__ double warp_max(double v)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fmax(v, __shfl_xor_sync(kAll, v, o));
    return v;
}
__device__ __forceinline__ float warp_max(float v)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(kAll, v, o));
    return v;
}

// the lowest index among the lanes' that has the largest value (kMaxE if that is -infinity)
__device__ __forceinline__ int warp_argmax(double v, int i)
{
    const long long b = __double_as_longlong(v + 0.0);                       // one zero
    const unsigned long long u = (unsigned long long)b ^ (b < 0 ? ~0ull : 1ull << 63);
    const uint32_t hi = (uint32_t)(u >> 32), most_hi = __reduce_max_sync(kAll, hi);
    const uint32_t lo = hi == most_hi ? (uint32_t)u : 0u, most_lo = __reduce_max_sync(kAll, lo);
    return (int)__reduce_min_sync(kAll, hi == most_hi && (uint32_t)u == most_lo && v > -INFINITY ? (unsigned)i : (unsigned)kMaxE);
}

// The chosen experts of one row, by arithmetic in 64 bits, by a whole warp: lane j % 32 holds place j in at0 (j < 32) or at1, -1
// where no expert is left.  key [E] is shared memory of the warp.  top and total: the largest open logit and the sum of
// exp(logit - top).
static __device__ __noinline__ void choose_exactly(const RouteArgs& a, int64_t row, double* key, int& at0, int& at1, float& top_out, float& total_out)
{
    const int lane = threadIdx.x & 31;
    const float* bias = a.bias ? a.bias + row / a.T * a.E : nullptr;
    double top = -INFINITY, total = 0.0;
    for (int e = lane; e < a.E; e += 32) {
        const double x = logit_at(a.logits, row * a.ld + e, a.dtype);
        key[e] = x;
        top = fmax(top, x);
    }
    top = warp_max(top);
    if (a.score == TAOT_SOFTMAX && top > -INFINITY) {
        for (int e = lane; e < a.E; e += 32) total += exp(key[e] - top);
#pragma unroll
        for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(kAll, total, o);
    }
    top_out = (float)top;
    total_out = (float)total;
    if (bias || a.groups > 1)
        for (int e = lane; e < a.E; e += 32) {
            const double x = key[e], b = bias ? (double)bias[e] : 0.0;
            const double s = a.score == TAOT_SOFTMAX ? exp(x - top) / total : 1.0 / (1.0 + exp(-x));
            key[e] = x > -INFINITY && isfinite(b) ? s + b : -INFINITY;
        }
    __syncwarp();
    if (a.groups > 1) {
        const int size = a.E / a.groups;
        double score0 = -INFINITY, score1 = -INFINITY;             // of groups lane and lane + 32
        for (int g = lane; g < a.groups; g += 32) {
            double m1 = -INFINITY, m2 = -INFINITY;
            for (int e = g * size; e < (g + 1) * size; ++e) {
                const double v = key[e];
                m2 = fmax(m2, fmin(m1, v));
                m1 = fmax(m1, v);
            }
            const double s = a.top == 2 && m2 > -INFINITY ? m1 + m2 : m1;
            if (g < 32) score0 = s; else score1 = s;
        }
        uint64_t kept = 0, left = a.groups == 64 ? ~0ull : (1ull << a.groups) - 1;
        for (int i = 0; i < a.kept; ++i) {
            const bool l0 = left >> lane & 1, l1 = left >> (lane + 32) & 1;
            const double v0 = l0 ? score0 : -INFINITY, v1 = l1 ? score1 : -INFINITY;
            int g = v1 > v0 ? warp_argmax(v1, lane + 32) : warp_argmax(v0, lane);
            if (g == kMaxE) g = __ffsll((long long)left) - 1;      // groups without open experts come last, in order
            kept |= 1ull << g;
            left &= ~(1ull << g);
        }
        for (int e = lane; e < a.E; e += 32) {
            const bool in_group = (kept >> (e / size)) & 1;
            if (!in_group) key[e] = -INFINITY;
            else if (!bias) key[e] = logit_at(a.logits, row * a.ld + e, a.dtype);
        }
    }
    // a lane's own largest, renewed by the lane that loses it
    double v = -INFINITY;
    int i = kMaxE;
    for (int e = lane; e < a.E; e += 32)
        if (key[e] > v) { v = key[e]; i = e; }
    at0 = at1 = -1;
    for (int j = 0; j < a.k; ++j) {
        const int e = warp_argmax(v, i);
        if (e == kMaxE) break;                                     // (the same for all lanes)
        if ((j & 31) == lane) {
            if (j < 32) at0 = e; else at1 = e;
        }
        if (e == i) {
            key[e] = -INFINITY;
            v = -INFINITY;
            i = kMaxE;
            for (int f = lane; f < a.E; f += 32)
                if (key[f] > v) { v = key[f]; i = f; }
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
        // relative to the largest chosen score, where the scores would leave the range of fp32 (below -40, where
        // 1 / (1 + exp(-x)) is exp(x) to 18 digits) or are a softmax
        const float most = warp_max(fmaxf(x[0], x[1]));
        const bool shift = a.score == TAOT_SOFTMAX || most < -40.0f;
#pragma unroll
        for (int h = 0; h < 2; ++h) w[h] = at[h] < 0 ? 0.0f : shift ? expf(x[h] - most) : sigmoid(x[h]);
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

// The score of an open logit in fp32, and how far it may be off.  The exponent t is rounded twice, by |t| 2^-24 each.
//   sigmoid: the exponential is off by 2 |t| 2^-24 ln 2 + 2^-22 of itself, the score by that times s (1 - s) (|t| s (1 - s) stays
//            below 0.33), and by 2^-23 and 2^-24 of itself: less than 4e-7 in all;
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
    return score == TAOT_SIGMOID ? 4e-7f : s.inv * ((float)(terms + 16) * 1.2e-7f);
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

}  // namespace route

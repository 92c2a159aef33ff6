// Routing of tokens to experts, and the gradient of the experts' weights (taot_layer.h).
#include <cfloat>
#include <cmath>

#include "layer_common.cuh"

namespace {

using namespace layer;

constexpr int kMaxE = 1024;
constexpr int kMaxK = 64;
constexpr int kMaxGroups = 64;
constexpr int kWarps = 4;                          // rows of a CTA, one per warp
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
};

// A logit as every kernel here sees it: -infinity if the expert is closed, an infinite one as the largest finite value of the type
__device__ __forceinline__ float logit_at(const void* p, int64_t i, int32_t dtype)
{
    float v, big;
    if (dtype == TAOT_F32) { v = static_cast<const float*>(p)[i]; big = FLT_MAX; }
    else if (dtype == TAOT_BF16) { v = to_f32(static_cast<const __nv_bfloat16*>(p)[i]); big = 3.38953139e38f; }
    else { v = to_f32(static_cast<const __half*>(p)[i]); big = 65504.0f; }
    return v > -big ? fminf(v, big) : -INFINITY;   // (false for a NaN)
}

// (down to the smallest values: the exponential is that of a number that is not positive)
__device__ __forceinline__ float sigmoid(float x)
{
    const float e = expf(-fabsf(x));
    return (x < 0.0f ? e : 1.0f) / (1.0f + e);
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

// the largest value of a warp and the lowest index that has it
__device__ __forceinline__ void warp_argmax(double& v, int& i)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        const double u = __shfl_xor_sync(kAll, v, o);
        const int j = __shfl_xor_sync(kAll, i, o);
        if (u > v || (u == v && j < i)) { v = u; i = j; }
    }
}

// The chosen experts of one row, by arithmetic in 64 bits: lane j % 32 holds place j in at[j / 32], -1 where no expert is left.
// key [E] is shared memory of the warp.  top and total: the largest open logit and the sum of exp(logit - top).
__device__ void choose_exactly(const RouteArgs& a, int64_t row, double* key, int (&at)[2], double& top, double& total)
{
    const int lane = threadIdx.x & 31;
    const float* bias = a.bias ? a.bias + row / a.T * a.E : nullptr;
    top = -INFINITY;
    for (int e = lane; e < a.E; e += 32) {
        const double x = logit_at(a.logits, row * a.ld + e, a.dtype);
        key[e] = x;
        top = fmax(top, x);
    }
    top = warp_max(top);
    total = 0.0;
    if (a.score == TAOT_SOFTMAX && top > -INFINITY) {
        for (int e = lane; e < a.E; e += 32) total += exp(key[e] - top);
#pragma unroll
        for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(kAll, total, o);
    }
    if (bias || a.groups > 1)
        for (int e = lane; e < a.E; e += 32) {
            const double x = key[e], b = bias ? (double)bias[e] : 0.0;
            const double s = a.score == TAOT_SOFTMAX ? exp(x - top) / total : 1.0 / (1.0 + exp(-x));
            key[e] = x > -INFINITY && isfinite(b) ? s + b : -INFINITY;
        }
    __syncwarp();
    if (a.groups > 1) {
        const int size = a.E / a.groups;
        double score[2] = {-INFINITY, -INFINITY};
        for (int h = 0; h < 2; ++h) {
            const int g = lane + 32 * h;
            if (g >= a.groups) continue;
            double m1 = -INFINITY, m2 = -INFINITY;
            for (int e = g * size; e < (g + 1) * size; ++e) {
                const double v = key[e];
                if (v > m1) { m2 = m1; m1 = v; }
                else if (v > m2) m2 = v;
            }
            score[h] = a.top == 2 && m2 > -INFINITY ? m1 + m2 : m1;
        }
        bool in[2] = {false, false};
        bool left[2] = {lane < a.groups, lane + 32 < a.groups};
        for (int i = 0; i < a.kept; ++i) {
            double v = -INFINITY;
            int g = kMaxGroups;
            for (int h = 1; h >= 0; --h)
                if (left[h] && score[h] >= v) { v = score[h]; g = lane + 32 * h; }
            warp_argmax(v, g);
            for (int h = 0; h < 2; ++h)
                if (g == lane + 32 * h) { in[h] = true; left[h] = false; }
        }
        const uint64_t kept = (uint64_t)__ballot_sync(kAll, in[0]) | (uint64_t)__ballot_sync(kAll, in[1]) << 32;
        for (int e = lane; e < a.E; e += 32) {
            const bool in_group = (kept >> (e / size)) & 1;
            if (!in_group) key[e] = -INFINITY;
            else if (!bias) key[e] = logit_at(a.logits, row * a.ld + e, a.dtype);
        }
        __syncwarp();
    }
    at[0] = at[1] = -1;
    for (int j = 0; j < a.k; ++j) {
        double v = -INFINITY;
        int i = kMaxE;
        for (int e = lane; e < a.E; e += 32)
            if (key[e] > v) { v = key[e]; i = e; }
        warp_argmax(v, i);
        if (v == -INFINITY) break;                 // (the same for all lanes)
        if ((j & 31) == lane) at[j >> 5] = i;
        if (lane == 0) key[i] = -INFINITY;
        __syncwarp();
    }
}

// Writes a row's table entries and weights: lane j % 32 holds place j in at[j / 32].
__device__ __forceinline__ void write_row(const RouteArgs& a, int64_t row, const int (&at)[2], float top, float total)
{
    const int lane = threadIdx.x & 31;
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

__global__ void __launch_bounds__(kWarps * 32)
route_kernel(RouteArgs a)
{
    extern __shared__ double keys[];
    const int64_t row = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
    if (row >= a.N) return;
    int at[2] = {-1, -1};
    double top = 0.0, total = 1.0;
    if (!a.mask || a.mask[row]) choose_exactly(a, row, keys + (threadIdx.x >> 5) * a.E, at, top, total);
    write_row(a, row, at, (float)top, (float)total);
}

struct RouteGradArgs {
    const void* logits;
    const int32_t* topk;
    const float* dweights;
    void* dlogits;
    int64_t N, ld, ld_out;
    float scale;
    int32_t E, k, score, renormalise, dtype;
};

__device__ __forceinline__ void put(void* p, int64_t i, int32_t dtype, float v)
{
    if (dtype == TAOT_F32) static_cast<float*>(p)[i] = v;
    else if (dtype == TAOT_BF16) static_cast<__nv_bfloat16*>(p)[i] = from_f32<__nv_bfloat16>(v);
    else static_cast<__half*>(p)[i] = from_f32<__half>(v);
}

// One warp per row, which is put together in shared memory: what reaches every expert, then the chosen ones' share in the
// order of their places.
__global__ void __launch_bounds__(kWarps * 32)
route_grad_kernel(RouteGradArgs a)
{
    extern __shared__ float rows[];
    const int lane = threadIdx.x & 31;
    const int64_t row = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
    if (row >= a.N) return;
    float* out = rows + (threadIdx.x >> 5) * a.E;
    int at[2];
    float g[2], x[2], d[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int j = lane + 32 * h;
        at[h] = j < a.k ? a.topk[row * a.k + j] : -1;
        if ((unsigned)at[h] >= (unsigned)a.E) at[h] = -1;
        g[h] = at[h] >= 0 ? a.scale * a.dweights[row * a.k + j] : 0.0f;
        x[h] = at[h] >= 0 ? logit_at(a.logits, row * a.ld + at[h], a.dtype) : -INFINITY;
    }
    if (a.score == TAOT_SOFTMAX && !a.renormalise) {
        float top = -INFINITY, total = 0.0f;
        for (int e = lane; e < a.E; e += 32) {
            out[e] = logit_at(a.logits, row * a.ld + e, a.dtype);
            top = fmaxf(top, out[e]);
        }
        top = warp_max(top);
        if (top == -INFINITY) top = 0.0f;          // no open expert: every score is zero
        for (int e = lane; e < a.E; e += 32) {
            out[e] = expf(out[e] - top);
            total += out[e];
        }
        total = fmaxf(warp_sum(total), FLT_MIN);
        __syncwarp();
#pragma unroll
        for (int h = 0; h < 2; ++h) d[h] = at[h] >= 0 ? g[h] * (out[at[h]] / total) : 0.0f;
        const float all = warp_sum(d[0] + d[1]) / total;
        __syncwarp();
        for (int e = lane; e < a.E; e += 32) out[e] *= -all;
    } else {
        for (int e = lane; e < a.E; e += 32) out[e] = 0.0f;
        float q[2];
        const float most = warp_max(fmaxf(x[0], x[1]));
        const bool shift = a.score == TAOT_SOFTMAX || most < -40.0f;
#pragma unroll
        for (int h = 0; h < 2; ++h) q[h] = x[h] == -INFINITY ? 0.0f : shift ? expf(x[h] - most) : sigmoid(x[h]);
        if (a.renormalise) {
            const float sum = fmaxf(warp_sum(q[0] + q[1]), FLT_MIN);
            q[0] /= sum; q[1] /= sum;
            const float mean = warp_sum(g[0] * q[0] + g[1] * q[1]);
#pragma unroll
            for (int h = 0; h < 2; ++h) d[h] = q[h] * (g[h] - mean);
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) d[h] = (shift ? q[h] * expf(most) : q[h]) * g[h];
        }
        if (a.score == TAOT_SIGMOID) {
#pragma unroll
            for (int h = 0; h < 2; ++h) d[h] *= sigmoid(-x[h]);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (x[h] == -INFINITY) d[h] = 0.0f;
    }
    __syncwarp();
    for (int j = 0; j < a.k; ++j) {
        const int e = __shfl_sync(kAll, j < 32 ? at[0] : at[1], j & 31);
        const float v = __shfl_sync(kAll, j < 32 ? d[0] : d[1], j & 31);
        if (e >= 0 && (e & 31) == lane) out[e] += v;
    }
    __syncwarp();
    for (int e = lane; e < a.E; e += 32) put(a.dlogits, row * a.ld_out + e, a.dtype, out[e]);
}

int check(const taot_route_params* p)
{
    if (!p) return TAOT_ERR_NULL;
    if (p->struct_size != (int32_t)sizeof(taot_route_params) || !known_type(p->dtype)) return TAOT_ERR_PARAM;
    if (p->L < 0 || p->T < 0 || p->E < 1 || p->k < 1) return TAOT_ERR_PARAM;
    if ((p->score != TAOT_SOFTMAX && p->score != TAOT_SIGMOID) || !std::isfinite(p->scale)) return TAOT_ERR_PARAM;
    if (p->renormalise != 0 && p->renormalise != 1) return TAOT_ERR_PARAM;
    const int64_t most = ((int64_t)1 << 31) - 1;
    if (p->E > kMaxE || p->k > kMaxK || p->L > most || p->T > most || p->L * p->T > most) return TAOT_ERR_UNSUPPORTED;
    if (!good_ld(p->ld_logits, p->E)) return TAOT_ERR_PARAM;
    return TAOT_OK;
}

}  // namespace

extern "C" int taot_route(const taot_route_params* p, const void* d_logits, const float* d_bias, const uint8_t* d_mask,
                          int32_t* d_topk, float* d_weights, void* stream)
{
    if (const int rc = check(p)) return rc;
    if (p->k > p->E || p->groups < 1 || p->groups > p->E || p->E % p->groups != 0 || p->groups_kept < 1 || p->groups_kept > p->groups ||
        (int64_t)p->k > (int64_t)p->groups_kept * (p->E / p->groups) || (p->group_top != 1 && p->group_top != 2))
        return TAOT_ERR_PARAM;
    if (p->groups > kMaxGroups) return TAOT_ERR_UNSUPPORTED;
    const int64_t N = p->L * p->T, e = type_bytes(p->dtype);
    if (N == 0) return TAOT_OK;
    if (!d_logits || !d_topk) return TAOT_ERR_NULL;
    if (misaligned(d_logits, e) || misaligned(d_bias, 4) || misaligned(d_topk, 4) || misaligned(d_weights, 4)) return TAOT_ERR_ALIGN;
    const Range in[] = {range_of(d_logits, N, p->E, p->ld_logits, e), range_of(d_bias, p->L, p->E, p->E, 4), range_of(d_mask, N, 1, 1, 1)};
    const Range out[] = {range_of(d_topk, N, p->k, p->k, 4), range_of(d_weights, N, p->k, p->k, 4)};
    for (const Range& o : out)
        for (const Range& i : in)
            if (overlap(o, i)) return TAOT_ERR_PARAM;
    if (overlap(out[0], out[1])) return TAOT_ERR_PARAM;
    RouteArgs a;
    a.logits = d_logits; a.bias = d_bias; a.mask = d_mask; a.topk = d_topk; a.weights = d_weights;
    a.N = N; a.T = p->T; a.ld = p->ld_logits; a.scale = p->scale;
    a.E = p->E; a.k = p->k; a.score = p->score; a.groups = p->groups; a.kept = p->groups_kept; a.top = p->group_top;
    a.renormalise = p->renormalise; a.dtype = p->dtype;
    route_kernel<<<(unsigned)((N + kWarps - 1) / kWarps), kWarps * 32, sizeof(double) * kWarps * p->E, static_cast<cudaStream_t>(stream)>>>(a);
    TAOT_CUDA_OK(cudaGetLastError());
    return TAOT_OK;
}

extern "C" int taot_route_backward(const taot_route_params* p, const void* d_logits, const int32_t* d_topk,
                                   const float* d_dweights, void* d_dlogits, void* stream)
{
    if (const int rc = check(p)) return rc;
    if (!good_ld(p->ld_dlogits, p->E)) return TAOT_ERR_PARAM;
    const int64_t N = p->L * p->T, e = type_bytes(p->dtype);
    if (N == 0) return TAOT_OK;
    if (!d_logits || !d_topk || !d_dweights || !d_dlogits) return TAOT_ERR_NULL;
    if (misaligned(d_logits, e) || misaligned(d_dlogits, e) || misaligned(d_topk, 4) || misaligned(d_dweights, 4)) return TAOT_ERR_ALIGN;
    const Range in[] = {range_of(d_logits, N, p->E, p->ld_logits, e), range_of(d_topk, N, p->k, p->k, 4), range_of(d_dweights, N, p->k, p->k, 4)};
    const Range out = range_of(d_dlogits, N, p->E, p->ld_dlogits, e);
    for (const Range& i : in)
        if (overlap(out, i)) return TAOT_ERR_PARAM;
    RouteGradArgs a;
    a.logits = d_logits; a.topk = d_topk; a.dweights = d_dweights; a.dlogits = d_dlogits;
    a.N = N; a.ld = p->ld_logits; a.ld_out = p->ld_dlogits; a.scale = p->scale;
    a.E = p->E; a.k = p->k; a.score = p->score; a.renormalise = p->renormalise; a.dtype = p->dtype;
    route_grad_kernel<<<(unsigned)((N + kWarps - 1) / kWarps), kWarps * 32, sizeof(float) * kWarps * p->E, static_cast<cudaStream_t>(stream)>>>(a);
    TAOT_CUDA_OK(cudaGetLastError());
    return TAOT_OK;
}

// Routing of tokens to experts, and the gradient of the experts' weights (taot_layer.h).
#include "route_common.cuh"

namespace {

using namespace layer;
using namespace route;

constexpr int kWarps = 4;                          // rows of a CTA, one per warp

// One warp per row, in 64 bits throughout: more than 16 places, or groups that the other kernels are not made for.
__global__ void __launch_bounds__(kWarps * 32)
route_kernel(const __grid_constant__ RouteArgs a)
{
    extern __shared__ uint64_t keys[];
    const int64_t row = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
    if (row >= a.N) return;
    int at0 = -1, at1 = -1;
    float top = 0.0f, total = 1.0f;
    if (!a.mask || a.mask[row]) choose_exactly(a, row, keys + (threadIdx.x >> 5) * a.E, at0, at1, top, total);
    write_row(a, row, at0, at1, top, total);
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
    a.chunk_bits = 1;
    while ((1 << a.chunk_bits) <= (p->E + 3) / 4) ++a.chunk_bits;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool lists = p->k <= 16 && (p->groups == 1 || ((p->groups == 2 || p->groups == 4 || p->groups == 8) && p->E % 32 == 0));
    if (lists) {
        TAOT_CUDA_OK(launch_lanes(a, wide_rows(d_logits, p->ld_logits, e), st));
    } else {
        route_kernel<<<(unsigned)((N + kWarps - 1) / kWarps), kWarps * 32, sizeof(uint64_t) * kWarps * p->E, st>>>(a);
        TAOT_CUDA_OK(cudaGetLastError());
    }
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

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

// kLanes lanes hold a row, kRuns runs of eight experts each: what reaches every expert (nothing, or for a softmax that is not
// renormalised -c p_e sum_j g_j p_j) is written first, then the chosen experts' whole value over it, each by the lane of its
// first place.  WIDE: rows of whole runs, 16 bytes at a time.
template <typename T, int kLanes, int kRuns, bool WIDE>
struct Row {
    int sub;
    __device__ __forceinline__ int expert(int r, int i) const
    {
        if (!WIDE) return (r * 8 + i) * kLanes + sub;
        return sizeof(T) == 2 ? (r * kLanes + sub) * 8 + i : r * kLanes * 8 + (i >> 2) * kLanes * 4 + 4 * sub + (i & 3);
    }
    __device__ __forceinline__ Run8<T> read(const T* row, int E, int r) const
    {
        constexpr int kPiece = 16 / (int)sizeof(T);
        Run8<T> v;
        if constexpr (WIDE) {
#pragma unroll
            for (int i = 0; i < 8; i += kPiece)
                reinterpret_cast<uint4*>(&v)[i / kPiece] = *reinterpret_cast<const uint4*>(row + min(expert(r, i), E - kPiece));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v.v[i] = row[min(expert(r, i), E - 1)];
        }
        return v;
    }
    // a NaN and what is closed as the lowest value, an infinity as the largest, minus infinity beyond the last expert
    __device__ __forceinline__ void numbers(const Run8<T>& v, int E, int r, float (&x)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = fminf(fmaxf(to_f32(v.v[i]), -Type<T>::big), Type<T>::big);
        if (E != kLanes * 8 * kRuns)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (expert(r, i) >= E) x[i] = -INFINITY;
    }
    __device__ __forceinline__ void write(T* row, int E, int r, const float (&x)[8]) const
    {
        constexpr int kPiece = 16 / (int)sizeof(T);
        const Run8<T> v = narrowed<T>(x);
        if constexpr (WIDE) {
#pragma unroll
            for (int i = 0; i < 8; i += kPiece)
                if (expert(r, i) < E) *reinterpret_cast<uint4*>(row + expert(r, i)) = reinterpret_cast<const uint4*>(&v)[i / kPiece];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (expert(r, i) < E) row[expert(r, i)] = v.v[i];
        }
    }
};
template <int kLanes>
__device__ __forceinline__ float lanes_max(float v)
{
#pragma unroll
    for (int o = 1; o < kLanes; o *= 2) v = fmaxf(v, __shfl_xor_sync(kAll, v, o));
    return v;
}
template <int kLanes>
__device__ __forceinline__ float lanes_sum(float v)
{
#pragma unroll
    for (int o = 1; o < kLanes; o *= 2) v += __shfl_xor_sync(kAll, v, o);
    return v;
}

template <typename T, int kLanes, int kRuns, bool WIDE, bool DENSE>
__global__ void __launch_bounds__(kWarps * 32)
route_grad_kernel(const __grid_constant__ RouteGradArgs a)
{
    constexpr float big = Type<T>::big;
    const int lane = threadIdx.x & 31;
    const int64_t first = ((int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5)) * (32 / kLanes);
    if (first >= a.N) return;
    const int64_t mine = first + lane / kLanes, row = mine < a.N ? mine : a.N - 1;       // (lanes past the end write nothing)
    const Row<T, kLanes, kRuns, WIDE> cols = {lane & (kLanes - 1)};
    const T* x_row = static_cast<const T*>(a.logits) + row * a.ld;
    T* out = static_cast<T*>(a.dlogits) + row * a.ld_out;
    int at[2];
    float g[2], x[2], d[2], base[2] = {0.0f, 0.0f};
    Run8<T> raw[DENSE ? kRuns : 1];                // (read before the table is waited for)
    if (DENSE) {
#pragma unroll
        for (int r = 0; r < kRuns; ++r) raw[r] = cols.read(x_row, a.E, r);
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int j = cols.sub + kLanes * h;
        at[h] = j < a.k ? a.topk[row * a.k + j] : -1;
        g[h] = j < a.k ? a.scale * a.dweights[row * a.k + j] : 0.0f;
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if ((unsigned)at[h] >= (unsigned)a.E) { at[h] = -1; g[h] = 0.0f; }
        x[h] = at[h] >= 0 ? seen(to_f32(x_row[at[h]]), big) : -INFINITY;
    }
    if (DENSE) {
        float e[kRuns][8], top = -INFINITY, total = 0.0f;
#pragma unroll
        for (int r = 0; r < kRuns; ++r) {
            cols.numbers(raw[r], a.E, r, e[r]);
#pragma unroll
            for (int i = 0; i < 8; ++i) top = fmaxf(top, e[r][i]);
        }
        top = lanes_max<kLanes>(top);
        // Exponentials relative to the largest, times 2^64, so that small ones stay normal numbers; the factor goes with their
        // sum's reciprocal.
        //   fp32 logits: the square of exp((x - top) / 2), to three ulps and the rounding of the difference.
        //   (2 x 65536 x 256: 51 us, 49 with the form below, which is off by up to 2^-19 of a value.)
        //   16 bits: one multiply-add each, whose rounding (of numbers up to 64 and more) leaves an error of 2^-19, far below half a step
        //   of the result (2^-11 or 2^-8); that of top * log2 e is common to the row and goes the same way.  Only where that is no
        //   small number, or the lowest value is not far below, the careful form is needed.
        constexpr bool kExact = sizeof(T) == 4;
        const auto whole = [&](float v) {
            const float half = expf(0.5f * (v - top)) * 0x1p32f;
            return half * half;
        };
        const bool careful = !kExact && __any_sync(kAll, fabsf(top) > 65536.0f || top < -0.5f * big);
        const float shift = 64.0f - top * kLog2e;
        if (kExact) {
#pragma unroll
            for (int r = 0; r < kRuns; ++r)
#pragma unroll
                for (int i = 0; i < 8; ++i) e[r][i] = e[r][i] > -big ? whole(e[r][i]) : 0.0f;
        } else if (!careful) {
#pragma unroll
            for (int r = 0; r < kRuns; ++r)
#pragma unroll
                for (int i = 0; i < 8; ++i) e[r][i] = fast_exp2(fmaf(e[r][i], kLog2e, shift));
        } else {
#pragma unroll
            for (int r = 0; r < kRuns; ++r)
#pragma unroll
                for (int i = 0; i < 8; ++i) e[r][i] = e[r][i] > -big ? fast_exp2(fmaf(e[r][i] - top, kLog2e, 64.0f)) : 0.0f;
        }
#pragma unroll
        for (int r = 0; r < kRuns; ++r)
#pragma unroll
            for (int i = 0; i < 8; ++i) total += e[r][i];
        const float inv = 1.0f / fmaxf(lanes_sum<kLanes>(total), FLT_MIN);
        float p[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float scaled = kExact ? whole(x[h]) : fast_exp2(careful ? fmaf(x[h] - top, kLog2e, 64.0f) : fmaf(x[h], kLog2e, shift));
            p[h] = x[h] > -INFINITY ? scaled * inv : 0.0f;
            d[h] = g[h] * p[h];
        }
        const float all = lanes_sum<kLanes>(d[0] + d[1]);
        base[0] = -p[0] * all;
        base[1] = -p[1] * all;
        float by = -all * inv;
        // (the reciprocal is as small as 2^-74, for 1024 equal logits)
        if (const bool tiny = fabsf(all) < 0x1p-50f; __any_sync(kAll, tiny)) {           // then the factor belongs to it
            by = -(tiny ? all * 0x1p64f : all) * inv;
#pragma unroll
            for (int r = 0; r < kRuns; ++r)
#pragma unroll
                for (int i = 0; i < 8; ++i) e[r][i] *= tiny ? 0x1p-64f : 1.0f;
        }
#pragma unroll
        for (int r = 0; r < kRuns; ++r) {
#pragma unroll
            for (int i = 0; i < 8; ++i) e[r][i] *= by;
            if (mine < a.N) cols.write(out, a.E, r, e[r]);
        }
    } else {
        const float zero[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int r = 0; r < kRuns; ++r)
            if (mine < a.N) cols.write(out, a.E, r, zero);
        float q[2];
        const float most = lanes_max<kLanes>(fmaxf(x[0], x[1]));
#pragma unroll
        for (int h = 0; h < 2; ++h) q[h] = x[h] == -INFINITY ? 0.0f : a.renormalise ? part_of(a.score, x[h], most) : sigmoid(x[h]);
        if (a.renormalise) {
            const float inv = 1.0f / fmaxf(lanes_sum<kLanes>(q[0] + q[1]), FLT_MIN);
            q[0] *= inv; q[1] *= inv;
            const float mean = lanes_sum<kLanes>(g[0] * q[0] + g[1] * q[1]);
#pragma unroll
            for (int h = 0; h < 2; ++h) d[h] = q[h] * (g[h] - mean);
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) d[h] = q[h] * g[h];
        }
        if (a.score == TAOT_SIGMOID) {
#pragma unroll
            for (int h = 0; h < 2; ++h) d[h] *= sigmoid(-x[h]);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (x[h] == -INFINITY) d[h] = 0.0f;
    }
    // an expert that stands in several places: its first place adds them up, in order
    float sum[2] = {d[0], d[1]};
    bool leads[2] = {at[0] >= 0, at[1] >= 0}, twice = a.k > kLanes;
#pragma unroll
    for (int o = 1; o < kLanes; ++o) {
        const int e = __shfl_xor_sync(kAll, at[0], o);
        twice = twice || (e == at[0] && e >= 0);
    }
    if (__any_sync(kAll, twice)) {
        sum[0] = sum[1] = 0.0f;
        for (int j = 0; j < a.k; ++j) {
            const int from = (lane & ~(kLanes - 1)) | (j & (kLanes - 1));
            const int e = __shfl_sync(kAll, j < kLanes ? at[0] : at[1], from);
            const float v = __shfl_sync(kAll, j < kLanes ? d[0] : d[1], from);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (e != at[h]) continue;
                sum[h] += v;
                if (j < cols.sub + kLanes * h) leads[h] = false;
            }
        }
    }
    __syncwarp();                                  // the row is written before its chosen experts
#pragma unroll
    for (int h = 0; h < 2; ++h)
        if (leads[h] && mine < a.N) out[at[h]] = from_f32<T>(base[h] + sum[h]);
}

template <typename T, int kLanes, int kRuns, bool WIDE>
cudaError_t launch_grad(const RouteGradArgs& a, cudaStream_t st)
{
    constexpr int kRows = kWarps * 32 / kLanes;
    const unsigned grid = (unsigned)((a.N + kRows - 1) / kRows);
    if (a.score == TAOT_SOFTMAX && !a.renormalise) route_grad_kernel<T, kLanes, kRuns, WIDE, true><<<grid, kWarps * 32, 0, st>>>(a);
    else route_grad_kernel<T, kLanes, kRuns, WIDE, false><<<grid, kWarps * 32, 0, st>>>(a);
    return cudaGetLastError();
}
template <typename T, bool WIDE>
cudaError_t launch_grad(const RouteGradArgs& a, cudaStream_t st)
{
    if (a.k <= 16 && a.E <= 64) return launch_grad<T, 8, 1, WIDE>(a, st);
    if (a.k <= 16 && a.E <= 128) return launch_grad<T, 8, 2, WIDE>(a, st);
    if (a.k <= 16 && a.E <= 256) return launch_grad<T, 8, 4, WIDE>(a, st);
    return a.E <= 512 ? launch_grad<T, 32, 2, WIDE>(a, st) : launch_grad<T, 32, 4, WIDE>(a, st);
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
    if (a.kept == a.groups) a.groups = a.kept = 1;         // all groups stay
    // chunks of four experts, which with groups may end inside a chunk of each of the eight lanes
    const int32_t chunks = a.groups == 1 || p->E % 32 == 0 ? (p->E + 3) / 4 : p->E / 4 + 12;
    a.chunk_bits = 1;
    while ((1 << a.chunk_bits) <= chunks) ++a.chunk_bits;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool lists = p->k <= 16 && (a.groups == 1 || a.groups == 2 || a.groups == 4 || a.groups == 8);
    if (lists) {
        const bool wide = wide_rows(d_logits, p->ld_logits, e);
        TAOT_CUDA_OK((streams(a, wide) ? launch_stream(a, st) : launch_lanes(a, wide, st)));
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
    const bool wide = p->E % 8 == 0 && wide_rows(d_logits, p->ld_logits, e) && wide_rows(d_dlogits, p->ld_dlogits, e);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (p->dtype == TAOT_F32) TAOT_CUDA_OK((wide ? launch_grad<float, true>(a, st) : launch_grad<float, false>(a, st)));
    else if (p->dtype == TAOT_BF16) TAOT_CUDA_OK((wide ? launch_grad<__nv_bfloat16, true>(a, st) : launch_grad<__nv_bfloat16, false>(a, st)));
    else TAOT_CUDA_OK((wide ? launch_grad<__half, true>(a, st) : launch_grad<__half, false>(a, st)));
    return TAOT_OK;
}

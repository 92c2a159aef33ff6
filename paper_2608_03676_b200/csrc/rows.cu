// Rows to the send buffer of the token all-to-all and back, by the positions that taot_dispatch gives (taot_layer.h).
#include "layer_common.cuh"

namespace {

using namespace layer;

constexpr int kThreads = 256;
constexpr int kMaxK = 64;
constexpr int kMaxCounts = 4096;

struct RowsArgs {
    const int32_t *perm, *counts;
    int32_t* info;
    int64_t n, ld_rows, ld_tokens, ld_residual;
    int32_t k, D, C, wide;
};

// The places of a token's entries in its send buffer, -1 for entries that are not delivered; a CTA per token.
__device__ __forceinline__ void places_of(const RowsArgs& a, int64_t token, int64_t b, int32_t* place, int64_t* sums)
{
    const int tid = threadIdx.x, lane = tid & 31;
    const int64_t cap = a.n * a.k;
    if (a.counts) {
        int64_t s = 0;
        for (int c = tid; c < a.C; c += kThreads) s += a.counts[b * a.C + c];
#pragma unroll
        for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (lane == 0) sums[tid >> 5] = s;
        __syncthreads();
    }
    if (tid < a.k) {
        int64_t valid = cap;
        if (a.counts) {
            int64_t s = 0;
            for (int w = 0; w < kThreads / 32; ++w) s += sums[w];
            valid = s < cap ? s : cap;
        }
        const int32_t at = a.perm[token * a.k + tid];
        const bool inside = at >= 0 && at < cap;
        if (!inside && a.info) atomicOr(a.info + b, TAOT_INFO_BAD_INDEX);
        place[tid] = inside && at < valid ? at : -1;
    }
    __syncthreads();
}

template <typename W>
__global__ void __launch_bounds__(kThreads)
send_kernel(RowsArgs a, const W* x, W* rows, const float* scales, float* row_scales, int32_t scale_cols)
{
    __shared__ int32_t place[kMaxK];
    __shared__ int64_t sums[kThreads / 32];
    const int64_t token = blockIdx.x, b = token / a.n, first = b * a.n * a.k;
    places_of(a, token, b, place, sums);
    for (int c = threadIdx.x; c < a.D; c += kThreads) {
        const W v = x[token * a.ld_tokens + c];
        for (int j = 0; j < a.k; ++j)
            if (place[j] >= 0) rows[(first + place[j]) * a.ld_rows + c] = v;
    }
    for (int c = threadIdx.x; c < scale_cols; c += kThreads) {
        const float v = scales[token * scale_cols + c];
        for (int j = 0; j < a.k; ++j)
            if (place[j] >= 0) row_scales[(first + place[j]) * scale_cols + c] = v;
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
combine_kernel(RowsArgs a, const T* y, const float* weights, const T* residual, T* out)
{
    __shared__ int32_t place[kMaxK];
    __shared__ int64_t sums[kThreads / 32];
    const int64_t token = blockIdx.x, b = token / a.n, first = b * a.n * a.k;
    places_of(a, token, b, place, sums);
    for (int c = threadIdx.x * 8; c < a.D; c += kThreads * 8) {
        float acc[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f}, f[8];
        if (residual) widen(read8(residual + token * a.ld_residual, c, a.D, a.wide), acc);
        for (int j = 0; j < a.k; ++j) {
            if (place[j] < 0) continue;
            const float w = weights ? weights[token * a.k + j] : 1.0f;
            widen(read8(y + (first + place[j]) * a.ld_rows, c, a.D, a.wide), f);
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] = fmaf(w, f[i], acc[i]);
        }
        write8(out + token * a.ld_tokens, c, a.D, a.wide, narrowed<T>(acc));
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads)
combine_grad_kernel(RowsArgs a, const T* dout, const T* y, const float* weights, T* dy, float* dweights)
{
    __shared__ int32_t place[kMaxK];
    __shared__ int64_t sums[kThreads / 32];
    __shared__ float part[kThreads / 32];
    const int64_t token = blockIdx.x, b = token / a.n, first = b * a.n * a.k;
    const int tid = threadIdx.x;
    places_of(a, token, b, place, sums);
    for (int j = 0; j < a.k; ++j) {
        float dot = 0.0f;
        if (place[j] >= 0) {
            const float w = weights ? weights[token * a.k + j] : 1.0f;
            const int64_t at = (first + place[j]) * a.ld_rows;
            for (int c = tid * 8; c < a.D; c += kThreads * 8) {
                float d[8], f[8];
                widen(read8(dout + token * a.ld_tokens, c, a.D, a.wide), d);
                if (dweights) {
                    widen(read8(y + at, c, a.D, a.wide), f);
#pragma unroll
                    for (int i = 0; i < 8; ++i) dot = fmaf(d[i], f[i], dot);
                }
                if (dy) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) d[i] *= w;
                    write8(dy + at, c, a.D, a.wide, narrowed<T>(d));
                }
            }
        }
        if (dweights) {
            dot = warp_sum(dot);
            if ((tid & 31) == 0) part[tid >> 5] = dot;
            __syncthreads();
            if (tid == 0) {
                float s = 0.0f;
                for (int w = 0; w < kThreads / 32; ++w) s += part[w];
                dweights[token * a.k + j] = s;
            }
            __syncthreads();
        }
    }
}

int check(const taot_rows_params* p)
{
    if (!p) return TAOT_ERR_NULL;
    if (p->struct_size != (int32_t)sizeof(taot_rows_params) || p->reserved != 0) return TAOT_ERR_PARAM;
    if (p->B < 0 || p->n < 0 || p->k < 0 || p->D < 1 || p->C < 0) return TAOT_ERR_PARAM;
    const int64_t most = ((int64_t)1 << 31) - 1;
    if (p->k > kMaxK || p->D > kMaxCols || p->C > kMaxCounts || p->B > most || p->n > most || (p->n > 0 && p->B > most / p->n) ||
        (p->n > 0 && p->B > 0 && p->k > most / (p->n * p->B)))
        return TAOT_ERR_UNSUPPORTED;
    return TAOT_OK;
}

RowsArgs args_of(const taot_rows_params* p, const int32_t* perm, const int32_t* counts, int32_t* info)
{
    RowsArgs a;
    a.perm = perm; a.counts = counts; a.info = info;
    a.n = p->n; a.ld_rows = p->ld_rows; a.ld_tokens = p->ld_tokens; a.ld_residual = p->ld_residual;
    a.k = p->k; a.D = p->D; a.C = p->C; a.wide = 0;
    return a;
}

template <typename F>
cudaError_t by_type(int32_t dtype, F&& f)
{
    if (dtype == TAOT_F32) return f(float());
    if (dtype == TAOT_BF16) return f(__nv_bfloat16());
    return f(__half());
}

// whether an output overlaps an input or another output; `allowed`: the one pair (output 0, input 0) that may be the same rows
bool clash(const Range* out, int outs, const Range* in, int ins, bool allowed)
{
    for (int o = 0; o < outs; ++o) {
        for (int i = 0; i < ins; ++i)
            if (overlap(out[o], in[i]) && !(allowed && o == 0 && i == 0 && same(out[o], in[i]))) return true;
        for (int i = 0; i < o; ++i)
            if (overlap(out[o], out[i])) return true;
    }
    return false;
}

}  // namespace

extern "C" int taot_send(const taot_rows_params* p, int32_t elem, const void* d_x, const float* d_scales, int32_t scale_cols,
                         const int32_t* d_perm, const int32_t* d_counts, void* d_rows, float* d_row_scales, int32_t* d_info,
                         void* stream)
{
    if (const int rc = check(p)) return rc;
    if (elem != 1 && elem != 2 && elem != 4) return TAOT_ERR_PARAM;
    if (p->B * p->n * p->k == 0) return TAOT_OK;
    if (!d_x || !d_perm || !d_rows || (p->C > 0 && !d_counts) || ((d_scales != nullptr) != (d_row_scales != nullptr))) return TAOT_ERR_NULL;
    if (d_scales && scale_cols < 1) return TAOT_ERR_PARAM;
    if (d_scales && scale_cols > kMaxCols) return TAOT_ERR_UNSUPPORTED;
    if (!good_ld(p->ld_rows, p->D) || !good_ld(p->ld_tokens, p->D)) return TAOT_ERR_PARAM;
    if (misaligned(d_x, elem) || misaligned(d_rows, elem) || misaligned(d_perm, 4) || misaligned(d_counts, 4) || misaligned(d_scales, 4) ||
        misaligned(d_row_scales, 4) || misaligned(d_info, 4))
        return TAOT_ERR_ALIGN;
    const int64_t tokens = p->B * p->n, entries = tokens * p->k;
    const int32_t* counts = p->C > 0 ? d_counts : nullptr;
    const Range in[] = {range_of(d_x, tokens, p->D, p->ld_tokens, elem), range_of(d_scales, tokens, scale_cols, scale_cols, 4),
                        range_of(d_perm, entries, 1, 1, 4), range_of(counts, p->B, p->C, p->C, 4)};
    const Range out[] = {range_of(d_rows, entries, p->D, p->ld_rows, elem), range_of(d_row_scales, entries, scale_cols, scale_cols, 4),
                         range_of(d_info, p->B, 1, 1, 4)};
    if (clash(out, 3, in, 4, false)) return TAOT_ERR_PARAM;
    RowsArgs a = args_of(p, d_perm, counts, d_info);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int32_t cols = d_scales ? scale_cols : 0;
    const auto launch = [&](auto t) {
        typedef decltype(t) W;
        send_kernel<W><<<(unsigned)tokens, kThreads, 0, st>>>(a, static_cast<const W*>(d_x), static_cast<W*>(d_rows), d_scales, d_row_scales, cols);
        return cudaGetLastError();
    };
    TAOT_CUDA_OK(elem == 1 ? launch(uint8_t()) : elem == 2 ? launch(uint16_t()) : launch(uint32_t()));
    return TAOT_OK;
}

extern "C" int taot_combine(const taot_rows_params* p, const void* d_y, const int32_t* d_perm, const int32_t* d_counts,
                            const float* d_weights, const void* d_residual, void* d_out, int32_t* d_info, void* stream)
{
    if (const int rc = check(p)) return rc;
    if (!known_type(p->dtype)) return TAOT_ERR_PARAM;
    const int64_t tokens = p->B * p->n, entries = tokens * p->k, e = type_bytes(p->dtype);
    if (tokens == 0) return TAOT_OK;
    if ((entries > 0 && (!d_y || !d_perm)) || !d_out || (p->C > 0 && !d_counts)) return TAOT_ERR_NULL;
    if ((entries > 0 && !good_ld(p->ld_rows, p->D)) || !good_ld(p->ld_tokens, p->D) || (d_residual && !good_ld(p->ld_residual, p->D))) return TAOT_ERR_PARAM;
    if (misaligned(d_y, e) || misaligned(d_out, e) || misaligned(d_residual, e) || misaligned(d_perm, 4) || misaligned(d_counts, 4) ||
        misaligned(d_weights, 4) || misaligned(d_info, 4))
        return TAOT_ERR_ALIGN;
    const int32_t* counts = p->C > 0 ? d_counts : nullptr;
    const Range in[] = {range_of(d_residual, tokens, p->D, p->ld_residual, e), range_of(d_y, entries, p->D, p->ld_rows, e),
                        range_of(d_perm, entries, 1, 1, 4), range_of(counts, p->B, p->C, p->C, 4), range_of(d_weights, entries, 1, 1, 4)};
    const Range out[] = {range_of(d_out, tokens, p->D, p->ld_tokens, e), range_of(d_info, p->B, 1, 1, 4)};
    if (clash(out, 2, in, 5, true)) return TAOT_ERR_PARAM;
    RowsArgs a = args_of(p, d_perm, counts, d_info);
    a.wide = wide_rows(d_y, p->ld_rows, e) && wide_rows(d_residual, p->ld_residual, e) && wide_rows(d_out, p->ld_tokens, e);
    TAOT_CUDA_OK(by_type(p->dtype, [&](auto t) {
        typedef decltype(t) T;
        combine_kernel<T><<<(unsigned)tokens, kThreads, 0, static_cast<cudaStream_t>(stream)>>>(
            a, static_cast<const T*>(d_y), d_weights, static_cast<const T*>(d_residual), static_cast<T*>(d_out));
        return cudaGetLastError();
    }));
    return TAOT_OK;
}

extern "C" int taot_combine_backward(const taot_rows_params* p, const void* d_dout, const void* d_y, const int32_t* d_perm,
                                     const int32_t* d_counts, const float* d_weights, void* d_dy, float* d_dweights,
                                     int32_t* d_info, void* stream)
{
    if (const int rc = check(p)) return rc;
    if (!known_type(p->dtype)) return TAOT_ERR_PARAM;
    const int64_t tokens = p->B * p->n, entries = tokens * p->k, e = type_bytes(p->dtype);
    if (entries == 0) return TAOT_OK;
    if (!d_dout || !d_perm || (!d_dy && !d_dweights) || (d_dweights && !d_y) || (p->C > 0 && !d_counts)) return TAOT_ERR_NULL;
    if (!good_ld(p->ld_rows, p->D) || !good_ld(p->ld_tokens, p->D)) return TAOT_ERR_PARAM;
    if (misaligned(d_dout, e) || misaligned(d_y, e) || misaligned(d_dy, e) || misaligned(d_perm, 4) || misaligned(d_counts, 4) ||
        misaligned(d_weights, 4) || misaligned(d_dweights, 4) || misaligned(d_info, 4))
        return TAOT_ERR_ALIGN;
    const int32_t* counts = p->C > 0 ? d_counts : nullptr;
    const Range in[] = {range_of(d_dweights ? d_y : nullptr, entries, p->D, p->ld_rows, e), range_of(d_dout, tokens, p->D, p->ld_tokens, e),
                        range_of(d_perm, entries, 1, 1, 4), range_of(counts, p->B, p->C, p->C, 4), range_of(d_weights, entries, 1, 1, 4)};
    const Range out[] = {range_of(d_dy, entries, p->D, p->ld_rows, e), range_of(d_dweights, entries, 1, 1, 4), range_of(d_info, p->B, 1, 1, 4)};
    if (clash(out, 3, in, 5, true)) return TAOT_ERR_PARAM;
    RowsArgs a = args_of(p, d_perm, counts, d_info);
    a.wide = wide_rows(d_dweights ? d_y : nullptr, p->ld_rows, e) && wide_rows(d_dy, p->ld_rows, e) && wide_rows(d_dout, p->ld_tokens, e);
    TAOT_CUDA_OK(by_type(p->dtype, [&](auto t) {
        typedef decltype(t) T;
        combine_grad_kernel<T><<<(unsigned)tokens, kThreads, 0, static_cast<cudaStream_t>(stream)>>>(
            a, static_cast<const T*>(d_dout), static_cast<const T*>(d_y), d_weights, static_cast<T*>(d_dy), d_dweights);
        return cudaGetLastError();
    }));
    return TAOT_OK;
}

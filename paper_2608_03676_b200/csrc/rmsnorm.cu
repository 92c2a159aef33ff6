// RMS norm with the residual's addition and an output in 8 bits with scales, and its gradients (taot_layer.h).
#include <cmath>

#include <cuda_fp8.h>

#include "layer_common.cuh"

namespace {

using namespace layer;

constexpr int kThreads = 256;
constexpr float kE4m3Max = 448.0f;
constexpr float kLeastScale = 1.17549435e-38f;        // 2^-126: its reciprocal is finite

struct NormArgs {
    const void *x, *residual, *weight;
    void *h, *y;
    uint8_t* q;
    float *scales, *rstd;
    int64_t ld_x, ld_residual, ld_h, ld_y, ld_q;
    int32_t D, group, scale_cols, wide;
    float eps;
};

template <int NW>
__device__ __forceinline__ float block_sum(float v, float* part)
{
    v = warp_sum(v);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < NW; ++w) s += part[w];
    return s;
}

// the 8-bit form of a lane's eight columns; the lanes of a group of columns share its scale
__device__ __forceinline__ void write_eight_bit(const NormArgs& a, int64_t row, int c, const float (&y)[8])
{
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = max_nan(most, fabsf(y[i]));
    const int lanes = a.group >> 3;
    for (int o = 1; o < lanes; o <<= 1) most = max_nan(most, __shfl_xor_sync(0xffffffffu, most, o));
    const float scale = max_nan(most / kE4m3Max, kLeastScale);
    const float inv = 1.0f / scale;
    if (c >= a.D) return;
    if ((c & (a.group - 1)) == 0) a.scales[row * a.scale_cols + c / a.group] = scale;
    union { __nv_fp8_storage_t b[8]; uint2 w; } q;
#pragma unroll
    for (int i = 0; i < 8; ++i) q.b[i] = __nv_cvt_float_to_fp8(y[i] * inv, __NV_SATFINITE, __NV_E4M3);
    uint8_t* to = a.q + row * a.ld_q + c;
    if (a.wide && c + 8 <= a.D) *reinterpret_cast<uint2*>(to) = q.w;
    else
        for (int i = 0; i < 8 && c + i < a.D; ++i) to[i] = q.b[i];
}

// One CTA per row, in two passes: the sum of squares (and h), then y from h.
template <typename T>
__global__ void __launch_bounds__(kThreads)
rms_norm_kernel(NormArgs a)
{
    __shared__ float part[kThreads / 32];
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x;
    const T* x = static_cast<const T*>(a.x) + row * a.ld_x;
    const T* res = a.residual ? static_cast<const T*>(a.residual) + row * a.ld_residual : nullptr;
    T* h = a.h ? static_cast<T*>(a.h) + row * a.ld_h : nullptr;
    T* y = a.y ? static_cast<T*>(a.y) + row * a.ld_y : nullptr;
    const T* w = static_cast<const T*>(a.weight);
    float sum = 0.0f;
    for (int c = tid * 8; c < a.D; c += kThreads * 8) {
        float f[8];
        widen(read8(x, c, a.D, a.wide), f);
        if (res) {
            float g[8];
            widen(read8(res, c, a.D, a.wide), g);
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = rounded<T>(f[i] + g[i]);
            write8(h, c, a.D, a.wide, narrowed<T>(f));
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fmaf(f[i], f[i], sum);
    }
    // (divided by D before the sums of the threads are added: those squares may add up to more than the mean may be)
    const float rstd = 1.0f / sqrtf(block_sum<kThreads / 32>(sum * (1.0f / (float)a.D), part) + a.eps);
    if (tid == 0 && a.rstd) a.rstd[row] = rstd;
    const T* from = res ? h : x;
    const int end = (a.D + 255) / 256 * 256;              // whole warps: the lanes of a group stay together
    for (int c = tid * 8; c < end; c += kThreads * 8) {
        float f[8], g[8];
        widen(read8(from, c, a.D, a.wide), f);
        widen(read8(w, c, a.D, a.wide), g);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = f[i] * rstd * g[i];
        if (a.q) write_eight_bit(a, row, c, f);
        if (y) write8(y, c, a.D, a.wide, narrowed<T>(f));
    }
}

struct NormGradArgs {
    const void *dy, *dh, *h, *weight;
    const float* rstd;
    void* dx;
    float *part, *dweight;
    int64_t ld_dy, ld_dh, ld_h, ld_dx, N;
    int32_t D, wide, parts;
};

// dx: one CTA per row, in two passes
template <typename T>
__global__ void __launch_bounds__(kThreads)
rms_norm_dx_kernel(NormGradArgs a)
{
    __shared__ float part[kThreads / 32];
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x;
    const T* dy = static_cast<const T*>(a.dy) + row * a.ld_dy;
    const T* dh = a.dh ? static_cast<const T*>(a.dh) + row * a.ld_dh : nullptr;
    const T* h = static_cast<const T*>(a.h) + row * a.ld_h;
    T* dx = static_cast<T*>(a.dx) + row * a.ld_dx;
    const T* w = static_cast<const T*>(a.weight);
    const float rstd = a.rstd[row];
    float sum = 0.0f;
    for (int c = tid * 8; c < a.D; c += kThreads * 8) {
        float d[8], x[8], g[8];
        widen(read8(dy, c, a.D, a.wide), d);
        widen(read8(h, c, a.D, a.wide), x);
        widen(read8(w, c, a.D, a.wide), g);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum = fmaf(d[i] * g[i], x[i] * rstd, sum);
    }
    const float mean = block_sum<kThreads / 32>(sum, part) / (float)a.D;
    for (int c = tid * 8; c < a.D; c += kThreads * 8) {
        float d[8], x[8], g[8];
        widen(read8(dy, c, a.D, a.wide), d);
        widen(read8(h, c, a.D, a.wide), x);
        widen(read8(w, c, a.D, a.wide), g);
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] = rstd * (d[i] * g[i] - x[i] * rstd * mean);
        if (dh) {
            widen(read8(dh, c, a.D, a.wide), g);
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] += g[i];
        }
        write8(dx, c, a.D, a.wide, narrowed<T>(d));
    }
}

// dweight: the sums of `parts` spans of rows, one thread per column
template <typename T>
__global__ void __launch_bounds__(kThreads)
rms_norm_dw_kernel(NormGradArgs a)
{
    const int c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= a.D) return;
    const int64_t first = a.N * blockIdx.y / a.parts, last = a.N * (blockIdx.y + 1) / a.parts;
    const T* dy = static_cast<const T*>(a.dy);
    const T* h = static_cast<const T*>(a.h);
    float sum = 0.0f;
    for (int64_t r = first; r < last; ++r)
        sum = fmaf(to_f32(dy[r * a.ld_dy + c]), to_f32(h[r * a.ld_h + c]) * a.rstd[r], sum);
    a.part[(int64_t)blockIdx.y * a.D + c] = sum;
}

__global__ void __launch_bounds__(kThreads)
rms_norm_dw_sum_kernel(NormGradArgs a)
{
    const int c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= a.D) return;
    float sum = 0.0f;
    for (int p = 0; p < a.parts; ++p) sum += a.part[(int64_t)p * a.D + c];
    a.dweight[c] = sum;
}

constexpr int kParts = 128;

template <typename F>
cudaError_t by_type(int32_t dtype, F&& f)
{
    if (dtype == TAOT_F32) return f(float());
    if (dtype == TAOT_BF16) return f(__nv_bfloat16());
    return f(__half());
}

int check(const taot_norm_params* p)
{
    if (!p) return TAOT_ERR_NULL;
    if (p->struct_size != (int32_t)sizeof(taot_norm_params) || !known_type(p->dtype) || p->reserved != 0) return TAOT_ERR_PARAM;
    if (p->N < 0 || p->D < 1) return TAOT_ERR_PARAM;
    if (p->N >= ((int64_t)1 << 31) || p->D > kMaxCols) return TAOT_ERR_UNSUPPORTED;
    return TAOT_OK;
}

}  // namespace

extern "C" int taot_rms_norm(const taot_norm_params* p, const void* d_x, const void* d_residual, const void* d_weight,
                             void* d_h, void* d_y, uint8_t* d_q, float* d_scales, float* d_rstd, void* stream)
{
    if (const int rc = check(p)) return rc;
    if (!(p->eps >= 0.0f) || !std::isfinite(p->eps)) return TAOT_ERR_PARAM;
    if (p->group != 0 && p->group != 32 && p->group != 64 && p->group != 128 && p->group != 256) return TAOT_ERR_PARAM;
    if (p->N == 0) return TAOT_OK;                         // (arrays of no rows have no address)
    if ((d_q != nullptr) != (p->group != 0)) return TAOT_ERR_PARAM;
    if (!d_x || !d_weight || (!d_y && !d_q) || (d_q && !d_scales) || (d_residual && !d_h)) return TAOT_ERR_NULL;
    if ((!d_residual && d_h) || (!d_q && d_scales)) return TAOT_ERR_PARAM;
    const int64_t N = p->N, D = p->D, e = type_bytes(p->dtype), cols = d_q ? (D + p->group - 1) / p->group : 0;
    if (!good_ld(p->ld_x, D) || (d_residual && (!good_ld(p->ld_residual, D) || !good_ld(p->ld_h, D))) ||
        (d_y && !good_ld(p->ld_y, D)) || (d_q && !good_ld(p->ld_q, D)))
        return TAOT_ERR_PARAM;
    if (misaligned(d_x, e) || misaligned(d_residual, e) || misaligned(d_weight, e) || misaligned(d_h, e) || misaligned(d_y, e) ||
        misaligned(d_scales, 4) || misaligned(d_rstd, 4))
        return TAOT_ERR_ALIGN;
    const Range in[] = {range_of(d_x, N, D, p->ld_x, e), range_of(d_residual, N, D, p->ld_residual, e), range_of(d_weight, 1, D, D, e)};
    const Range out[] = {range_of(d_h, N, D, p->ld_h, e), range_of(d_y, N, D, p->ld_y, e), range_of(d_q, N, D, p->ld_q, 1),
                         range_of(d_scales, N, cols, cols, 4), range_of(d_rstd, N, 1, 1, 4)};
    for (int o = 0; o < 5; ++o) {
        for (int i = 0; i < 3; ++i)
            if (overlap(out[o], in[i]) && !(((o == 0 && i < 2) || (o == 1 && i == 0)) && same(out[o], in[i]))) return TAOT_ERR_PARAM;
        for (int i = 0; i < o; ++i)
            if (overlap(out[o], out[i])) return TAOT_ERR_PARAM;
    }
    NormArgs a;
    a.x = d_x; a.residual = d_residual; a.weight = d_weight; a.h = d_h; a.y = d_y; a.q = d_q; a.scales = d_scales; a.rstd = d_rstd;
    a.ld_x = p->ld_x; a.ld_residual = p->ld_residual; a.ld_h = p->ld_h; a.ld_y = p->ld_y; a.ld_q = p->ld_q;
    a.D = p->D; a.group = p->group; a.scale_cols = (int32_t)cols; a.eps = p->eps;
    a.wide = wide_rows(d_x, p->ld_x, e) && wide_rows(d_residual, p->ld_residual, e) && wide_rows(d_weight, 0, e) &&
             wide_rows(d_h, p->ld_h, e) && wide_rows(d_y, p->ld_y, e) && !misaligned(d_q, 8) && (!d_q || p->ld_q % 8 == 0);
    TAOT_CUDA_OK(by_type(p->dtype, [&](auto t) {
        rms_norm_kernel<decltype(t)><<<(unsigned)N, kThreads, 0, static_cast<cudaStream_t>(stream)>>>(a);
        return cudaGetLastError();
    }));
    return TAOT_OK;
}

extern "C" int taot_rms_norm_backward_workspace(const taot_norm_params* p, size_t* bytes)
{
    if (!bytes) return TAOT_ERR_NULL;
    if (const int rc = check(p)) return rc;
    *bytes = sizeof(float) * (size_t)kParts * p->D;
    return TAOT_OK;
}

extern "C" int taot_rms_norm_backward(const taot_norm_params* p, const void* d_dy, const void* d_dh, const void* d_h,
                                      const void* d_weight, const float* d_rstd, void* d_dx, float* d_dweight, void* ws,
                                      void* stream)
{
    if (const int rc = check(p)) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (misaligned(d_dweight, 4) || misaligned(ws, 16)) return TAOT_ERR_ALIGN;
    const int64_t N = p->N, D = p->D, e = type_bytes(p->dtype);
    if (N == 0) {
        if (d_dweight) TAOT_CUDA_OK(cudaMemsetAsync(d_dweight, 0, sizeof(float) * (size_t)D, st));
        return TAOT_OK;
    }
    if (!d_dy || !d_h || !d_weight || !d_rstd || !d_dx || (d_dweight && !ws)) return TAOT_ERR_NULL;
    if (!good_ld(p->ld_y, D) || !good_ld(p->ld_h, D) || !good_ld(p->ld_x, D) || (d_dh && !good_ld(p->ld_residual, D))) return TAOT_ERR_PARAM;
    if (misaligned(d_dy, e) || misaligned(d_dh, e) || misaligned(d_h, e) || misaligned(d_weight, e) || misaligned(d_dx, e) || misaligned(d_rstd, 4))
        return TAOT_ERR_ALIGN;
    const Range in[] = {range_of(d_dy, N, D, p->ld_y, e), range_of(d_dh, N, D, p->ld_residual, e), range_of(d_h, N, D, p->ld_h, e),
                        range_of(d_weight, 1, D, D, e), range_of(d_rstd, N, 1, 1, 4)};
    const Range out[] = {range_of(d_dx, N, D, p->ld_x, e), range_of(d_dweight, 1, D, D, 4),
                         range_of(d_dweight ? ws : nullptr, kParts, D, D, 4)};
    for (int o = 0; o < 3; ++o) {
        for (int i = 0; i < 5; ++i)
            if (overlap(out[o], in[i]) && !(o == 0 && i < 2 && same(out[o], in[i]))) return TAOT_ERR_PARAM;
        for (int i = 0; i < o; ++i)
            if (overlap(out[o], out[i])) return TAOT_ERR_PARAM;
    }
    NormGradArgs a;
    a.dy = d_dy; a.dh = d_dh; a.h = d_h; a.weight = d_weight; a.rstd = d_rstd; a.dx = d_dx;
    a.part = static_cast<float*>(ws); a.dweight = d_dweight;
    a.ld_dy = p->ld_y; a.ld_dh = p->ld_residual; a.ld_h = p->ld_h; a.ld_dx = p->ld_x; a.N = N; a.D = p->D;
    a.parts = kParts;
    a.wide = wide_rows(d_dy, p->ld_y, e) && wide_rows(d_dh, p->ld_residual, e) && wide_rows(d_h, p->ld_h, e) &&
             wide_rows(d_weight, 0, e) && wide_rows(d_dx, p->ld_x, e);
    const unsigned cols = (unsigned)((D + kThreads - 1) / kThreads);
    TAOT_CUDA_OK(by_type(p->dtype, [&](auto t) {
        if (d_dweight) {                                   // before dx, which may take the place of dy
            rms_norm_dw_kernel<decltype(t)><<<dim3(cols, kParts), kThreads, 0, st>>>(a);
            rms_norm_dw_sum_kernel<<<cols, kThreads, 0, st>>>(a);
        }
        rms_norm_dx_kernel<decltype(t)><<<(unsigned)N, kThreads, 0, st>>>(a);
        return cudaGetLastError();
    }));
    return TAOT_OK;
}

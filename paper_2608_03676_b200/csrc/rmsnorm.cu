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
    int64_t N;
    int32_t D, group, group_shift, scale_cols, wide;
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

// two products (and sums) in an instruction, each rounded as by itself
__device__ __forceinline__ uint64_t two(float a, float b)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void apart(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t times(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t times_plus(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
// eight columns times rstd, times their weights
__device__ __forceinline__ void normalise(float (&f)[8], float rstd, const float (&w)[8])
{
    const uint64_t r = two(rstd, rstd);
#pragma unroll
    for (int i = 0; i < 8; i += 2) apart(times(times(two(f[i], f[i + 1]), r), two(w[i], w[i + 1])), f[i], f[i + 1]);
}

// The scale of columns whose largest magnitude is `most`, a product (its last bit matters to nobody, as long as the columns are divided
// by the scale as it is written), and the columns divided by it.  The 8-bit values are those of the fp32
// quotients to the bit: quotients in the middle of two 8-bit values are frequent (16-bit inputs, weights of one), and a product
// with the reciprocal takes the other one there (8192 x 4096 bf16: 56.8 us with the product, 58.9 with the quotient).
//   a / b: with b's reciprocal in two parts (`by` rounded to nearest, and what it lacks, `low`) the product q = a by + a low is
//   within an ulp, and Markstein's step (1990), q + (a - q b) by, whose remainder is exact, is the quotient rounded to nearest, as
//   long as no remainder comes below 2^-149: a scale below 2^-70 and its columns are taken times 2^100.  There is no branch: an infinite
//   scale has the reciprocal 0 (0 for finite columns, a NaN for infinite ones), a NaN spreads.
struct Scale {
    float value, up, b, by, low;                   // b = value * up
    __device__ __forceinline__ explicit Scale(float most)
    {
        value = max_nan(most * (1.0f / kE4m3Max), kLeastScale);
        up = value < 0x1p-70f ? 0x1p100f : 1.0f;
        b = value * up;
        // the approximation is within an ulp; a step of Newton's method rounds it to nearest, except where all bits of the mantissa are
        // set (Markstein): there the nearest one's last bit is set too
        asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(by) : "f"(b));
        by = fmaf(by, fmaf(-by, b, 1.0f), by);
        if ((__float_as_uint(b) & 0x7fffffu) == 0x7fffffu) by = __uint_as_float(__float_as_uint(by) | 1u);
        low = fmaf(-by, b, 1.0f) * by;
        if (value == INFINITY) { b = 1.0f; by = low = 0.0f; }
    }
    __device__ __forceinline__ float divide(float f) const
    {
        const float a = f * up, q = fmaf(a, by, a * low);
        return copysignf(fmaf(fmaf(-q, b, a), by, q), f);          // (zeros have signs)
    }
    template <int n>
    __device__ __forceinline__ void divide(const float* f, float (&out)[n]) const      // the same, two at a time
    {
        static_assert(n % 2 == 0, "two at a time");
        const uint64_t ups = two(up, up), minus = two(-b, -b), bys = two(by, by), lows = two(low, low);
#pragma unroll
        for (int i = 0; i < n; i += 2) {
            const uint64_t a = times(two(f[i], f[i + 1]), ups), q = times_plus(a, bys, times(a, lows));
            apart(times_plus(times_plus(q, minus, a), bys, q), out[i], out[i + 1]);
            out[i] = copysignf(out[i], f[i]);
            out[i + 1] = copysignf(out[i + 1], f[i + 1]);
        }
    }
};
// four columns in e4m3
__device__ __forceinline__ uint32_t four_bytes(float a, float b, float c, float d)
{
    return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3) |
           (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3) << 16;
}
// 1 / sqrt(v), a root and a division rounded to nearest: 8-bit rows hold many quotients in the middle of two values, which an rstd that is
// an ulp off sends the other way (8192 x 4096 bf16: 316 values differ from those of elementwise fp32 operations, 1010 with the
// approximate root and a step of Newton's method, which takes as long)
__device__ __forceinline__ float inverse_root(float v) { return 1.0f / sqrtf(v); }

// the 8-bit form of a lane's eight columns; the lanes of a group of columns share its scale
__device__ __forceinline__ void write_eight_bit(const NormArgs& a, int64_t row, int c, const float (&y)[8])
{
    float most = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) most = max_nan(most, fabsf(y[i]));
    if (c >= a.D) most = 0.0f;
#pragma unroll
    for (int o = 1; o < 32; o *= 2)
        if (o < 4 || a.group > 8 * o) most = max_nan(most, __shfl_xor_sync(0xffffffffu, most, o));
    if (c >= a.D) return;
    const Scale scale(most);
    if ((c & (a.group - 1)) == 0) a.scales[row * a.scale_cols + (c >> a.group_shift)] = scale.value;
    float v[8];
    scale.divide(y, v);
    union { uint8_t b[8]; uint2 w; } q;
    q.w.x = four_bytes(v[0], v[1], v[2], v[3]);
    q.w.y = four_bytes(v[4], v[5], v[6], v[7]);
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
    const float inv = 1.0f / (float)a.D;
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
        float eight = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) eight = fmaf(f[i], f[i], eight);
        sum = fmaf(eight, inv, sum);               // (divided by D eight at a time: more of them may add up to more than the mean may be)
    }
    const float rstd = inverse_root(block_sum<kThreads / 32>(sum, part) + a.eps);
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

// the sum of n warps' values (n a power of two up to 16), by each warp
template <int n>
__device__ __forceinline__ float sum_of_warps(const float* part)
{
    float v = part[threadIdx.x & (n - 1)];
#pragma unroll
    for (int o = n / 2; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Rows of up to 8192 columns: `kLanes` threads hold a row, `kRuns` runs of eight columns each, from the addition to the 8-bit form.
// Registers are bounded so that more rows are on their way: 16-bit rows to 48 or 40 (8192 x 4096 bf16: 59 us, 64 without a bound), rows
// read one by one to 64 (4439 x 4733 bf16: 104 us, 139 without; fp32: the same with and without); wide fp32 rows, which
// memory bounds either way, are not.
template <typename T, int kLanes, int kRuns, bool WIDE>
__global__ void __launch_bounds__(kLanes > kThreads ? kLanes : kThreads, !WIDE ? (kLanes > kThreads ? 2 : 4) : sizeof(T) == 2 && kLanes <= kThreads ? (kRuns == 1 ? 6 : 5) : 1)
rms_norm_row_kernel(const __grid_constant__ NormArgs a)
{
    constexpr int kCta = kLanes > kThreads ? kLanes : kThreads;
    constexpr int kWarpsOfRow = kLanes / 32;
    __shared__ float part[kCta / 32];
    const int tid = threadIdx.x, lane = tid & 31, slot = tid / kLanes, start = (tid % kLanes >> 5) * 256;
    const int64_t row = (int64_t)blockIdx.x * (kCta / kLanes) + slot;
    const bool there = row < a.N;
    // (pieces of 16 bytes are within the row or beyond it as a whole)
    constexpr int kPiece = WIDE ? 16 / (int)sizeof(T) : 1;
    const auto live = [&](int r, int i) { return column<WIDE, T>(start + r * kLanes * 8, lane, i / kPiece * kPiece) < a.D; };
    Run8<T> h[kRuns], w[kRuns];
    float sum = 0.0f;
    if (there) {
        const T* x = static_cast<const T*>(a.x) + row * a.ld_x;
#pragma unroll
        for (int r = 0; r < kRuns; ++r) h[r] = load8<WIDE>(x, start + r * kLanes * 8, lane, a.D);
        if (a.residual) {
            const T* res = static_cast<const T*>(a.residual) + row * a.ld_residual;
            Run8<T> e[kRuns];
#pragma unroll
            for (int r = 0; r < kRuns; ++r) e[r] = load8<WIDE>(res, start + r * kLanes * 8, lane, a.D);
#pragma unroll
            for (int r = 0; r < kRuns; ++r) {
                float f[8], g[8];
                widen(h[r], f);
                widen(e[r], g);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] += g[i];
                h[r] = narrowed<T>(f);
                store8<WIDE>(static_cast<T*>(a.h) + row * a.ld_h, start + r * kLanes * 8, lane, a.D, h[r]);
            }
        }
#pragma unroll
        for (int r = 0; r < kRuns; ++r) {
            w[r] = load8<WIDE>(static_cast<const T*>(a.weight), start + r * kLanes * 8, lane, a.D);
            float f[8];
            widen(h[r], f);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (live(r, i)) sum = fmaf(f[i], f[i], sum);
        }
    }
    // (divided by D before the sums of the threads are added: those squares may add up to more than the mean may be)
    sum = warp_sum(sum * (1.0f / (float)a.D));
    if (kWarpsOfRow > 1) {
        if (lane == 0) part[tid >> 5] = sum;
        __syncthreads();
        sum = sum_of_warps<kWarpsOfRow>(part + slot * kWarpsOfRow);
    }
    if (!there) return;                            // (whole warps)
    const float rstd = inverse_root(sum + a.eps);
    if (a.rstd && tid % kLanes == 0) a.rstd[row] = rstd;
#pragma unroll
    for (int r = 0; r < kRuns; ++r) {
        const int c0 = start + r * kLanes * 8;
        float f[8], g[8];
        widen(h[r], f);
        widen(w[r], g);
        normalise(f, rstd, g);                     // (what is beyond D is not written)
        if (a.y) store8<WIDE>(static_cast<T*>(a.y) + row * a.ld_y, c0, lane, a.D, narrowed<T>(f));
        if (!a.q || c0 >= a.D) continue;           // (the same for a warp)
        if (WIDE && sizeof(T) == 2) {
            write_eight_bit(a, row, c0 + 8 * lane, f);
        } else if (WIDE) {
            // columns 4 lane to 4 lane + 3 of either half of the warp's 256
            float most[2];
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                most[q] = max_nan(max_nan(fabsf(f[4 * q]), fabsf(f[4 * q + 1])), max_nan(fabsf(f[4 * q + 2]), fabsf(f[4 * q + 3])));
                if (!live(r, 4 * q)) most[q] = 0.0f;
            }
            if (a.group == 256) most[0] = most[1] = max_nan(most[0], most[1]);
            for (int o = 1; o < min(a.group >> 2, 32); o <<= 1) {
                most[0] = max_nan(most[0], __shfl_xor_sync(0xffffffffu, most[0], o));
                most[1] = max_nan(most[1], __shfl_xor_sync(0xffffffffu, most[1], o));
            }
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int c = column<WIDE, T>(c0, lane, 4 * q);
                if (c >= a.D) continue;
                const Scale scale(most[q]);
                if ((c & (a.group - 1)) == 0) a.scales[row * a.scale_cols + (c >> a.group_shift)] = scale.value;
                float v[4];
                scale.divide(f + 4 * q, v);
                const uint32_t word = four_bytes(v[0], v[1], v[2], v[3]);
                *reinterpret_cast<uint32_t*>(a.q + row * a.ld_q + c) = word;
            }
        } else {
            // column 32 i + lane of the warp's 256: a group is 1, 2, 4 or 8 of the i
            float most[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) most[i] = live(r, i) ? fabsf(f[i]) : 0.0f;
            const int n = a.group >> 5;
#pragma unroll
            for (int o = 1; o < 8; o *= 2)
                if (o < n) {
                    float other[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) other[i] = most[i ^ o];
#pragma unroll
                    for (int i = 0; i < 8; ++i) most[i] = max_nan(most[i], other[i]);
                }
            Scale scale(0.0f);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int c = c0 + 32 * i + lane;
                if ((i & (n - 1)) == 0) {          // the first of a group (the same for a warp)
                    float m = most[i];
#pragma unroll
                    for (int o = 16; o; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
                    scale = Scale(m);
                    if (lane == 0 && c < a.D) a.scales[row * a.scale_cols + (c >> a.group_shift)] = scale.value;
                }
                if (c < a.D) a.q[row * a.ld_q + c] = __nv_cvt_float_to_fp8(scale.divide(f[i]), __NV_SATFINITE, __NV_E4M3);
            }
        }
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

// dx and the sums for dweight in one pass over the rows: `kLanes` threads hold a row, `kRuns` runs of eight columns each, and keep the
// weights and the sums of their columns in registers for all rows that they take, one after another.  The rows to come are
// on their way to shared memory meanwhile, kStages of them (each thread copies, waits for and reads its own columns: no
// barrier is needed for that); rows that cannot be copied 16 bytes at a time are read when they are due.  A CTA's sums go to the
// workspace (rms_norm_dw_join_kernel).
constexpr int kSms = 148;
constexpr int kSpans = 128;                        // of rows, where a CTA cannot hold a row
// the most CTAs whose sums a call leaves in the workspace
int32_t most_parts(int32_t D) { return D <= 2048 ? 4 * kSms : D <= 16384 ? 2 * kSms : kSpans; }

template <typename T, int kLanes, int kRuns>
struct GradShape {
    static constexpr int kCta = kLanes > kThreads ? kLanes : kThreads;
    static constexpr int kRows = kCta / kLanes;    // at a time
    static constexpr int kPieces = kRuns * (int)sizeof(Run8<T>) / 16;        // 16-byte pieces of a thread, row and array
    // 1024 runs per SM, whose rows to come take 196 KB: four of 16 bits, two of fp32
    static constexpr int kStages = sizeof(T) == 2 ? (kRuns == 4 ? 2 : 4) : 2;
    static constexpr int kCtasPerSm = kRuns == 4 ? 1 : 1024 / (kCta * kRuns);
    static constexpr size_t kRing = (size_t)kStages * 3 * kPieces * 16 * kCta;
    static constexpr size_t kSums = sizeof(float) * kCta * 8 * kRuns;
};

__device__ __forceinline__ void copy_async(uint32_t to, const void* from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copy_async_word(uint32_t to, const void* from)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_queued() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int n>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(n) : "memory"); }

template <typename T, int kLanes, int kRuns, bool WIDE>
__global__ void __launch_bounds__(GradShape<T, kLanes, kRuns>::kCta, WIDE ? GradShape<T, kLanes, kRuns>::kCtasPerSm : kLanes > kThreads ? 1 : 2)
rms_norm_grad_kernel(const __grid_constant__ NormGradArgs a)
{
    typedef GradShape<T, kLanes, kRuns> S;
    constexpr bool kAsync = WIDE || sizeof(T) == 4;
    constexpr int kStages = kAsync ? S::kStages : 1;
    constexpr int kWarpsOfRow = kLanes / 32;
    extern __shared__ __align__(16) uint4 ring[];  // [stage][array][piece][thread]
    __shared__ float part[2][S::kCta / 32];
    const int tid = threadIdx.x, lane = tid & 31;
    const int slot = tid / kLanes, start = (tid % kLanes >> 5) * 256;       // first column of the warp's runs, which are kLanes * 8 apart
    const auto live = [&](int r, int i) { return column<WIDE, T>(start + r * kLanes * 8, lane, i) < a.D; };
    taot_release();                                // (the next kernel's CTAs come as these end)
    Run8<T> w[kRuns];
    float dw[kRuns][8];
#pragma unroll
    for (int r = 0; r < kRuns; ++r) {
        w[r] = load8<WIDE>(static_cast<const T*>(a.weight), start + r * kLanes * 8, lane, a.D);
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[r][i] = 0.0f;
    }
    const auto array = [&](int which, int64_t row) {
        return which == 0 ? static_cast<const T*>(a.dy) + row * a.ld_dy : which == 1 ? static_cast<const T*>(a.h) + row * a.ld_h : static_cast<const T*>(a.dh) + row * a.ld_dh;
    };
    const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring) + (WIDE ? 16u : 4u) * (uint32_t)tid;
    float rstd[kStages];
    const auto queue = [&](int stage, int64_t row) {               // (an empty group where there is no such row)
        if (row < a.N) {
            rstd[stage] = a.rstd[row];
#pragma unroll
            for (int which = 0; which < 3; ++which) {
                if (which == 2 && !a.dh) break;
                const T* from = array(which, row);
#pragma unroll
                for (int r = 0; r < kRuns; ++r)
                    if (!WIDE) {
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (live(r, i))
                                copy_async_word(ring_at + 4u * (uint32_t)((((stage * 3 + which) * kRuns + r) * 8 + i) * S::kCta), from + column<WIDE, T>(start + r * kLanes * 8, lane, i));
                    } else {
#pragma unroll
                        for (int q = 0; q < S::kPieces / kRuns; ++q) {
                            const int c = column<WIDE, T>(start + r * kLanes * 8, lane, q * (8 / (S::kPieces / kRuns)));
                            if (c < a.D) copy_async(ring_at + 16u * (uint32_t)(((stage * 3 + which) * S::kPieces + r * (S::kPieces / kRuns) + q) * S::kCta), from + c);
                        }
                    }
            }
        }
        copies_queued();
    };
    const auto take = [&](int stage, int which, int r, int64_t row) {
        if constexpr (WIDE) {
            Run8<T> v;
            uint4* to = reinterpret_cast<uint4*>(&v);
#pragma unroll
            for (int q = 0; q < S::kPieces / kRuns; ++q) to[q] = ring[((stage * 3 + which) * S::kPieces + r * (S::kPieces / kRuns) + q) * S::kCta + tid];
            return v;
        } else if constexpr (kAsync) {
            Run8<T> v;
#pragma unroll
            for (int i = 0; i < 8; ++i) v.v[i] = reinterpret_cast<const T*>(ring)[(((stage * 3 + which) * kRuns + r) * 8 + i) * S::kCta + tid];
            return v;
        } else {
            return load8<false>(array(which, row), start + r * kLanes * 8, lane, a.D);
        }
    };
    const int64_t step = (int64_t)gridDim.x * S::kRows;
    int64_t first = (int64_t)blockIdx.x * S::kRows, row = first + slot;
    const float inv = 1.0f / (float)a.D;
    if (kAsync)
#pragma unroll
        for (int s = 0; s < kStages; ++s) queue(s, row + s * step);
    int turn = 0;
    while (first < a.N) {
#pragma unroll
        for (int s = 0; s < kStages; ++s) {
            if (first >= a.N) break;                               // (the same for all threads of the CTA)
            const bool there = row < a.N;
            if (kAsync) copies_wait<kStages - 1>();
            else if (there) rstd[0] = a.rstd[row];
            float sum = 0.0f;
            Run8<T> dy[kRuns], h[kRuns];
            if (there)
#pragma unroll
                for (int r = 0; r < kRuns; ++r) {
                    dy[r] = take(s, 0, r, row);
                    h[r] = take(s, 1, r, row);
                }
            if (there)
#pragma unroll
                for (int r = 0; r < kRuns; ++r) {
                    float d[8], x[8], f[8];
                    widen(dy[r], d);
                    widen(h[r], x);
                    widen(w[r], f);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        if (!live(r, i)) continue;
                        const float t = x[i] * rstd[s];
                        dw[r][i] = fmaf(d[i], t, dw[r][i]);
                        sum = fmaf(d[i] * f[i], t, sum);
                    }
                }
            sum = warp_sum(sum);
            if (kWarpsOfRow > 1) {
                if (lane == 0) part[turn][tid >> 5] = sum;
                __syncthreads();
                sum = sum_of_warps<kWarpsOfRow>(part[turn] + slot * kWarpsOfRow);
            }
            if (there) {
                const float shift = rstd[s] * (sum * inv);
#pragma unroll
                for (int r = 0; r < kRuns; ++r) {
                    float d[8], x[8], f[8];
                    widen(dy[r], d);
                    widen(h[r], x);
                    widen(w[r], f);
#pragma unroll
                    for (int i = 0; i < 8; ++i) d[i] = rstd[s] * (d[i] * f[i] - x[i] * shift);
                    if (a.dh) {
                        widen(take(s, 2, r, row), f);
#pragma unroll
                        for (int i = 0; i < 8; ++i) d[i] += f[i];
                    }
                    store8<WIDE>(static_cast<T*>(a.dx) + row * a.ld_dx, start + r * kLanes * 8, lane, a.D, narrowed<T>(d));
                }
            }
            if (kAsync) queue(s, row + kStages * step);
            turn ^= 1;
            first += step;
            row += step;
        }
    }
    if (!a.dweight) return;
    if (kAsync) copies_wait<0>();
    __syncthreads();
    // the rows that a CTA takes at a time have their own sums
    float* const sums = reinterpret_cast<float*>(ring);
    constexpr int kCols = kLanes * 8 * kRuns;
#pragma unroll
    for (int r = 0; r < kRuns; ++r)
#pragma unroll
        for (int i = 0; i < 8; ++i) sums[slot * kCols + column<WIDE, T>(start + r * kLanes * 8, lane, i)] = dw[r][i];
    __syncthreads();
    for (int c = tid; c < a.D; c += S::kCta) {
        float s = 0.0f;
#pragma unroll
        for (int q = 0; q < S::kRows; ++q) s += sums[q * kCols + c];
        a.part[(int64_t)blockIdx.x * a.D + c] = s;
    }
}

// Adds up the CTAs' sums: a CTA takes 32 columns, a warp every 32nd of the CTAs.
constexpr int kJoinThreads = 1024;
__global__ void __launch_bounds__(kJoinThreads)
rms_norm_dw_join_kernel(NormGradArgs a)
{
    __shared__ float part[kJoinThreads / 32][33];
    taot_await();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * 32 + lane;
    float s = 0.0f;
    if (c < a.D)
#pragma unroll 10
        for (int p = warp; p < a.parts; p += kJoinThreads / 32) s += a.part[(int64_t)p * a.D + c];
    part[warp][lane] = s;
    __syncthreads();
    s = warp_sum(part[lane][warp]);                // column `warp` of the CTA's
    const int mine = blockIdx.x * 32 + warp;
    if (lane == 0 && mine < a.D) a.dweight[mine] = s;
}

template <typename F>
cudaError_t by_type(int32_t dtype, F&& f)
{
    if (dtype == TAOT_F32) return f(float());
    if (dtype == TAOT_BF16) return f(__nv_bfloat16());
    return f(__half());
}

template <typename T, bool WIDE, int kLanes, int kRuns>
cudaError_t fused_as(NormGradArgs& a, cudaStream_t st)
{
    typedef GradShape<T, kLanes, kRuns> S;
    constexpr size_t ring = WIDE || sizeof(T) == 4 ? S::kRing : 0, most_smem = ring > S::kSums ? ring : S::kSums;
    const size_t sums = a.dweight ? S::kSums : 0, smem = ring > sums ? ring : sums;
    const int64_t ctas = (a.N + S::kRows - 1) / S::kRows, most = kSms * (WIDE ? S::kCtasPerSm : S::kCta > kThreads ? 1 : 2);
    a.parts = (int32_t)(ctas < most ? ctas : most);
    const auto kernel = rms_norm_grad_kernel<T, kLanes, kRuns, WIDE>;
    cudaError_t e = allow_shared(kernel, most_smem);
    if (e != cudaSuccess) return e;
    kernel<<<(unsigned)a.parts, S::kCta, smem, st>>>(a);
    e = cudaGetLastError();
    if (e != cudaSuccess || !a.dweight) return e;
    return taot_launch_chained(rms_norm_dw_join_kernel, (unsigned)((a.D + 31) / 32), (unsigned)kJoinThreads, 0, st, a);
}

// 16-bit rows: two runs of columns per thread (8192 rows of 4096: 56 us with one, 50 with two), fp32 rows and those that cannot be
// copied 16 bytes at a time one; more where a CTA could not hold the row.
template <typename T, bool WIDE>
cudaError_t fused(NormGradArgs& a, cudaStream_t st)
{
    if (a.D <= 256) return fused_as<T, WIDE, 32, 1>(a, st);
    if constexpr (sizeof(T) == 2 && WIDE) {
        if (a.D <= 512) return fused_as<T, WIDE, 32, 2>(a, st);
        if (a.D <= 1024) return fused_as<T, WIDE, 64, 2>(a, st);
        if (a.D <= 2048) return fused_as<T, WIDE, 128, 2>(a, st);
        if (a.D <= 4096) return fused_as<T, WIDE, 256, 2>(a, st);
        if (a.D > 8192) return fused_as<T, WIDE, 512, 4>(a, st);
    } else {
        if (a.D <= 512) return fused_as<T, WIDE, 64, 1>(a, st);
        if (a.D <= 1024) return fused_as<T, WIDE, 128, 1>(a, st);
        if (a.D <= 2048) return fused_as<T, WIDE, 256, 1>(a, st);
        if (a.D <= 4096) return fused_as<T, WIDE, 512, 1>(a, st);
    }
    return fused_as<T, WIDE, 512, 2>(a, st);
}

template <typename T, bool WIDE, int kLanes, int kRuns>
cudaError_t by_row_as(const NormArgs& a, cudaStream_t st)
{
    constexpr int kCta = kLanes > kThreads ? kLanes : kThreads, kRows = kCta / kLanes;
    rms_norm_row_kernel<T, kLanes, kRuns, WIDE><<<(unsigned)((a.N + kRows - 1) / kRows), kCta, 0, st>>>(a);
    return cudaGetLastError();
}
template <typename T, bool WIDE>
cudaError_t by_row(const NormArgs& a, cudaStream_t st)
{
    if (a.D <= 256) return by_row_as<T, WIDE, 32, 1>(a, st);
    if constexpr (WIDE) {
        if (a.D <= 512) return by_row_as<T, WIDE, 32, 2>(a, st);
        if (a.D <= 1024) return by_row_as<T, WIDE, 64, 2>(a, st);
        if (a.D <= 2048) return by_row_as<T, WIDE, 128, 2>(a, st);
        if (a.D <= 4096) return by_row_as<T, WIDE, 256, 2>(a, st);
    } else {
        if (a.D <= 512) return by_row_as<T, WIDE, 64, 1>(a, st);
        if (a.D <= 1024) return by_row_as<T, WIDE, 128, 1>(a, st);
        if (a.D <= 2048) return by_row_as<T, WIDE, 256, 1>(a, st);
        if (a.D <= 4096) return by_row_as<T, WIDE, 512, 1>(a, st);
    }
    return by_row_as<T, WIDE, 512, 2>(a, st);
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
    a.group_shift = p->group == 32 ? 5 : p->group == 64 ? 6 : p->group == 128 ? 7 : 8;
    a.N = N; a.D = p->D; a.group = p->group; a.scale_cols = (int32_t)cols; a.eps = p->eps;
    a.wide = wide_rows(d_x, p->ld_x, e) && wide_rows(d_residual, p->ld_residual, e) && wide_rows(d_weight, 0, e) &&
             wide_rows(d_h, p->ld_h, e) && wide_rows(d_y, p->ld_y, e) && !misaligned(d_q, 8) && (!d_q || p->ld_q % 8 == 0);
    if (D <= 8192) {                                       // beyond, two passes are faster (2048 x 16384 bf16: 72 us against 89)
        a.wide = a.wide && D % 8 == 0;
        TAOT_CUDA_OK(by_type(p->dtype, [&](auto t) {
            return a.wide ? by_row<decltype(t), true>(a, static_cast<cudaStream_t>(stream)) : by_row<decltype(t), false>(a, static_cast<cudaStream_t>(stream));
        }));
        return TAOT_OK;
    }
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
    *bytes = sizeof(float) * (size_t)most_parts(p->D) * p->D;
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
                         range_of(d_dweight ? ws : nullptr, most_parts(p->D), D, D, 4)};
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
    a.parts = 0;
    a.wide = wide_rows(d_dy, p->ld_y, e) && wide_rows(d_dh, p->ld_residual, e) && wide_rows(d_h, p->ld_h, e) &&
             wide_rows(d_weight, 0, e) && wide_rows(d_dx, p->ld_x, e);
    const unsigned cols = (unsigned)((D + kThreads - 1) / kThreads);
    const bool wide = a.wide && D % 8 == 0;
    if (D <= 8192 || (D <= 16384 && wide && e == 2)) {     // rows that the threads of a CTA can hold
        a.wide = wide;
        TAOT_CUDA_OK(by_type(p->dtype, [&](auto t) { return a.wide ? fused<decltype(t), true>(a, st) : fused<decltype(t), false>(a, st); }));
        return TAOT_OK;
    }
    a.parts = kSpans;
    TAOT_CUDA_OK(by_type(p->dtype, [&](auto t) {
        if (d_dweight) {                                   // before dx, which may take the place of dy
            rms_norm_dw_kernel<decltype(t)><<<dim3(cols, (unsigned)a.parts), kThreads, 0, st>>>(a);
            rms_norm_dw_sum_kernel<<<cols, kThreads, 0, st>>>(a);
        }
        rms_norm_dx_kernel<decltype(t)><<<(unsigned)N, kThreads, 0, st>>>(a);
        return cudaGetLastError();
    }));
    return TAOT_OK;
}

// What the layer's operators (rmsnorm.cu, route.cu, rows.cu) share: element types, runs of eight elements, argument checks.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "taot_internal.cuh"
#include "taot_layer.h"

namespace layer {

constexpr int64_t kMaxLd = (int64_t)1 << 28;      // elements between rows: no byte offset comes near 2^63
constexpr int32_t kMaxCols = 1 << 20;

static inline bool known_type(int32_t t) { return t == TAOT_F32 || t == TAOT_BF16 || t == TAOT_F16; }
static inline int64_t type_bytes(int32_t t) { return t == TAOT_F32 ? 4 : 2; }
static inline bool good_ld(int64_t ld, int64_t cols) { return ld >= cols && ld <= kMaxLd; }
static inline bool misaligned(const void* p, int64_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)) != 0; }

// An array of a call: rows of `cols` elements of `elem` bytes, `ld` elements apart
struct Range {
    uintptr_t at;
    int64_t bytes, ld, pitch, row;                // from the first element to the last; in bytes: from row to row, of a row
};
static inline Range range_of(const void* p, int64_t rows, int64_t cols, int64_t ld, int64_t elem)
{
    return {reinterpret_cast<uintptr_t>(p), p && rows > 0 && cols > 0 ? ((rows - 1) * ld + cols) * elem : 0, ld, ld * elem, cols * elem};
}
static inline bool overlap(const Range& a, const Range& b)
{
    if (a.bytes == 0 || b.bytes == 0 || a.at >= b.at + (uintptr_t)b.bytes || b.at >= a.at + (uintptr_t)a.bytes) return false;
    if (a.pitch != b.pitch) return true;
    // rows equally far apart: different columns of one wider array do not meet
    const uintptr_t pitch = (uintptr_t)a.pitch, off = b.at >= a.at ? (b.at - a.at) % pitch : (pitch - (a.at - b.at) % pitch) % pitch;
    return off < (uintptr_t)a.row || off + (uintptr_t)b.row > pitch;
}
// the same rows at the same place: every element is read before it is written, by the thread that writes it
static inline bool same(const Range& a, const Range& b) { return a.at == b.at && a.ld == b.ld && a.bytes == b.bytes; }

// whether rows of this array can be read or written 16 bytes at a time from their start
static inline bool wide_rows(const void* p, int64_t ld, int64_t elem)
{
    return !p || (!misaligned(p, 16) && ld * elem % 16 == 0);
}

// Lets a kernel have up to `most` bytes of dynamic shared memory.  The limit belongs to the kernel, in all of the context: a call that
// set its own could lower it between another host thread's setting and launch.  So `most` is the most that any call's launch of
// the kernel takes, whatever the call at hand needs.
constexpr size_t kWithoutLimit = 46 * 1024;        // 48 KB less what these kernels declare
template <typename K>
cudaError_t allow_shared(K kernel, size_t most)
{
    return most <= kWithoutLimit ? cudaSuccess : cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most);
}

#ifdef __CUDACC__
__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <typename T> __device__ __forceinline__ float rounded(float v) { return to_f32(from_f32<T>(v)); }

// eight consecutive elements as they stand in memory
template <typename T>
struct alignas(16) Run8 {
    T v[8];
};

template <typename T>
__device__ __forceinline__ void widen(const Run8<T>& r, float (&f)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = to_f32(r.v[i]);
}
// (two at a time: one conversion instruction for both)
__device__ __forceinline__ uint32_t narrowed_pair(float a, float b, __nv_bfloat16)
{
    const __nv_bfloat162 r = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t narrowed_pair(float a, float b, __half)
{
    const __half2 r = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&r);
}
template <typename T>
__device__ __forceinline__ Run8<T> narrowed(const float (&f)[8])
{
    Run8<T> r;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < 4; ++i) reinterpret_cast<uint32_t*>(&r)[i] = narrowed_pair(f[2 * i], f[2 * i + 1], T());
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) r.v[i] = f[i];
    }
    return r;
}

// Reads and writes of up to eight elements from column c of a row of D: 16 bytes at a time where the array allows it (wide),
// one by one at the end of a row and elsewhere.  Columns from D on read as zero and are not written.
template <typename T>
__device__ __forceinline__ Run8<T> read8(const T* row, int c, int D, bool wide)
{
    Run8<T> r;
    if (wide && c + 8 <= D) {
        const uint4* p = reinterpret_cast<const uint4*>(row + c);
        uint4* q = reinterpret_cast<uint4*>(&r);
#pragma unroll
        for (int i = 0; i < (int)sizeof(Run8<T>) / 16; ++i) q[i] = p[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) r.v[i] = c + i < D ? row[c + i] : from_f32<T>(0.0f);
    }
    return r;
}
template <typename T>
__device__ __forceinline__ void write8(T* row, int c, int D, bool wide, const Run8<T>& r)
{
    if (wide && c + 8 <= D) {
        uint4* p = reinterpret_cast<uint4*>(row + c);
        const uint4* q = reinterpret_cast<const uint4*>(&r);
#pragma unroll
        for (int i = 0; i < (int)sizeof(Run8<T>) / 16; ++i) p[i] = q[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (c + i < D) row[c + i] = r.v[i];
    }
}

// A warp's 256 columns from c0 on, eight per lane: WIDE (rows of a multiple of eight columns that can be read 16 bytes at a time) in
// pieces of 16 bytes, those of a load next to each other; otherwise one by one, 32 apart.  The column of a lane's element i:
template <bool WIDE, typename T>
__device__ __forceinline__ int column(int c0, int lane, int i)
{
    if (!WIDE) return c0 + 32 * i + lane;
    return sizeof(T) == 2 ? c0 + 8 * lane + i : c0 + 128 * (i >> 2) + 4 * lane + (i & 3);
}
// What is beyond D is read from the last columns instead, without a branch, and not written.
template <bool WIDE, typename T>
__device__ __forceinline__ Run8<T> load8(const T* row, int c0, int lane, int D)
{
    constexpr int kPiece = 16 / (int)sizeof(T);
    Run8<T> r;
    if constexpr (WIDE) {
        uint4* q = reinterpret_cast<uint4*>(&r);
#pragma unroll
        for (int i = 0; i < 8; i += kPiece) q[i / kPiece] = *reinterpret_cast<const uint4*>(row + min(column<WIDE, T>(c0, lane, i), D - kPiece));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) r.v[i] = row[min(column<WIDE, T>(c0, lane, i), D - 1)];
    }
    return r;
}
template <bool WIDE, typename T>
__device__ __forceinline__ void store8(T* row, int c0, int lane, int D, const Run8<T>& r)
{
    constexpr int kPiece = 16 / (int)sizeof(T);
    if constexpr (WIDE) {
        const uint4* q = reinterpret_cast<const uint4*>(&r);
#pragma unroll
        for (int i = 0; i < 8; i += kPiece) {
            const int c = column<WIDE, T>(c0, lane, i);
            if (c < D) *reinterpret_cast<uint4*>(row + c) = q[i / kPiece];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int c = column<WIDE, T>(c0, lane, i);
            if (c < D) row[c] = r.v[i];
        }
    }
}

__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// the larger of two, a NaN if one is a NaN
__device__ __forceinline__ float max_nan(float a, float b)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
#endif

}  // namespace layer

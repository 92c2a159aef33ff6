// Routing with a lane per row: calls of many rows by their logits alone (route_common.cuh: how the choice is made).
//
// A warp brings 32 rows to shared memory, with a pitch of an odd number of 16-byte pieces, so that the lanes read their rows without
// bank conflicts.  With a row to itself a lane needs no shuffles, and no two lanes make the same comparison: 64 warp instructions
// per row of 128 bf16 logits, against 157 with eight lanes (counted).
#include "route_common.cuh"

namespace route {

namespace {

constexpr int K = 8;

__device__ __forceinline__ void copy_async(void* to, const void* from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}

// two 16-bit numbers in a word
template <typename T> struct Pair;
template <> struct Pair<__nv_bfloat16> {
    static constexpr uint32_t lowest = 0xff7fff7fu, big = 0x7f7f7f7fu;
    static __device__ __forceinline__ uint32_t most(uint32_t a, uint32_t b)     // (a NaN only if both are)
    {
        uint32_t r;
        asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    static __device__ __forceinline__ uint32_t least(uint32_t a, uint32_t b)
    {
        uint32_t r;
        asm("min.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    static __device__ __forceinline__ uint32_t plus_zero(uint32_t a)
    {
        const __nv_bfloat162 r = __hadd2_rn(*reinterpret_cast<const __nv_bfloat162*>(&a), __nv_bfloat162(__float2bfloat16_rn(0.0f), __float2bfloat16_rn(0.0f)));
        return *reinterpret_cast<const uint32_t*>(&r);
    }
    static __device__ __forceinline__ float number(uint32_t bits) { return __uint_as_float(bits << 16); }
};
template <> struct Pair<__half> {
    static constexpr uint32_t lowest = 0xfbfffbffu, big = 0x7bff7bffu;
    static __device__ __forceinline__ uint32_t most(uint32_t a, uint32_t b)
    {
        uint32_t r;
        asm("max.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    static __device__ __forceinline__ uint32_t least(uint32_t a, uint32_t b)
    {
        uint32_t r;
        asm("min.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    static __device__ __forceinline__ uint32_t plus_zero(uint32_t a)
    {
        const __half2 r = __hadd2_rn(*reinterpret_cast<const __half2*>(&a), __half2(__float2half_rn(0.0f), __float2half_rn(0.0f)));
        return *reinterpret_cast<const uint32_t*>(&r);
    }
    static __device__ __forceinline__ float number(uint32_t bits) { return __half2float(__ushort_as_half((unsigned short)bits)); }
};

// The order-preserving images of two 16-bit logits: a NaN and what is closed as the lowest value, an infinity as the largest, one zero.
template <typename T>
__device__ __forceinline__ uint32_t ordered_pair(uint32_t m)
{
    m = Pair<T>::plus_zero(Pair<T>::least(Pair<T>::most(m, Pair<T>::lowest), Pair<T>::big));
    const uint32_t negative = (m >> 15) & 0x00010001u;
    return m ^ (negative * 0x7fffu) ^ 0x80008000u;
}
template <typename T>
__device__ __forceinline__ float pair_number(uint32_t key)         // of the upper half
{
    const uint32_t u = key >> 16;
    return Pair<T>::number(u & 0x8000u ? u ^ 0x8000u : ~u & 0xffffu);
}

// What a lane has chosen: experts (-1 where there is none) and their logits (-infinity), largest first
struct Chosen {
    int at[K];
    float x[K];
};

// 16-bit logits: keys lose nothing
template <typename T>
__device__ __forceinline__ void choose(const RouteArgs& a, const uint4* row, Chosen& r)
{
    constexpr uint32_t kLow = 0xffffu, kShut = Pair<T>::lowest & 0xffffu ^ 0xffffu;    // the image of the lowest value
    const int C = a.E / 4;
    uint32_t best[K], list[K], none = 0;
    for (int c0 = 0; c0 < C; c0 += K) {
#pragma unroll
        for (int u = 0; u < K; u += 2) {
            const int c = c0 + u;
            if (c < C) {
                const uint4 v = row[c / 2];
                const uint32_t p = Pair<T>::most(v.x, v.y), q = Pair<T>::most(v.z, v.w);
                const uint32_t m = ordered_pair<T>(Pair<T>::most(__byte_perm(p, q, 0x5410), __byte_perm(p, q, 0x7632)));
                list[u] = (m << 16) + (kLow - (uint32_t)c);
                list[u + 1] = (m & 0xffff0000u) + (kLow - (uint32_t)c - 1u);
            } else {
                list[u] = list[u + 1] = 0;
            }
        }
        sort_list(list);
        if (c0 == 0) {
#pragma unroll
            for (int i = 0; i < K; ++i) best[i] = list[i];
        } else {
            merge_list<false>(best, list, none);
        }
    }
    uint32_t first[K];
#pragma unroll
    for (int i = 0; i < K; i += 2) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int c = (int)(kLow - (best[i + h] & kLow));
            uint2 v = make_uint2(Pair<T>::lowest, Pair<T>::lowest);
            if (c < C) v = reinterpret_cast<const uint2*>(row)[c];
            const uint32_t e = kLow - 4u * (uint32_t)c, m = ordered_pair<T>(v.x), n = ordered_pair<T>(v.y);
            list[4 * h] = (m << 16) + (e & kLow);
            list[4 * h + 1] = (m & 0xffff0000u) + ((e - 1u) & kLow);
            list[4 * h + 2] = (n << 16) + ((e - 2u) & kLow);
            list[4 * h + 3] = (n & 0xffff0000u) + ((e - 3u) & kLow);
        }
        sort_list(list);
        if (i == 0) {
#pragma unroll
            for (int q = 0; q < K; ++q) first[q] = list[q];
        } else {
            merge_list<false>(first, list, none);
        }
    }
#pragma unroll
    for (int i = 0; i < K; ++i) {
        const bool there = i < a.k && first[i] >> 16 > kShut;
        r.at[i] = there ? (int)(kLow - (first[i] & kLow)) : -1;
        r.x[i] = there ? pair_number<T>(first[i]) : -INFINITY;
    }
}

// fp32 logits.  Returns whether the choice is settled; `least`: a lower bound of the last one's logit where it is not.
__device__ __forceinline__ bool choose(const RouteArgs& a, const uint4* row, Chosen& r, float& least)
{
    constexpr float big = Type<float>::big;
    constexpr uint32_t kSlots = 4 * K - 1;
    const int C = a.E / 4;
    const uint32_t cmask = (1u << a.chunk_bits) - 1, drop = max(cmask, kSlots);
    uint32_t best[K], list[K], lost = 0, bits = 0;
    for (int c0 = 0; c0 < C; c0 += K) {
#pragma unroll
        for (int u = 0; u < K; ++u) {
            const int c = c0 + u;
            list[u] = 0;
            if (c < C) {
                const uint4 v = row[c];
                bits |= v.x | v.y | v.z | v.w;
                const float m = fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
                list[u] = (ordered(fminf(fmaxf(m, -big), big) + 0.0f) & ~cmask) | (cmask - (uint32_t)c);
            }
        }
        sort_list(list);
        if (c0 == 0) {
#pragma unroll
            for (int i = 0; i < K; ++i) best[i] = list[i];
        } else {
            merge_list<true>(best, list, lost);
        }
    }
    uint32_t ids[K], first[K];                     // chunks in ascending order (none: cmask, behind all others)
#pragma unroll
    for (int i = 0; i < K; ++i) ids[i] = ~(cmask - (best[i] & cmask));
    sort_list(ids);
#pragma unroll
    for (int i = 0; i < K; i += 2) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int c = (int)~ids[i + h];
            float x[4] = {-big, -big, -big, -big};
            if (c < C) four(reinterpret_cast<const float*>(row) + 4 * c, x);
#pragma unroll
            for (int q = 0; q < 4; ++q) list[4 * h + q] = (ordered(fminf(fmaxf(x[q], -big), big) + 0.0f) & ~kSlots) | (kSlots - (uint32_t)(4 * (i + h) + q));
        }
        sort_list(list);
        if (i == 0) {
#pragma unroll
            for (int q = 0; q < K; ++q) first[q] = list[q];
        } else {
            merge_list<true>(first, list, lost);
        }
    }
    // the chunks' numbers as bytes of two words (up to 256 chunks: 8 bits; none is never asked for)
    uint32_t lo = 0, hi = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        lo |= (~ids[i] & 0xffu) << (8 * i);
        hi |= (~ids[i + 4] & 0xffu) << (8 * i);
    }
    uint32_t beyond = lost, last = 0;
#pragma unroll
    for (int i = 0; i < K; ++i) {
        const uint32_t slot = kSlots - (first[i] & kSlots);
        const int e = 4 * (int)(__byte_perm(lo, hi, slot >> 2) & 0xffu) + (int)(slot & 3);
        r.x[i] = -INFINITY;
        r.at[i] = -1;
        if (i < a.k) last = first[i];
        else beyond = max(beyond, first[i]);
        if (i < a.k && e < a.E) {
            const float x = seen(reinterpret_cast<const float*>(row)[e], big);
            if (x > -INFINITY) { r.at[i] = e; r.x[i] = x; }
        }
    }
    // neighbours that the lost bits have turned round; more than that is left to settle_choice
    bool settled = (bits & drop) == 0 || ((beyond ^ last) & ~drop) != 0;
    least = number_of(last & ~drop);
#pragma unroll
    for (int i = 0; i + 1 < K; ++i)
        if (r.x[i + 1] > r.x[i]) {
            const float x = r.x[i];
            const int e = r.at[i];
            r.x[i] = r.x[i + 1]; r.at[i] = r.at[i + 1];
            r.x[i + 1] = x; r.at[i + 1] = e;
        }
#pragma unroll
    for (int i = 0; i + 1 < K; ++i)
        if (r.x[i + 1] > r.x[i] || (r.x[i + 1] == r.x[i] && r.at[i + 1] >= 0 && r.at[i + 1] < r.at[i])) settled = false;
    return settled;
}

template <typename T>
__global__ void __launch_bounds__(32)
route_stream_kernel(const __grid_constant__ RouteArgs a, int32_t pitch, int32_t quads)
{
    extern __shared__ uint4 tile[];
    constexpr float big = Type<T>::big;
    const int lane = threadIdx.x;
    const int64_t first = (int64_t)blockIdx.x * 32, row = first + lane;
    const int pieces = a.E * (int)sizeof(T) / 16, rows = (int)min((int64_t)32, a.N - first);
    {
        const int lanes = pieces > 16 ? 32 : pieces > 8 ? 16 : 8;  // that copy a row
        const char* from = reinterpret_cast<const char*>(static_cast<const T*>(a.logits) + (first + lane / lanes) * a.ld) + 16 * (lane & (lanes - 1));
        uint4* to = tile + lane / lanes * pitch + (lane & (lanes - 1));
        const int64_t step = a.ld * (int64_t)sizeof(T) * (32 / lanes);
        for (int r = lane / lanes; r < rows; r += 32 / lanes, from += step, to += 32 / lanes * pitch)
            for (int c = lane & (lanes - 1), o = 0; c < pieces; c += lanes, o += lanes) copy_async(to + o, from + 16 * o);
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    const bool mine = row < a.N, routed = mine && (!a.mask || a.mask[row]);
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncwarp();
    const uint4* own = tile + (mine ? lane : 0) * pitch;           // (lanes past the end repeat the first row and write nothing)
    Chosen r;
    bool settled = true;
    float least = 0.0f;
    if constexpr (sizeof(T) == 2) choose<T>(a, own, r);
    else settled = choose(a, own, r, least);

    float total = 1.0f, w[K];
    if (a.weights) {
        const bool direct = a.score == TAOT_SOFTMAX && !a.renormalise;
        if (direct) {                                              // the sum of the row's exponentials
            float part[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            for (int c = 0; c < a.E / 4; ++c) {
                float x[4];
                four(reinterpret_cast<const T*>(own) + 4 * c, x);
#pragma unroll
                for (int q = 0; q < 4; ++q) part[q] += x[q] > -big ? fast_exp2((fminf(x[q], big) - r.x[0]) * kLog2e) : 0.0f;
            }
            total = (part[0] + part[1]) + (part[2] + part[3]);
        }
        const bool relative = a.score == TAOT_SOFTMAX || a.renormalise;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < K; ++i) {
            w[i] = 0.0f;
            if (i >= a.k) continue;
            if (r.at[i] >= 0) w[i] = relative ? part_of(a.score, r.x[i], r.x[0]) : sigmoid(r.x[i]);
            sum += w[i];
        }
        if (direct) sum = total;
        const float by = direct || a.renormalise ? (sum > 0.0f ? a.scale / sum : 0.0f) : a.scale;
#pragma unroll
        for (int i = 0; i < K; ++i) w[i] *= by;
    }
    if (!routed)
#pragma unroll
        for (int i = 0; i < K; ++i) { r.at[i] = -1; w[i] = 0.0f; }
    if (mine && (settled || !routed)) {
        int32_t* to = a.topk + row * a.k;
        float* wo = a.weights + row * a.k;
        if (quads) {                                               // k is 4 or 8, 16 bytes at a time
#pragma unroll
            for (int i = 0; i < K; i += 4)
                if (i < a.k) {
                    reinterpret_cast<int4*>(to)[i / 4] = make_int4(r.at[i], r.at[i + 1], r.at[i + 2], r.at[i + 3]);
                    if (a.weights) reinterpret_cast<float4*>(wo)[i / 4] = make_float4(w[i], w[i + 1], w[i + 2], w[i + 3]);
                }
        } else {
#pragma unroll
            for (int i = 0; i < K; ++i)
                if (i < a.k) {
                    to[i] = r.at[i];
                    if (a.weights) wo[i] = w[i];
                }
        }
    }
    if constexpr (sizeof(T) == 4) {
        unsigned left = __ballot_sync(kAll, routed && !settled);
        while (left) {
            const int from = __ffs(left) - 1;
            left &= left - 1;
            __syncwarp();                                          // the tile is done with
            int at0 = -1, at1 = -1;
            float t = __shfl_sync(kAll, r.x[0], from), z = __shfl_sync(kAll, total, from);
            const float limit = __shfl_sync(kAll, least, from);
            int32_t* const found = reinterpret_cast<int32_t*>(tile);
            if (settle_choice(a, first + from, Scores{t, 1.0f}, 1u, limit, found)) at0 = lane < a.k ? found[lane] : -1;
            else choose_exactly(a, first + from, reinterpret_cast<uint64_t*>(tile), at0, at1, t, z);
            write_row(a, first + from, at0, at1, t, z);
        }
    }
}

template <typename T>
cudaError_t launch(const RouteArgs& a, cudaStream_t st)
{
    const int32_t pieces = a.E * (int32_t)sizeof(T) / 16, pitch = pieces | 1;
    const size_t smem = (size_t)32 * pitch * 16;                   // (rows of up to 512 bytes: 17 KB)
    const int32_t quads = a.k % 4 == 0 && !misaligned(a.topk, 16) && !misaligned(a.weights, 16);
    route_stream_kernel<T><<<(unsigned)((a.N + 31) / 32), 32, smem, st>>>(a, pitch, quads);
    return cudaGetLastError();
}

}  // namespace

// Against eight lanes per row, us:   rows of 256 B (128 bf16, 64 fp32)  32768: 6.1 : 8.0, 8.5 : 12.4    2^20: 81 : 198
//                                     512 B (256 bf16, 128 fp32)        16384: 7.5 : 5.7, 10.2 : 8.7    65536: 17.9 : 17.6, 19.4 : 24.3
//                                                                       262144: 46 : 63, 50 : 84
//                                     1 KB (512 bf16, 256 fp32)         131072: 56 : 46,  262144: 104 : 104
// With long rows too few warps fit in shared memory, with few rows there are too few warps.
bool streams(const RouteArgs& a, bool wide)
{
    const int64_t bytes = (int64_t)a.E * layer::type_bytes(a.dtype);
    return wide && !a.bias && a.groups == 1 && a.k <= K && bytes % 16 == 0 && bytes <= 512 && a.N >= 128 * bytes;
}

cudaError_t launch_stream(const RouteArgs& a, cudaStream_t st)
{
    if (a.dtype == TAOT_F32) return launch<float>(a, st);
    if (a.dtype == TAOT_BF16) return launch<__nv_bfloat16>(a, st);
    return launch<__half>(a, st);
}

}  // namespace route

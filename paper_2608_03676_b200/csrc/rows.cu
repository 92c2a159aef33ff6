// Rows to the send buffer of the token all-to-all and back, by the positions that taot_dispatch gives (taot_layer.h).
#include "layer_common.cuh"

namespace {

using namespace layer;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxK = 64;
constexpr int kMaxCounts = 4096;
constexpr unsigned kAll = 0xffffffffu;

struct RowsArgs {
    const int32_t *perm, *counts;
    const float* weights;
    int32_t* info;
    int64_t ld_rows, ld_tokens, ld_residual;
    uint32_t tokens, n, cap;      // of all buffers; of one; positions of one buffer
    int32_t k, D, C, wide;
    int32_t share;                // log2 of the warps that share a token (at most kWarps)
};

// What a warp works on: a token, or its part of one.
struct Part {
    uint32_t token;               // tokens: none is left
    int32_t start, step;          // its runs of columns: start + lane, then `step` further on
    int64_t first;                // the first row of its buffer
    int32_t entries;              // that are delivered, in the order of j: lane i has the i-th (0) and the (32 + i)-th (1)
    int32_t place0, place1;       // where they stand in the buffer
    float w0, w1;                 // their weights (1 without weights)
    int32_t j0, j1;               // which of the token's entries they are
    bool out0, out1;              // whether entries lane and lane + 32 of the token exist and are not delivered
};
__device__ __forceinline__ Part part_of(const RowsArgs& a)
{
    Part p;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    p.token = (uint32_t)(((uint64_t)blockIdx.x * kWarps + warp) >> a.share);
    p.start = (int32_t)(warp & ((1u << a.share) - 1)) * 32;
    p.step = 32 << a.share;
    p.first = 0;
    p.entries = 0;
    p.out0 = p.out1 = false;
    if (p.token >= a.tokens) {
        p.token = a.tokens;
        return p;
    }
    // all reads first
    const int64_t entry = (int64_t)p.token * a.k + lane;
    int32_t at0 = 0, at1 = 0;
    float w0 = 1.0f, w1 = 1.0f;
    if (lane < a.k) {
        at0 = a.perm[entry];
        if (a.weights) w0 = a.weights[entry];
    }
    if (lane + 32 < a.k) {
        at1 = a.perm[entry + 32];
        if (a.weights) w1 = a.weights[entry + 32];
    }
    const uint32_t b = p.token / a.n;
    p.first = (int64_t)b * a.cap;
    uint32_t limit = a.cap;
    if (a.counts) {
        int64_t s = 0;
        for (int c = lane; c < a.C; c += 32) s += a.counts[(int64_t)b * a.C + c];
#pragma unroll
        for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(kAll, s, o);
        limit = s < 0 ? 0u : s < (int64_t)a.cap ? (uint32_t)s : a.cap;
    }
    const bool in0 = lane >= a.k || (uint32_t)at0 < a.cap, in1 = lane + 32 >= a.k || (uint32_t)at1 < a.cap;
    if (!(in0 && in1) && a.info && p.start == 0) atomicOr(a.info + b, TAOT_INFO_BAD_INDEX);
    // those that are delivered move to the front
    const bool d0 = lane < a.k && in0 && (uint32_t)at0 < limit, d1 = lane + 32 < a.k && in1 && (uint32_t)at1 < limit;
    const unsigned m0 = __ballot_sync(kAll, d0), m1 = __ballot_sync(kAll, d1);
    const int n0 = __popc(m0);
    p.entries = n0 + __popc(m1);
    p.out0 = lane < a.k && !d0;
    p.out1 = lane + 32 < a.k && !d1;
    const auto front = [&](int i, int32_t& place, float& w, int32_t& j) {
        j = i < n0 ? __fns(m0, 0, i + 1) : i < p.entries ? 32 + __fns(m1, 0, i - n0 + 1) : 0;
        const int32_t s0 = __shfl_sync(kAll, at0, j & 31), s1 = __shfl_sync(kAll, at1, j & 31);
        const float v0 = __shfl_sync(kAll, w0, j & 31), v1 = __shfl_sync(kAll, w1, j & 31);
        place = j < 32 ? s0 : s1;
        w = j < 32 ? v0 : v1;
    };
    if (p.entries == a.k) {                                        // all of them
        p.place0 = at0; p.place1 = at1; p.w0 = w0; p.w1 = w1; p.j0 = lane; p.j1 = lane + 32;
    } else {
        front(lane, p.place0, p.w0, p.j0);
        front(lane + 32, p.place1, p.w1, p.j1);
    }
    return p;
}
__device__ __forceinline__ int32_t place_of(const Part& p, int i) { return __shfl_sync(kAll, i < 32 ? p.place0 : p.place1, i & 31); }
__device__ __forceinline__ float weight_of(const Part& p, int i) { return __shfl_sync(kAll, i < 32 ? p.w0 : p.w1, i & 31); }

// Rows of W, the widest words that all rows are made of: a lane holds four of the token's words and writes them to all its places.
template <typename W>
__global__ void __launch_bounds__(kThreads)
send_kernel(RowsArgs a, const W* x, W* rows, const float* scales, float* row_scales, int32_t scale_cols)
{
    const Part p = part_of(a);
    if (p.token >= a.tokens) return;
    const int lane = threadIdx.x & 31;
    const W* from = x + p.token * a.ld_tokens;
    for (int c0 = p.start; c0 < a.D; c0 += 4 * p.step) {
        const int c = c0 + lane;
        W v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c + i * p.step < a.D) v[i] = from[c + i * p.step];
        for (int j = 0; j < p.entries; ++j) {
            W* to = rows + (p.first + place_of(p, j)) * a.ld_rows + c;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (c + i * p.step < a.D) to[i * p.step] = v[i];
        }
    }
    for (int c0 = p.start; c0 < scale_cols; c0 += p.step) {
        const int c = c0 + lane;
        const float v = c < scale_cols ? scales[(int64_t)p.token * scale_cols + c] : 0.0f;
        for (int j = 0; j < p.entries; ++j) {
            const int64_t at = (p.first + place_of(p, j)) * scale_cols + c;
            if (c < scale_cols) row_scales[at] = v;
        }
    }
}

// adds n of a token's rows from entry i on to a run of eight columns; all are read before the first is used
template <int n, bool WIDE, typename T>
__device__ __forceinline__ void add_rows(const RowsArgs& a, const Part& p, const T* y, int i, int c0, float (&acc)[8])
{
    const int lane = threadIdx.x & 31;
    Run8<T> row[n];
#pragma unroll
    for (int u = 0; u < n; ++u) row[u] = load8<WIDE>(y + (p.first + place_of(p, i + u)) * a.ld_rows, c0, lane, a.D);
#pragma unroll
    for (int u = 0; u < n; ++u) {
        const float w = weight_of(p, i + u);
        float f[8];
        widen(row[u], f);
#pragma unroll
        for (int q = 0; q < 8; ++q) acc[q] = fmaf(w, f[q], acc[q]);
    }
}

template <typename T, bool WIDE>
__global__ void __launch_bounds__(kThreads)
combine_kernel(RowsArgs a, const T* y, const T* residual, T* out)
{
    const Part p = part_of(a);
    if (p.token >= a.tokens) return;
    const int lane = threadIdx.x & 31;
    for (int c0 = 8 * p.start; c0 < a.D; c0 += 8 * p.step) {
        float acc[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
        if (residual) widen(load8<WIDE>(residual + p.token * a.ld_residual, c0, lane, a.D), acc);
        int i = 0;
        for (; i + 8 <= p.entries; i += 8) add_rows<8, WIDE>(a, p, y, i, c0, acc);
        if (i + 4 <= p.entries) { add_rows<4, WIDE>(a, p, y, i, c0, acc); i += 4; }
        if (i + 2 <= p.entries) { add_rows<2, WIDE>(a, p, y, i, c0, acc); i += 2; }
        if (i < p.entries) add_rows<1, WIDE>(a, p, y, i, c0, acc);
        store8<WIDE>(out + p.token * a.ld_tokens, c0, lane, a.D, narrowed<T>(acc));
    }
}

// The sums of eight values over a warp: nine shuffles; lane 4 i has value i.
__device__ __forceinline__ float sum_of_eight(float (&v)[8])
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int o = 16, n = 4; n >= 1; o >>= 1, n >>= 1)
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const bool upper = lane & o;
            const float keep = upper ? v[i + n] : v[i], send = upper ? v[i] : v[i + n];
            v[i] = keep + __shfl_xor_sync(kAll, send, o);
        }
    v[0] += __shfl_xor_sync(kAll, v[0], 2);
    v[0] += __shfl_xor_sync(kAll, v[0], 1);
    return v[0];
}

// The gradients of n of a token's rows, from entry i on: a run of dout is read once for them, their rows are read for the products
// (all before the first is used) and written.
template <int n, bool WIDE, typename T>
__device__ __forceinline__ void grad_rows(const RowsArgs& a, const Part& p, const T* dout, const T* y, T* dy, float* dweights, int i, float (&part)[kWarps][8])
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    float dot[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f}, w[n];
    int64_t at[n];
#pragma unroll
    for (int u = 0; u < n; ++u) {
        at[u] = (p.first + place_of(p, i + u)) * a.ld_rows;
        w[u] = weight_of(p, i + u);
    }
    for (int c0 = 8 * p.start; c0 < a.D; c0 += 8 * p.step) {
        float d[8];
        Run8<T> row[n];
        const Run8<T> grad = load8<WIDE>(dout + p.token * a.ld_tokens, c0, lane, a.D);
        if (dweights)
#pragma unroll
            for (int u = 0; u < n; ++u) row[u] = load8<WIDE>(y + at[u], c0, lane, a.D);
        widen(grad, d);
        if (dweights) {
#pragma unroll
            for (int u = 0; u < n; ++u) {
                float f[8];
                widen(row[u], f);
#pragma unroll
                for (int q = 0; q < 8; ++q)
                    if (column<WIDE, T>(c0, lane, q) < a.D) dot[u] = fmaf(d[q], f[q], dot[u]);
            }
        }
        if (dy)
#pragma unroll
            for (int u = 0; u < n; ++u) {
                float f[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) f[q] = w[u] * d[q];
                store8<WIDE>(dy + at[u], c0, lane, a.D, narrowed<T>(f));
            }
    }
    if (!dweights) return;
    float s = sum_of_eight(dot);
    if (a.share > 0) {                                             // (all warps of a token come here for the same entries)
        const int warps = 1 << a.share, first = warp >> a.share << a.share;
        if ((lane & 3) == 0) part[warp][lane >> 2] = s;
        asm volatile("bar.sync %0, %1;" ::"r"(1 + (warp >> a.share)), "r"(32 * warps) : "memory");
        s = 0.0f;
        for (int v = 0; v < warps; ++v) s += part[first + v][lane >> 2];
        asm volatile("bar.sync %0, %1;" ::"r"(1 + (warp >> a.share)), "r"(32 * warps) : "memory");
        if (p.start != 0) return;
    }
    const int u = lane >> 2, first_j = __shfl_sync(kAll, p.j0, (i + u) & 31), second_j = __shfl_sync(kAll, p.j1, (i + u) & 31);
    const int j = i + u < 32 ? first_j : second_j;
    if ((lane & 3) == 0 && u < n) dweights[(int64_t)p.token * a.k + j] = s;
}

template <typename T, bool WIDE>
__global__ void __launch_bounds__(kThreads, WIDE && sizeof(T) == 2 ? 3 : 2)
combine_grad_kernel(RowsArgs a, const T* dout, const T* y, T* dy, float* dweights)
{
    __shared__ float part[kWarps][8];
    const Part p = part_of(a);
    if (p.token >= a.tokens) return;
    const int lane = threadIdx.x & 31;
    if (dweights && p.start == 0) {
        if (p.out0) dweights[(int64_t)p.token * a.k + lane] = 0.0f;
        if (p.out1) dweights[(int64_t)p.token * a.k + lane + 32] = 0.0f;
    }
    int i = 0;
    for (; i + 4 <= p.entries; i += 4) grad_rows<4, WIDE>(a, p, dout, y, dy, dweights, i, part);
    if (i + 2 <= p.entries) { grad_rows<2, WIDE>(a, p, dout, y, dy, dweights, i, part); i += 2; }
    if (i < p.entries) grad_rows<1, WIDE>(a, p, dout, y, dy, dweights, i, part);
}

// How many warps share a token.  Of many tokens as many as leave at most a fifth of the lanes idle at the row's end, so that a row is
// read and written in long pieces; of few tokens as many as there is work for.  Returns the CTAs.
constexpr uint32_t kFewTokens = 592;                   // four CTAs per SM
unsigned set_share(RowsArgs& a, int64_t runs)
{
    a.share = 0;
    for (int s = 1; (1 << s) <= kWarps && runs > 32 << (s - 1); ++s) {
        const int64_t lanes = (int64_t)32 << s;
        if (a.tokens <= kFewTokens || (runs + lanes - 1) / lanes * lanes * 4 <= runs * 5) a.share = s;
    }
    return (unsigned)((((uint64_t)a.tokens << a.share) + kWarps - 1) / kWarps);
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

RowsArgs args_of(const taot_rows_params* p, const int32_t* perm, const int32_t* counts, const float* weights, int32_t* info)
{
    RowsArgs a;
    a.perm = perm; a.counts = counts; a.weights = weights; a.info = info;
    a.tokens = (uint32_t)(p->B * p->n); a.n = (uint32_t)p->n; a.cap = (uint32_t)(p->n * p->k); a.share = 0;
    a.ld_rows = p->ld_rows; a.ld_tokens = p->ld_tokens; a.ld_residual = p->ld_residual;
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
    RowsArgs a = args_of(p, d_perm, counts, nullptr, d_info);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int32_t cols = d_scales ? scale_cols : 0;
    // the widest words that every row is made of
    const uint64_t all = reinterpret_cast<uintptr_t>(d_x) | reinterpret_cast<uintptr_t>(d_rows) | (uint64_t)(p->ld_tokens * elem) |
                         (uint64_t)(p->ld_rows * elem) | (uint64_t)((int64_t)p->D * elem);
    const int64_t word = all % 16 == 0 ? 16 : all % 8 == 0 ? 8 : all % 4 == 0 ? 4 : all % 2 == 0 ? 2 : 1;
    a.ld_tokens = p->ld_tokens * elem / word;
    a.ld_rows = p->ld_rows * elem / word;
    a.D = (int32_t)((int64_t)p->D * elem / word);
    const unsigned grid = set_share(a, a.tokens <= kFewTokens ? a.D : (a.D + 3) / 4);       // (a lane takes four words)
    const auto launch = [&](auto t) {
        typedef decltype(t) W;
        send_kernel<W><<<grid, kThreads, 0, st>>>(a, static_cast<const W*>(d_x), static_cast<W*>(d_rows), d_scales, d_row_scales, cols);
        return cudaGetLastError();
    };
    TAOT_CUDA_OK(word == 16 ? launch(uint4()) : word == 8 ? launch(uint2()) : word == 4 ? launch(uint32_t()) : word == 2 ? launch(uint16_t()) : launch(uint8_t()));
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
    RowsArgs a = args_of(p, d_perm, counts, d_weights, d_info);
    a.wide = p->D % 8 == 0 && wide_rows(d_y, p->ld_rows, e) && wide_rows(d_residual, p->ld_residual, e) && wide_rows(d_out, p->ld_tokens, e);
    const unsigned grid = set_share(a, (p->D + 7) / 8);
    TAOT_CUDA_OK(by_type(p->dtype, [&](auto t) {
        typedef decltype(t) T;
        const auto kernel = a.wide ? combine_kernel<T, true> : combine_kernel<T, false>;
        kernel<<<grid, kThreads, 0, static_cast<cudaStream_t>(stream)>>>(
            a, static_cast<const T*>(d_y), static_cast<const T*>(d_residual), static_cast<T*>(d_out));
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
    RowsArgs a = args_of(p, d_perm, counts, d_weights, d_info);
    a.wide = p->D % 8 == 0 && wide_rows(d_dweights ? d_y : nullptr, p->ld_rows, e) && wide_rows(d_dy, p->ld_rows, e) && wide_rows(d_dout, p->ld_tokens, e);
    const unsigned grid = set_share(a, (p->D + 7) / 8);
    TAOT_CUDA_OK(by_type(p->dtype, [&](auto t) {
        typedef decltype(t) T;
        const auto kernel = a.wide ? combine_grad_kernel<T, true> : combine_grad_kernel<T, false>;
        kernel<<<grid, kThreads, 0, static_cast<cudaStream_t>(stream)>>>(
            a, static_cast<const T*>(d_dout), static_cast<const T*>(d_y), static_cast<T*>(d_dy), d_dweights);
        return cudaGetLastError();
    }));
    return TAOT_OK;
}

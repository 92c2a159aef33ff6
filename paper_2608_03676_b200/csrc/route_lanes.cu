// Routing with eight lanes per row: calls with a bias or groups, of few rows (whose time is that of one row), of long rows, and of rows
// that cannot be read in 16-byte pieces (route_common.cuh: how the choice is made).
#include "route_common.cuh"

namespace route {

namespace {

constexpr int kWarps = 4;
constexpr int kLanes = 8;
constexpr int kRows = 32 / kLanes;                 // of a warp

__device__ __forceinline__ float row_max(float v)
{
#pragma unroll
    for (int o = 1; o < kLanes; o *= 2) v = fmaxf(v, __shfl_xor_sync(kAll, v, o));
    return v;
}
__device__ __forceinline__ float row_min(float v) { return -row_max(-v); }
__device__ __forceinline__ float row_sum(float v)
{
#pragma unroll
    for (int o = 1; o < kLanes; o *= 2) v += __shfl_xor_sync(kAll, v, o);
    return v;
}

// merges the lists of the eight lanes of a row; all lanes end with the same list
template <bool LOST, int K>
__device__ __forceinline__ void merge_lanes(uint32_t (&v)[K], uint32_t& lost)
{
#pragma unroll
    for (int o = 1; o < kLanes; o *= 2) {
        uint32_t w[K];
#pragma unroll
        for (int i = 0; i < K; ++i) w[i] = __shfl_xor_sync(kAll, v[i], o);
        if (LOST) lost = max(lost, __shfl_xor_sync(kAll, lost, o));
        merge_list<LOST>(v, w, lost);
    }
}

// The lane of a row's eight that has its sub-th place by keys, larger ones first, equal ones by expert; lanes without an expert
// (-1) have the smallest key and come last.
__device__ __forceinline__ int lane_of_place(uint64_t key, int at)
{
    const int lane = threadIdx.x & 31, sub = lane & (kLanes - 1), base = lane - sub;
    int rank = 0, from = 0;
#pragma unroll
    for (int o = 1; o < kLanes; ++o) {
        const uint64_t u = __shfl_xor_sync(kAll, key, o);
        const int e = __shfl_xor_sync(kAll, at, o);
        const bool before = at < 0 ? e >= 0 || (sub ^ o) < sub : e >= 0 && (u > key || (u == key && e < at));
        if (before) ++rank;
    }
#pragma unroll
    for (int o = 0; o < kLanes; ++o)
        if (__shfl_sync(kAll, rank, base + o) == sub) from = o;
    return base + from;
}

__device__ __forceinline__ void copy_async(void* to, const void* from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}

// A row's logits: in memory (WIDE: rows of whole chunks, 16-byte aligned), or STAGED in shared memory, to which the warp has brought
// it: where a lane's chunks follow one another, the lanes of a load would be far apart in memory.  There a lane's own
// chunks are one 16-byte piece further from the next lane's than they would be, so that the lanes read different banks: piece p
// stands at p + (p * spread >> 16).
template <typename T, bool WIDE, bool STAGED>
struct Logits {
    const T* row;
    const uint4* tile;
    uint32_t spread;
    int E;
    __device__ __forceinline__ const T* at(int e) const
    {
        if (!STAGED) return row + e;
        constexpr int kPiece = 16 / (int)sizeof(T);
        const uint32_t p = (uint32_t)e / kPiece;
        return reinterpret_cast<const T*>(tile + p + (p * spread >> 16)) + e % kPiece;
    }
    // four logits from expert e on, NaN from `end` on
    __device__ __forceinline__ void chunk(int e, int end, float (&x)[4]) const
    {
        if (WIDE) four(at(e), x);
        else
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = e + i < end ? to_f32(row[e + i]) : __int_as_float(0x7fc00000);
    }
};

// BIAS: keys are scores with a bias added.  GROUP: 2, 4 or 8 groups; a lane's chunks follow one another, so that a group lies in
// 4, 2 or 1 lanes.  WIDE: rows of whole chunks that can be read as such (and with groups whole chunks in every lane).  U: chunks
// of a lane that are taken at a time (4 where it has no more).
// Registers for six CTAs per SM with K = 8 (80, and up to 300 bytes of spills with a bias or groups), four with K = 16.  Six against four
// CTAs (128 registers, no spills), us: 131072 x 256 fp32 64 : 73, bf16 with a bias 78 : 85, 2^20 x 256 fp32 with a bias and groups
// 773 : 795, 131072 of them 113 : 110; but four rows of them, which need no second CTA, 12.3 : 10.3.
template <typename T, int K, int U, bool BIAS, bool GROUP, bool WIDE>
__global__ void __launch_bounds__(kWarps * 32, K == 8 ? 6 : 4)
route_lanes_kernel(const __grid_constant__ RouteArgs a, uint32_t spread, int32_t pitch, int32_t warp_bytes)
{
    constexpr bool STAGED = WIDE && GROUP;         // (without groups 65536 x 256 bf16 take 17.6 us from memory, 19 staged)
    extern __shared__ uint4 shared[];
    constexpr int kOwn = K / kLanes;                               // places of the list that a lane stands for
    constexpr uint32_t kSlots = 4 * K - 1;
    constexpr bool kExact = !BIAS && sizeof(T) == 2;               // keys lose nothing
    constexpr uint32_t kLow = 0x1fff;                              // bits that the fp32 form of a 16-bit number leaves
    constexpr float big = Type<T>::big;
    const int lane = threadIdx.x & 31, sub = lane & (kLanes - 1);
    const int64_t first = ((int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5)) * kRows;
    if (first >= a.N) return;
    const int64_t mine = first + lane / kLanes;
    const int64_t row = mine < a.N ? mine : a.N - 1;               // (lanes past the end repeat the last row and write nothing)
    const bool routed = mine < a.N && (!a.mask || a.mask[row]);
    // the warp's shared memory: a list of experts, then its rows; the latter's place serves choose_exactly at the end
    int32_t* const found = reinterpret_cast<int32_t*>(reinterpret_cast<char*>(shared) + (threadIdx.x >> 5) * warp_bytes);
    uint4* const tile = reinterpret_cast<uint4*>(found + 32);
    if (STAGED) {
        const int pieces = a.E * (int)sizeof(T) / 16;
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const int64_t from = min(first + r, a.N - 1);
            const char* p = reinterpret_cast<const char*>(static_cast<const T*>(a.logits) + from * a.ld);
            for (int c = lane; c < pieces; c += 32) copy_async(tile + r * pitch + c + ((uint32_t)c * spread >> 16), p + 16 * c);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    }
    const Logits<T, WIDE, STAGED> logits = {static_cast<const T*>(a.logits) + row * a.ld, tile + lane / kLanes * pitch, spread, a.E};
    const float* b_row = BIAS ? a.bias + row / a.T * a.E : nullptr;
    constexpr bool CUT = GROUP && !WIDE;                           // a lane's part of its group may be any number of experts
    const int shift = GROUP ? __ffs(kLanes / a.groups) - 1 : 0, lanes = 1 << shift;       // of a group
    const int size = CUT ? a.E / a.groups : 0, part = CUT ? (size + lanes - 1) >> shift : 0;
    const int per = CUT ? (part + 3) / 4 : ((a.E + 3) / 4 + kLanes - 1) / kLanes;         // chunks of a lane
    const int C = CUT ? per * kLanes : (a.E + 3) / 4;
    // where chunk i of lane s, or chunk c, begins, and where that lane's (or the row's) experts end
    const auto begin = [&](int s, int i) { return (s >> shift) * size + (s & (lanes - 1)) * part + 4 * i; };
    const auto end = [&](int s) { return min((s >> shift) * size + ((s & (lanes - 1)) + 1) * part, ((s >> shift) + 1) * size); };
    const auto chunk = [&](int c, int& e, int& stop) {
        const int s = CUT ? c / per : 0;
        e = CUT ? begin(s, c - s * per) : 4 * c;
        stop = CUT ? end(s) : a.E;
    };
    const uint32_t cmask = (1u << a.chunk_bits) - 1;
    const uint32_t drop = max(cmask, kSlots);                      // the bits of a key that are no value

    if (STAGED) {
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncwarp();
    }
    Scores sc = {0.0f, 1.0f};
    float total = 1.0f;
    if (a.score == TAOT_SOFTMAX && (BIAS || GROUP || (!a.renormalise && a.weights))) {
        float top = -big;
        for (int e = 4 * sub; e < a.E; e += 4 * kLanes) {
            float x[4];
            logits.chunk(e, a.E, x);
#pragma unroll
            for (int q = 0; q < 4; ++q) top = fmaxf(top, x[q]);
        }
        sc.top = top = fminf(row_max(top), big);
        total = 0.0f;
        for (int e = 4 * sub; e < a.E; e += 4 * kLanes) {
            float x[4];
            logits.chunk(e, a.E, x);
#pragma unroll
            for (int q = 0; q < 4; ++q) total += x[q] > -big ? fast_exp2((fminf(x[q], big) - top) * kLog2e) : 0.0f;
        }
        total = row_sum(total);
        sc.inv = 1.0f / total;
    }
    const float off = score_error(a.score, sc, (a.E + kLanes - 1) / kLanes);

    // the K best chunks
    uint32_t best[K], lost = 0, bits = 0;
    float ref = 0.0f;
    float g1 = -INFINITY, g2 = -INFINITY;                          // the two largest keys of the lane's part of its group
    for (int i0 = 0; i0 < per; i0 += U) {
        uint32_t list[K];
#pragma unroll
        for (int u = 0; u < K; ++u) list[u] = 0;
        float xs[STAGED ? 1 : U][4], m[U];                           // (read from memory before any of them is used)
        if (!STAGED)
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int i = i0 + u;
                const int c = min(GROUP ? sub * per + i : i * kLanes + sub, C - 1);
                logits.chunk(CUT ? begin(sub, i) : 4 * c, CUT ? end(sub) : a.E, xs[STAGED ? 0 : u]);
            }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u;
            const int c = GROUP ? sub * per + i : i * kLanes + sub;
            m[u] = -INFINITY;
            if (i >= per || c >= C) continue;
            float (&x)[4] = xs[STAGED ? 0 : u];
            if (STAGED) logits.chunk(4 * c, a.E, x);
            const int e = CUT ? begin(sub, i) : 4 * c, stop = CUT ? end(sub) : a.E;
            if (BIAS) {
                float b[4];
                if (WIDE) four(b_row + e, b);
                else
#pragma unroll
                    for (int q = 0; q < 4; ++q) b[q] = e + q < stop ? b_row[e + q] : INFINITY;
                if (a.score == TAOT_SIGMOID) {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {                  // (an infinite logit has score 1 as it is)
                        const float v = score_of(TAOT_SIGMOID, sc, x[q]) + b[q];
                        x[q] = x[q] > -big && fabsf(v) < INFINITY ? v : -INFINITY;
                    }
                } else {
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float v = score_of(TAOT_SOFTMAX, sc, fminf(x[q], big)) + b[q];
                        x[q] = x[q] > -big && fabsf(v) < INFINITY ? v : -INFINITY;
                    }
                }
            } else if (GROUP || !kExact) {
                if (!kExact) bits |= __float_as_uint(x[0]) | __float_as_uint(x[1]) | __float_as_uint(x[2]) | __float_as_uint(x[3]);
#pragma unroll
                for (int q = 0; q < 4; ++q) x[q] = seen(x[q], big);
            }
            if (GROUP) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    g2 = fmaxf(g2, fminf(g1, x[q]));
                    g1 = fmaxf(g1, x[q]);
                }
            }
            m[u] = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3]));
            if (!BIAS) m[u] = seen(m[u], big) + 0.0f;              // (+ 0: one zero)
        }
        if (!kExact && i0 == 0) {
            // keys are of the distance to the largest (of the first block), which keeps more of what tells the best apart; not so
            // where the logits' own bits are fewer than a key's
            float most = -INFINITY;
#pragma unroll
            for (int u = 0; u < U; ++u) most = fmaxf(most, m[u]);
            most = row_max(most);
            if (BIAS || (per <= U && (__reduce_or_sync(kAll, bits) & drop) != 0)) ref = most > -INFINITY ? most : 0.0f;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int i = i0 + u, c = GROUP ? sub * per + i : i * kLanes + sub;
            if (m[u] > -INFINITY) list[u] = (ordered(kExact ? m[u] : m[u] - ref) & ~cmask) | (cmask - (uint32_t)c);
        }
        sort_list(list);
        if (i0 == 0) {
#pragma unroll
            for (int i = 0; i < K; ++i) best[i] = list[i];
        } else {
            merge_list<!kExact>(best, list, lost);
        }
    }
    bool redo = false;
    uint32_t kept_lanes = 1u;                                      // of the row, by its lanes
    if (GROUP) {
        for (int o = 1; o < lanes; o *= 2) {
            const float h1 = __shfl_xor_sync(kAll, g1, o), h2 = __shfl_xor_sync(kAll, g2, o);
            g2 = fmaxf(fminf(g1, h1), fmaxf(g2, h2));
            g1 = fmaxf(g1, h1);
        }
        float s1 = g1, s2 = g2;
        if (!BIAS) {
            s1 = g1 > -INFINITY ? score_of(a.score, sc, g1) : -INFINITY;
            s2 = g2 > -INFINITY ? score_of(a.score, sc, g2) : -INFINITY;
        }
        const float score = a.top == 2 && s2 > -INFINITY ? s1 + s2 : s1;
        const int g = sub >> shift;
        int rank = 0;
#pragma unroll
        for (int o = 1; o < kLanes; ++o) {
            const float other = __shfl_xor_sync(kAll, score, o);
            const int h = (sub ^ o) >> shift;
            if (h != g && ((sub ^ o) & (lanes - 1)) == 0 && (other > score || (other == score && h < g))) ++rank;
        }
        bool kept = rank < a.kept;
        const float worst = row_min(kept ? score : INFINITY), next = row_max(kept ? -INFINITY : score);
        const float size = row_max(s1 > -INFINITY ? fmaxf(fabsf(s1), s2 > -INFINITY ? fabsf(s2) : 0.0f) : 0.0f);
        const bool close = routed && a.kept < a.groups && !(worst - next > 4.0f * off + 8.0f * size * 1.2e-7f);
        // (a key that counts in a group is at most twice the error below the last one that counts here)
        const float least = (a.top == 2 ? g2 : g1) - (BIAS ? 2.0f * off + 2.4e-7f * size : 0.0f);
        for (unsigned left = __ballot_sync(kAll, close); left;) {
            const int from = (__ffs(left) - 1) & ~(kLanes - 1);
            left &= ~(((1u << kLanes) - 1) << from);
            const Scores s = {__shfl_sync(kAll, sc.top, from), __shfl_sync(kAll, sc.inv, from)};
            uint32_t groups;
            const bool settled = settle_groups(a, first + from / kLanes, s, least, from, lanes, found, groups);
            if ((lane & ~(kLanes - 1)) == from) {
                if (settled) kept = groups >> g & 1;
                else redo = true;
            }
        }
        kept_lanes = __ballot_sync(kAll, kept) >> (lane & ~(kLanes - 1)) & ((1u << kLanes) - 1);
        if (!kept) {
#pragma unroll
            for (int i = 0; i < K; ++i) best[i] = 0;
            lost = 0;
        }
    }
    merge_lanes<!kExact>(best, lost);

    // their experts: a lane takes chunks sub, sub + 8
    int id[kOwn];
    if (kExact) {
#pragma unroll
        for (int i = 0; i < K; ++i)
            if (i % kLanes == sub) id[i / kLanes] = (int)(cmask - (best[i] & cmask));    // (none: cmask, which is behind all chunks)
    } else {
        uint32_t ids[K];                                           // in ascending order, so that places are in the experts' order
#pragma unroll
        for (int i = 0; i < K; ++i) ids[i] = ~(cmask - (best[i] & cmask));
        sort_list(ids);
#pragma unroll
        for (int i = 0; i < K; ++i)
            if (i % kLanes == sub) id[i / kLanes] = (int)~ids[i];
    }
    uint32_t list[K];
#pragma unroll
    for (int i = 0; i < K; ++i) list[i] = 0;
#pragma unroll
    for (int h = 0; h < kOwn; ++h) {
        if (id[h] >= C) continue;
        float x[4];
        int e0, stop;
        chunk(id[h], e0, stop);
        logits.chunk(e0, stop, x);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int e = e0 + q;
            float v = seen(x[q], big) + 0.0f;
            if (BIAS) {
                const float b = WIDE || e < stop ? b_row[e] : INFINITY;
                v = v > -INFINITY && fabsf(b) < INFINITY ? score_of(a.score, sc, v) + b : -INFINITY;
            }
            const uint32_t low = kExact ? kLow - (uint32_t)e : kSlots - (uint32_t)(4 * (sub + kLanes * h) + q);
            list[4 * h + q] = v > -INFINITY ? (ordered(kExact ? v : v - ref) & ~(kExact ? kLow : kSlots)) | low : 0u;
        }
    }
    sort_list(list);
    merge_lanes<!kExact>(list, lost);

    // a lane's places
    int at[kOwn];
    float x[kOwn], v[kOwn];
#pragma unroll
    for (int h = 0; h < kOwn; ++h) {
        uint32_t key = 0;
#pragma unroll
        for (int i = 0; i < K; ++i)
            if (i == sub + kLanes * h) key = list[i];
        const bool there = key != 0 && sub + kLanes * h < a.k;
        if (kExact) {
            at[h] = there ? (int)(kLow - (key & kLow)) : -1;
        } else {
            const int slot = (int)(kSlots - (key & kSlots));
            const int from = (lane & ~(kLanes - 1)) | ((slot >> 2) & (kLanes - 1));
            int number = __shfl_sync(kAll, id[0], from);
            if constexpr (kOwn > 1) {
                const int other = __shfl_sync(kAll, id[1], from);
                if (slot >> 5) number = other;
            }
            int e0, stop;
            chunk(number, e0, stop);
            at[h] = there ? e0 + (slot & 3) : -1;
        }
        x[h] = there ? seen(to_f32(*logits.at(at[h])), big) : -INFINITY;
        v[h] = x[h];
    }
    bool settle = false;
    float least = -INFINITY;                                       // a lower bound of the last chosen one's key
    if (!kExact) {
        // Is what was left out far enough below the last chosen one (the k-th, or the last there is)?  And are neighbours in order?
        uint32_t beyond = lost, last = 0;
#pragma unroll
        for (int i = 0; i < K; ++i) {
            if (i >= a.k) beyond = max(beyond, list[i]);
            else last = list[i];
        }
        const bool lossless = !BIAS && (__reduce_or_sync(kAll, bits) & drop) == 0;
        bool fine = true;                                          // this lane's places and their successors
        if (BIAS) {
            float b[kOwn];
#pragma unroll
            for (int h = 0; h < kOwn; ++h) {
                b[h] = at[h] >= 0 ? b_row[at[h]] : 0.0f;
                v[h] = at[h] >= 0 ? score_of(a.score, sc, x[h]) + b[h] : -INFINITY;
            }
            const float size = row_max(fmaxf(v[0] > -INFINITY ? fabsf(v[0]) : 0.0f, v[kOwn - 1] > -INFINITY ? fabsf(v[kOwn - 1]) : 0.0f));
            const float err = 2.0f * off + 2.4e-7f * size;
            if (K == 8) {                                          // put right what the lost bits have turned round
                const float after = __shfl_down_sync(kAll, v[0], 1);
                const int e_after = __shfl_down_sync(kAll, at[0], 1);
                const bool turned = sub < kLanes - 1 && e_after >= 0 && (after > v[0] || (after == v[0] && e_after < at[0]));
                if (__any_sync(kAll, turned)) {
                    const int from = lane_of_place((uint64_t)ordered(v[0]), at[0]);
                    at[0] = __shfl_sync(kAll, at[0], from);
                    x[0] = __shfl_sync(kAll, x[0], from);
                    v[0] = __shfl_sync(kAll, v[0], from);
                    b[0] = __shfl_sync(kAll, b[0], from);
                }
            }
#pragma unroll
            for (int h = 0; h < kOwn; ++h) {
                // the next place: the next lane's, or the next list's first
                const int from = (lane & ~(kLanes - 1)) | ((sub + 1) & (kLanes - 1));
                const bool wraps = sub == kLanes - 1;
                float u = __shfl_sync(kAll, v[h], from), y = __shfl_sync(kAll, x[h], from), c = __shfl_sync(kAll, b[h], from);
                int e = __shfl_sync(kAll, at[h], from);
                if constexpr (kOwn > 1) {
                    const float u1 = __shfl_sync(kAll, v[1], from), y1 = __shfl_sync(kAll, x[1], from), c1 = __shfl_sync(kAll, b[1], from);
                    const int e1 = __shfl_sync(kAll, at[1], from);
                    if (wraps && h == 0) { u = u1; y = y1; c = c1; e = e1; }
                }
                if (wraps && h == kOwn - 1) e = -1;
                if (e >= 0 && !(v[h] - u > err) && !(x[h] == y && b[h] == c && at[h] < e)) fine = false;
            }
            if (K == 8 && a.score == TAOT_SIGMOID && __any_sync(kAll, !fine)) {          // the order of the chosen ones in 64 bits
                const int from = lane_of_place(at[0] >= 0 ? exact_key(a, b_row, true, row, at[0], 0.0f, 1.0) : 0ull, at[0]);
                at[0] = __shfl_sync(kAll, at[0], from);
                x[0] = __shfl_sync(kAll, x[0], from);
                fine = true;
            }
            least = row_min(fminf(v[0] > -INFINITY ? v[0] : INFINITY, v[kOwn - 1] > -INFINITY ? v[kOwn - 1] : INFINITY));
            // (both are distances from ref, which may be far larger than the chosen keys: each was rounded by half an ulp of its own)
            if (beyond != 0 && !(least - ref > number_of(beyond | drop) + err + 1.2e-7f * (fabsf(ref) + size))) fine = false;
            least -= err;
        } else if (!lossless) {
            least = row_min(fminf(x[0] > -INFINITY ? x[0] : INFINITY, x[kOwn - 1] > -INFINITY ? x[kOwn - 1] : INFINITY));
            if (beyond != 0 && ((beyond ^ last) & ~drop) == 0) fine = false;
            if (K == 8) {
                const float after = __shfl_down_sync(kAll, x[0], 1);
                if (sub < kLanes - 1 && after > x[0]) fine = false;
            } else {
#pragma unroll
                for (int i = 0; i + 1 < K; ++i)
                    if (i + 1 < a.k && list[i + 1] != 0 && ((list[i] ^ list[i + 1]) & ~drop) == 0) fine = false;
            }
        }
        const unsigned bad = __ballot_sync(kAll, !fine);
        settle = routed && !redo && ((bad >> (lane & ~(kLanes - 1))) & ((1u << kLanes) - 1)) != 0;
    }
    redo = redo && routed;
    if (!routed) {
#pragma unroll
        for (int h = 0; h < kOwn; ++h) { at[h] = -1; x[h] = -INFINITY; }
    }
    if (BIAS || GROUP || !kExact) {
        for (unsigned left = __ballot_sync(kAll, settle || redo); left;) {             // (all lanes are done with the staged rows)
            const int from = (__ffs(left) - 1) & ~(kLanes - 1);
            left &= ~(((1u << kLanes) - 1) << from);
            const int64_t r = first + from / kLanes;
            const Scores s = {__shfl_sync(kAll, sc.top, from), __shfl_sync(kAll, sc.inv, from)};
            const float limit = __shfl_sync(kAll, least, from);
            const uint32_t lanes_kept = __shfl_sync(kAll, kept_lanes, from);
            uint32_t groups = 1u;
            if (GROUP) {
                groups = 0;
                for (int g = 0; g < a.groups; ++g) groups |= (lanes_kept >> (g << shift) & 1u) << g;
            }
            if (__shfl_sync(kAll, (int)redo, from) || !settle_choice(a, r, s, groups, limit, found)) {
                int at0 = -1, at1 = -1;
                float t, z;
                choose_exactly(a, r, reinterpret_cast<uint64_t*>(tile), at0, at1, t, z);
                found[lane] = at0;
                __syncwarp();
            }
            if ((lane & ~(kLanes - 1)) == from)
#pragma unroll
                for (int h = 0; h < kOwn; ++h) {
                    at[h] = sub + kLanes * h < a.k ? found[sub + kLanes * h] : -1;
                    x[h] = at[h] >= 0 ? logit_at(a.logits, r * a.ld + at[h], a.dtype) : -INFINITY;
                }
            __syncwarp();
        }
    }
    float w[kOwn];
    if (a.weights) {
        float most = -INFINITY;
        if (a.renormalise) most = row_max(fmaxf(x[0], x[kOwn - 1]));
        float sum = 0.0f;
#pragma unroll
        for (int h = 0; h < kOwn; ++h) {
            w[h] = at[h] < 0 ? 0.0f : a.renormalise ? part_of(a.score, x[h], most) : a.score == TAOT_SIGMOID ? sigmoid(x[h]) : expf(x[h] - sc.top) * sc.inv;
            sum += w[h];
        }
        if (a.renormalise) {
            sum = row_sum(sum);
            const float share = sum > 0.0f ? 1.0f / sum : 0.0f;
#pragma unroll
            for (int h = 0; h < kOwn; ++h) w[h] *= share;
        }
    }
#pragma unroll
    for (int h = 0; h < kOwn; ++h)
        if (mine < a.N && sub + kLanes * h < a.k) {
            a.topk[row * a.k + sub + kLanes * h] = at[h];
            if (a.weights) a.weights[row * a.k + sub + kLanes * h] = a.scale * w[h];
        }
}

// a warp's shared memory: a list of 32 experts, and its rows of `pitch` pieces each or the keys of choose_exactly
constexpr int32_t warp_memory(int32_t pitch, int32_t E)
{
    const int32_t tile = kRows * pitch * 16, exact = (int32_t)sizeof(uint64_t) * E;
    return 128 + ((tile > exact ? tile : exact) + 15) / 16 * 16;
}

template <typename T, int K, int U, bool WIDE>
cudaError_t launch(const RouteArgs& a, cudaStream_t st)
{
    const unsigned grid = (unsigned)((a.N + kWarps * kRows - 1) / (kWarps * kRows));
    const int32_t pieces = a.E * (int32_t)sizeof(T) / 16, chunks = (a.E + 3) / 4;
    // a lane's pieces, where its chunks follow one another and are whole pieces
    const int32_t own = a.groups > 1 && chunks % kLanes == 0 ? chunks / kLanes * 4 * (int32_t)sizeof(T) : 0;
    const uint32_t spread = WIDE && own > 0 && own % 16 == 0 ? (65536u + own / 16 - 1) / (own / 16) : 0u;      // (exact for up to 256 pieces)
    const int32_t pitch = WIDE && a.groups > 1 ? pieces + (spread ? kLanes : 0) : 0;
    const int32_t warp_bytes = warp_memory(pitch, a.E);
    const size_t smem = (size_t)warp_bytes * kWarps, most = a.groups > 1 ? (size_t)kWarps * warp_memory(WIDE ? kMaxE * (int32_t)sizeof(T) / 16 + kLanes : 0, kMaxE) : 0;
    const auto run = [&](auto kernel) {
        const cudaError_t e = allow_shared(kernel, most);          // (without groups 33 KB at most)
        if (e != cudaSuccess) return e;
        kernel<<<grid, kWarps * 32, smem, st>>>(a, spread, pitch, warp_bytes);
        return cudaGetLastError();
    };
    if (a.groups > 1) return a.bias ? run(route_lanes_kernel<T, K, U, true, true, WIDE>) : run(route_lanes_kernel<T, K, U, false, true, WIDE>);
    return a.bias ? run(route_lanes_kernel<T, K, U, true, false, WIDE>) : run(route_lanes_kernel<T, K, U, false, false, WIDE>);
}

template <typename T>
cudaError_t by_shape(const RouteArgs& a, bool wide, cudaStream_t st)
{
    if (a.k > 8) return wide ? launch<T, 16, 8, true>(a, st) : launch<T, 16, 8, false>(a, st);
    if (wide) return a.E <= 128 ? launch<T, 8, 4, true>(a, st) : launch<T, 8, 8, true>(a, st);
    return launch<T, 8, 8, false>(a, st);
}

}  // namespace

cudaError_t launch_lanes(const RouteArgs& a, bool wide, cudaStream_t st)
{
    wide = wide && a.E * layer::type_bytes(a.dtype) % 16 == 0 && !misaligned(a.bias, 16) && (a.groups == 1 || a.E % 32 == 0);
    if (a.dtype == TAOT_F32) return by_shape<float>(a, wide, st);
    if (a.dtype == TAOT_BF16) return by_shape<__nv_bfloat16>(a, wide, st);
    return by_shape<__half>(a, wide, st);
}

}  // namespace route

// The rows of the parallel-group layout from token ids, and the gradients of the two tables they come from (see
// include/ps_train.h; Section 4.3).  Everything here is bound by memory: a row of the layout is written, or read, once.
// 8 x 2048 tokens, k 4, H 4096, bf16: the rows 125 us (5.4 TB/s written), the gradients 226 (933 MB at a copy's 5.1 TB/s: 181).  203 tokens, k 5,
// H 5120: the gradients 74 us, of which writing the table's 32000 rows takes 62.
#include <math.h>

#include "ps_train_device.h"

namespace {

constexpr int GE_THREADS = 256;

__device__ __forceinline__ void stg_stream16_u(void* p, u32x4 v) { __builtin_nontemporal_store((u32x4_q)v, reinterpret_cast<u32x4_q*>(p)); }
__device__ __forceinline__ u32x4 ldg_u(const void* p) { return (u32x4)*reinterpret_cast<const u32x4_q*>(p); }
__device__ __forceinline__ u32x4 ldg_stream_u(const void* p) { return (u32x4)__builtin_nontemporal_load(reinterpret_cast<const u32x4_q*>(p)); }

template <typename WT> __device__ __forceinline__ void widen16(u32x4 x, float* v) { unpack_group<WT>(make_uint4(x[0], x[1], x[2], x[3]), v); }
template <typename WT> __device__ __forceinline__ u32x4 narrow16(const float* v) {
    u32x4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (Traits<WT>::BF) r[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
        else r[i] = __float_as_uint(v[i]);
    }
    return r;
}
template <typename WT> __device__ __forceinline__ u32x4 scaled16(u32x4 x, float scale) {
    constexpr int GE = Traits<WT>::GE;
    float v[GE];
    widen16<WT>(x, v);
#pragma unroll
    for (int e = 0; e < GE; ++e) v[e] *= scale;
    return narrow16<WT>(v);
}

struct GeParams {
    int n, T, k, pieces, vocab;       // positions (seqs * tokens); 16-byte pieces of a row
    float scale;
    const int* ids;
    const char *embed, *mask_emb, *dx;
    char *x, *d_embed, *d_mask;
    // gradients: positions sorted by token, the tokens' ranges in them; sums of pieces of long ranges; sums of [MASK] rows
    u64 *keys, *sorted;
    int2* range;
    float *part, *mask_part;
    int chunk_log, chunks;            // positions are sorted in chunks of 2^chunk_log
    int parts, part_n, lanes;         // [MASK] rows: parts of part_n groups, of which `lanes` threads share a piece
    int mask_wgs;                     // workgroups of the last kernel that add up the parts of the [MASK] rows
};

// One group of the layout per workgroup: the token's row of the table and the k [MASK] rows, which every group has and the L2 holds.
template <typename WT>
__global__ void __launch_bounds__(GE_THREADS) ge_embed_kernel(const GeParams P) {
    const unsigned n = blockIdx.x;
    const int id = P.ids[n];
    const bool known = (unsigned)id < (unsigned)P.vocab;
    const size_t rb = (size_t)P.pieces * 16;
    const char* src = P.embed + (known ? (size_t)id * rb : 0);
    char* dst = P.x + (size_t)n * (P.k + 1) * rb;
    for (int c = threadIdx.x; c < P.pieces; c += GE_THREADS) {
        const u32x4 e = ldg_u(src + (size_t)c * 16);
        for (int s = 1; s <= P.k; ++s) stg_stream16_u(dst + s * rb + (size_t)c * 16, scaled16<WT>(ldg_u(P.mask_emb + (size_t)(s - 1) * rb + (size_t)c * 16), P.scale));
        const u32x4 z = {0u, 0u, 0u, 0u};
        stg_stream16_u(dst + (size_t)c * 16, known ? scaled16<WT>(e, P.scale) : z);
    }
}

// ------------------------------------------------------------------------------------------
// Gradients.  Three or four launches:
//   1  chunks of up to 16384 positions sorted by (token, position) in LDS, one workgroup each, beside partial sums of the [MASK] rows,
//      one workgroup for a slot and a part of the groups
//   2  (more than one chunk) an element's place among all is the sum of its places in every chunk, found by bisection;
//      then the tokens' ranges
//   3  long ranges (more than GE_WINDOW positions) are added up window by window: the sorted positions in windows of
//      GE_WINDOW, each with a sum for the range that its first position is in and one for that of its last
//   4  a workgroup per row of the table: its few positions, or its windows' sums, or zeros; others add up the [MASK] parts
// Every sum is taken in the order of the sorted positions (or parts), so the bits depend on the ids and sizes alone.
// ------------------------------------------------------------------------------------------
constexpr int GE_SORT_THREADS = 1024, GE_CHUNK_LOG = 14, GE_SMALL_LOG = 12, GE_WINDOW = 64;

// The elements of one chunk in LDS, ascending: compare-and-exchange networks of strides below the size (Batcher's bitonic sort).  A thread holds
// 2^E elements and does E strides in registers between two visits to the LDS: 2^14 elements by 16 take 29 visits instead of 105.  16 a
// thread for more than 4096 positions, 4 below, where 16 would leave few threads (203 positions 10 us by 4 and 16 by 16; 16384
// positions, beside the partial sums, 107 by 16 and 167 with a visit per stride).
// Element i lies at i + i / 16, so that the contiguous ones of neighbouring threads lie in other banks.
__device__ __forceinline__ int ge_place(int i) { return i + (i >> 4); }
__device__ __forceinline__ void ge_order(u64& x, u64& y, bool up) {
    const u64 a = x, b = y;
    const bool swap = (a > b) == up;
    x = swap ? b : a;
    y = swap ? a : b;
}
template <int E> __device__ __forceinline__ void ge_sort_lds(u64* s, int log_n, int tid) {
    constexpr int N = 1 << E;
    const bool active = tid < 1 << (log_n - E);
    u64 x[N];
    __syncthreads();
    if (active) {                                            // runs of 2^E, every second one descending
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = s[ge_place(N * tid + e)];
#pragma unroll
        for (int a = 1; a <= E; ++a)
#pragma unroll
            for (int b = a - 1; b >= 0; --b)
#pragma unroll
                for (int e = 0; e < N; ++e)
                    if (!(e >> b & 1)) ge_order(x[e], x[e | 1 << b], a < E ? !(e >> a & 1) : !(tid & 1));
#pragma unroll
        for (int e = 0; e < N; ++e) s[ge_place(N * tid + e)] = x[e];
    }
    for (int a = E + 1; a <= log_n; ++a)                     // runs of 2^a; (the last merge: all ascending)
        for (int b = a - 1; b >= 0;) {
            const int w = max(b - E + 1, 0), first = (tid >> w) << (w + E) | (tid & ((1 << w) - 1));   // strides 2^b .. 2^w
            const bool up = !(first >> a & 1);
            __syncthreads();
            if (active) {
#pragma unroll
                for (int e = 0; e < N; ++e) x[e] = s[ge_place(first | e << w)];
#pragma unroll
                for (int j = E - 1; j >= 0; --j)
                    if (j <= b - w) {
#pragma unroll
                        for (int e = 0; e < N; ++e)
                            if (!(e >> j & 1)) ge_order(x[e], x[e | 1 << j], up);
                    }
#pragma unroll
                for (int e = 0; e < N; ++e) s[ge_place(first | e << w)] = x[e];
            }
            b = w - 1;
        }
    __syncthreads();
}
__device__ __forceinline__ int ge_id(const GeParams& P, u64 key) { return (int)(key >> 32); }
// where a sorted run of equal tokens begins and ends (tokens that are none, P.vocab, have no range)
__device__ __forceinline__ void ge_mark(const GeParams& P, int i, u64 before, u64 me, u64 after) {
    const int id = ge_id(P, me);
    if (id >= P.vocab) return;
    if (i == 0 || ge_id(P, before) != id) P.range[id].x = i;
    if (i == P.n - 1 || ge_id(P, after) != id) P.range[id].y = i + 1;
}

// (LOG: the LDS holds a chunk of up to 2^LOG elements; 0: nothing is sorted.  With 2^12 two workgroups share a compute unit.)
template <typename WT, int LOG>
__global__ void __launch_bounds__(GE_SORT_THREADS) ge_sort_kernel(const GeParams P) {
    __shared__ u64 s[(1 << LOG) * 17 / 16];
    const int tid = threadIdx.x;
    if (LOG > 0 && (int)blockIdx.x < P.chunks) {
        const int ch = blockIdx.x, first = ch << P.chunk_log, size = 1 << P.chunk_log;
        for (int i = tid; i < size; i += GE_SORT_THREADS) {
            u64 key = ~0ull;                                // (behind all: not an element)
            if (first + i < P.n) {
                const int id = P.ids[first + i];
                key = (u64)((unsigned)id < (unsigned)P.vocab ? (unsigned)id : (unsigned)P.vocab) << 32 | (unsigned)(first + i);
            }
            s[ge_place(i)] = key;
        }
        for (int v = ch * GE_SORT_THREADS + tid; v < P.vocab; v += P.chunks * GE_SORT_THREADS) P.range[v] = make_int2(0, 0);
        ge_sort_lds<(LOG > GE_SMALL_LOG ? 4 : 2)>(s, P.chunk_log, tid);
        u64* out = P.chunks == 1 ? P.sorted : P.keys;
        const int n = min(size, P.n - first);
        for (int i = tid; i < n; i += GE_SORT_THREADS) {
            const u64 me = s[ge_place(i)];
            out[first + i] = me;
            if (P.chunks == 1) ge_mark(P, i, s[ge_place(max(i - 1, 0))], me, s[ge_place(min(i + 1, n - 1))]);
        }
        return;
    }
    // ---- a slot's rows in one part of the groups: `lanes` threads per piece take every lanes-th group
    constexpr int GE = Traits<WT>::GE;
    const int wg = blockIdx.x - P.chunks, slot = wg / P.parts + 1, part = wg % P.parts;
    const size_t rb = (size_t)P.pieces * 16, step = (size_t)P.lanes * (P.k + 1) * rb;
    const int lane = P.lanes > 1 ? tid / P.pieces : 0, lo = part * P.part_n + lane, hi = min((part + 1) * P.part_n, P.n);
    if (P.lanes > 1 && lane >= P.lanes) return;
    for (int c = P.lanes > 1 ? tid % P.pieces : tid; c < P.pieces; c += GE_SORT_THREADS) {
        float sum[GE];
#pragma unroll
        for (int e = 0; e < GE; ++e) sum[e] = 0.f;
        const char* p = P.dx + ((size_t)lo * (P.k + 1) + slot) * rb + (size_t)c * 16;
        int g = lo;
        for (; g + 7 * P.lanes < hi; g += 8 * P.lanes, p += 8 * step) {
            u32x4 x[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) x[u] = ldg_stream_u(p + u * step);
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                float v[GE];
                widen16<WT>(x[u], v);
#pragma unroll
                for (int e = 0; e < GE; ++e) sum[e] += v[e];
            }
        }
        for (; g < hi; g += P.lanes, p += step) {
            float v[GE];
            widen16<WT>(ldg_stream_u(p), v);
#pragma unroll
            for (int e = 0; e < GE; ++e) sum[e] += v[e];
        }
        float* out = P.mask_part + (((size_t)(slot - 1) * P.parts + part) * P.lanes + lane) * P.pieces * GE + (size_t)c * GE;
#pragma unroll
        for (int e = 0; e < GE; e += 4) *reinterpret_cast<f32x4*>(out + e) = f32x4{sum[e], sum[e + 1], sum[e + 2], sum[e + 3]};
    }
}

// an element's place: how many elements of every chunk are smaller (elements are all different)
__global__ void __launch_bounds__(GE_THREADS) ge_rank_kernel(const GeParams P) {
    const int i = blockIdx.x * GE_THREADS + threadIdx.x;
    if (i >= P.n) return;
    const u64 key = P.keys[i];
    int place = 0;
    for (int c = 0; c < P.chunks; ++c) {
        const int first = c << P.chunk_log, end = min(first + (1 << P.chunk_log), P.n);
        if (i >= first && i < end) {
            place += i - first;
            continue;
        }
        int lo = first, hi = end;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (P.keys[mid] < key) lo = mid + 1;
            else hi = mid;
        }
        place += lo - first;
    }
    P.sorted[place] = key;
}
__global__ void __launch_bounds__(GE_THREADS) ge_range_kernel(const GeParams P) {
    const int i = blockIdx.x * GE_THREADS + threadIdx.x;
    if (i < P.n) ge_mark(P, i, P.sorted[max(i - 1, 0)], P.sorted[i], P.sorted[min(i + 1, P.n - 1)]);
}

// sum[] += the 16-byte pieces c of the rows of sorted positions lo .. hi - 1, in that order
template <typename WT>
__device__ __forceinline__ void ge_add_rows(const GeParams& P, int lo, int hi, int c, float* sum) {
    constexpr int GE = Traits<WT>::GE;
    const size_t gb = (size_t)(P.k + 1) * P.pieces * 16;
    for (int i0 = lo; i0 < hi; i0 += 8) {
        u32x4 x[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) x[u] = ldg_stream_u(P.dx + (size_t)(unsigned)P.sorted[min(i0 + u, hi - 1)] * gb + (size_t)c * 16);
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (i0 + u < hi) {
                float v[GE];
                widen16<WT>(x[u], v);
#pragma unroll
                for (int e = 0; e < GE; ++e) sum[e] += v[e];
            }
    }
}

template <typename WT>
__global__ void __launch_bounds__(GE_THREADS) ge_window_kernel(const GeParams P) {
    constexpr int GE = Traits<WT>::GE;
    const int w = blockIdx.x, lo = w * GE_WINDOW, hi = min(lo + GE_WINDOW, P.n);
    const int id0 = ge_id(P, P.sorted[lo]), id1 = ge_id(P, P.sorted[hi - 1]);
#pragma unroll 1
    for (int which = 0; which < 2; ++which) {
        const int id = which ? id1 : id0;
        if (id >= P.vocab || (which && id1 == id0)) continue;
        const int2 r = P.range[id];
        if (r.y - r.x <= GE_WINDOW) continue;
        float* out = P.part + ((size_t)2 * w + which) * P.pieces * GE;
        for (int c = blockIdx.y * GE_THREADS + threadIdx.x; c < P.pieces; c += gridDim.y * GE_THREADS) {
            float sum[GE];
#pragma unroll
            for (int e = 0; e < GE; ++e) sum[e] = 0.f;
            ge_add_rows<WT>(P, max(r.x, lo), min(r.y, hi), c, sum);
#pragma unroll
            for (int e = 0; e < GE; e += 4) *reinterpret_cast<f32x4*>(out + (size_t)c * GE + e) = f32x4{sum[e], sum[e + 1], sum[e + 2], sum[e + 3]};
        }
    }
}

template <typename WT>
__global__ void __launch_bounds__(GE_THREADS) ge_rows_kernel(const GeParams P) {
    constexpr int GE = Traits<WT>::GE, Q = GE / 4;
    const int tid = threadIdx.x;
    if ((int)blockIdx.x < P.mask_wgs) {
        // ---- 16 groups of four columns of a slot, 16 threads each: a thread adds up every 16th part, the first of them the 16 sums
        __shared__ f32x4 s[16][16];
        const int quads = P.pieces * Q, per_slot = (quads + 15) / 16, slot = blockIdx.x / per_slot, q = (blockIdx.x % per_slot) * 16 + (tid & 15);
        const int all = P.parts * P.lanes;
        const f32x4* src = reinterpret_cast<const f32x4*>(P.mask_part) + (size_t)slot * all * quads + min(q, quads - 1);
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
        for (int i = tid >> 4; i < all; i += 16) sum += src[(size_t)i * quads];
        s[tid >> 4][tid & 15] = sum;
        __syncthreads();
        if (tid >= 16 || q >= quads) return;
        for (int i = 1; i < 16; ++i) sum += s[i][tid];
        sum *= P.scale;
        if constexpr (Traits<WT>::BF) {
            const u32x2 v = {pack_bf16x2(sum[0], sum[1]), pack_bf16x2(sum[2], sum[3])};
            *reinterpret_cast<u32x2_q*>(P.d_mask + ((size_t)slot * quads + q) * 8) = (u32x2_q)v;
        } else {
            *reinterpret_cast<f32x4_q*>(P.d_mask + ((size_t)slot * quads + q) * 16) = (f32x4_q)sum;
        }
        return;
    }
    const int id = blockIdx.x - P.mask_wgs;
    const int2 r = P.range[id];
    char* out = P.d_embed + (size_t)id * P.pieces * 16;
    for (int c = tid; c < P.pieces; c += GE_THREADS) {
        float sum[GE];
#pragma unroll
        for (int e = 0; e < GE; ++e) sum[e] = 0.f;
        if (r.y - r.x <= GE_WINDOW) {
            ge_add_rows<WT>(P, r.x, r.y, c, sum);
        } else {
            for (int w = r.x / GE_WINDOW; w <= (r.y - 1) / GE_WINDOW; ++w) {   // (a window that the range begins in has its sum as its second)
                const f32x4* p = reinterpret_cast<const f32x4*>(P.part + ((size_t)2 * w + (w * GE_WINDOW < r.x)) * P.pieces * GE + (size_t)c * GE);
#pragma unroll
                for (int e = 0; e < Q; ++e) {
                    const f32x4 v = p[e];
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[4 * e + i] += v[i];
                }
            }
        }
#pragma unroll
        for (int e = 0; e < GE; ++e) sum[e] *= P.scale;
        stg_stream16_u(out + (size_t)c * 16, narrow16<WT>(sum));
    }
}

template <typename A> int check(const A* a) {
    if (!a) return PS_ERR_NULL;
    if (a->seqs < 1 || a->tokens < 1 || a->k < 0 || a->hidden < 1 || a->vocab < 1) return PS_ERR_SHAPE;
    if ((a->dtype != PS_F32 && a->dtype != PS_BF16) || !isfinite(a->scale)) return PS_ERR_SHAPE;
    if (a->hidden % (a->dtype == PS_BF16 ? 32 : 16) != 0 || a->hidden > 1 << 16 || a->k > 15) return PS_ERR_UNSUPPORTED;
    if ((long long)a->seqs * a->tokens > 1 << 22 || a->vocab > 1 << 23) return PS_ERR_UNSUPPORTED;
    return PS_OK;
}
bool aligned4(const void* p) { return ((uintptr_t)p & 3) == 0; }

template <typename A> GeParams shape(const A* a) {
    GeParams P = {};
    P.n = a->seqs * a->tokens; P.T = a->tokens; P.k = a->k; P.vocab = a->vocab; P.scale = a->scale;
    P.pieces = a->hidden * (a->dtype == PS_BF16 ? 2 : 4) / 16;
    P.ids = a->token_ids;
    return P;
}

// How the gradients' work is cut, and the workspace: the sorted positions twice, the tokens' ranges, the windows' and the parts' sums
struct GeLayout { size_t keys, sorted, range, part, mask_part, total; };
GeLayout plan(GeParams& P, int dtype) {
    P.chunk_log = 6;
    while (P.chunk_log < GE_CHUNK_LOG && 1 << P.chunk_log < P.n) ++P.chunk_log;
    P.chunks = (P.n + (1 << P.chunk_log) - 1) >> P.chunk_log;
    P.lanes = std::max(1, GE_SORT_THREADS / P.pieces);
    // parts of the groups: some 1024 workgroups (four per compute unit) where every thread still has 8 rows to add up, at most 1024 sums
    const int per = std::max(8 * P.lanes, (int)(((long long)P.n * std::max(P.k, 1) + 1023) / 1024));
    P.part_n = std::max(per, (P.n + 1023 / P.lanes) / std::max(1, 1024 / P.lanes));
    P.parts = (P.n + P.part_n - 1) / P.part_n;
    const size_t row = (size_t)P.pieces * (dtype == PS_BF16 ? 8 : 4) * sizeof(float);
    P.mask_wgs = P.k * (int)((row / 16 + 15) / 16);
    GeLayout L;
    L.keys = 0;
    L.sorted = L.keys + a256((size_t)P.n * 8);
    L.range = L.sorted + a256((size_t)P.n * 8);
    L.part = L.range + a256((size_t)P.vocab * sizeof(int2));
    L.mask_part = L.part + a256((size_t)(P.n + GE_WINDOW - 1) / GE_WINDOW * 2 * row);
    L.total = L.mask_part + a256((size_t)P.k * P.parts * P.lanes * row);
    return L;
}

template <typename WT> int launch_grad(GeParams P, hipStream_t s) {
    const bool mask = P.d_mask && P.k > 0, table = P.d_embed != nullptr;
    const int chunks = P.chunks;
    if (!table) P.chunks = 0;
    if (!mask) P.mask_wgs = 0;
    const dim3 first(P.chunks + (mask ? P.k * P.parts : 0));
    if (!table) hipLaunchKernelGGL((ge_sort_kernel<WT, 0>), first, dim3(GE_SORT_THREADS), 0, s, P);
    else if (P.chunk_log <= GE_SMALL_LOG) hipLaunchKernelGGL((ge_sort_kernel<WT, GE_SMALL_LOG>), first, dim3(GE_SORT_THREADS), 0, s, P);
    else hipLaunchKernelGGL((ge_sort_kernel<WT, GE_CHUNK_LOG>), first, dim3(GE_SORT_THREADS), 0, s, P);
    if (table) {
        if (chunks > 1) {
            hipLaunchKernelGGL(ge_rank_kernel, dim3((P.n + GE_THREADS - 1) / GE_THREADS), dim3(GE_THREADS), 0, s, P);
            hipLaunchKernelGGL(ge_range_kernel, dim3((P.n + GE_THREADS - 1) / GE_THREADS), dim3(GE_THREADS), 0, s, P);
        }
        if (P.n > GE_WINDOW) hipLaunchKernelGGL((ge_window_kernel<WT>), dim3((P.n + GE_WINDOW - 1) / GE_WINDOW, (P.pieces + GE_THREADS - 1) / GE_THREADS), dim3(GE_THREADS), 0, s, P);
    }
    hipLaunchKernelGGL((ge_rows_kernel<WT>), dim3(P.mask_wgs + (table ? P.vocab : 0)), dim3(GE_THREADS), 0, s, P);
    return hipGetLastError() == hipSuccess ? PS_OK : PS_ERR_DEVICE;
}

}   // namespace

extern "C" int ps_group_embed(const ps_group_embed_args* a, void* stream) {
    const int st = check(a);
    if (st != PS_OK) return st;
    if (!a->token_ids || !a->embed || (a->k > 0 && !a->mask_emb) || !a->x) return PS_ERR_NULL;
    if (!aligned4(a->token_ids) || !aligned4(a->embed) || !aligned4(a->mask_emb) || !aligned4(a->x)) return PS_ERR_UNSUPPORTED;
    GeParams P = shape(a);
    P.embed = (const char*)a->embed; P.mask_emb = (const char*)a->mask_emb; P.x = (char*)a->x;
    const dim3 grid(P.n);
    if (a->dtype == PS_BF16) hipLaunchKernelGGL((ge_embed_kernel<bf16_t>), grid, dim3(GE_THREADS), 0, (hipStream_t)stream, P);
    else hipLaunchKernelGGL((ge_embed_kernel<float>), grid, dim3(GE_THREADS), 0, (hipStream_t)stream, P);
    return hipGetLastError() == hipSuccess ? PS_OK : PS_ERR_DEVICE;
}

extern "C" size_t ps_group_embed_grad_workspace_bytes(const ps_group_embed_grad_args* a) {
    if (check(a) != PS_OK) return 0;
    GeParams P = shape(a);
    return plan(P, a->dtype).total;
}

extern "C" int ps_group_embed_grad(const ps_group_embed_grad_args* a, void* stream) {
    const int st = check(a);
    if (st != PS_OK) return st;
    if (!a->token_ids || !a->d_x || !a->workspace || (!a->d_embed && (!a->d_mask || a->k == 0))) return PS_ERR_NULL;
    if (!aligned4(a->token_ids) || !aligned4(a->d_x) || !aligned4(a->d_embed) || !aligned4(a->d_mask)) return PS_ERR_UNSUPPORTED;
    GeParams P = shape(a);
    const GeLayout L = plan(P, a->dtype);
    if (a->workspace_bytes < L.total || ((uintptr_t)a->workspace & 255)) return PS_ERR_WORKSPACE;
    char* ws = (char*)a->workspace;
    P.dx = (const char*)a->d_x; P.d_embed = (char*)a->d_embed; P.d_mask = (char*)a->d_mask;
    P.keys = (u64*)(ws + L.keys); P.sorted = (u64*)(ws + L.sorted); P.range = (int2*)(ws + L.range);
    P.part = (float*)(ws + L.part); P.mask_part = (float*)(ws + L.mask_part);
    return a->dtype == PS_BF16 ? launch_grad<bf16_t>(P, (hipStream_t)stream) : launch_grad<float>(P, (hipStream_t)stream);
}

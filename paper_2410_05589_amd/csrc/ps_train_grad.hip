// Backward pass of the attention of group-wise parallel training (see include/ps_train.h; Section 4.1).
//
// With q~, k~ rotated, s = q~ k~ / sqrt(d), P = exp(s - lse), delta_i = sum_d d_out_i out_i:
//   dP = d_out V^T;  dS = P (dP - delta);  dV = P^T d_out;  dK~ = dS^T q~ / sqrt(d);  dQ~ = dS k~ / sqrt(d), turned back.
// The probabilities are worked out again where they are needed, twice: by workgroups that own query rows (gb_dq_kernel) and by
// workgroups that own keys (gb_dkv_kernel: real tokens; gb_own_kernel: [MASK] tokens, which only their own group's rows see).
// Nobody adds to what another writes: no atomics, the same bits every time.  That is 7 products where one pass would do with 5.
//
// All products are 32 x 32 MFMA tiles, as in ga_attn_wide_kernel: what the wavefront owns (queries, or keys) lies along the lanes,
// so a score tile leaves the matrix core in the operand layout of the products that follow it (a lane holds 16 of the 32 rows of the other
// side for its own query or key; the contraction may take them in any order as long as both operands do).  -lse and
// -delta are the accumulators' initial values.  The other side's rows are staged in LDS once per workgroup and read both ways: as rows
// (scores) and as columns (gradients; bf16: transposed by the LDS unit).
#include "ps_train_device.h"

namespace {

constexpr int GB_THREADS = 256, GB_WAVES = GB_THREADS / 64, GB_ROWS = 32 * GB_WAVES;   // rows, or keys, of a workgroup

struct GbParams {
    int seqs, T, k, nq, nkv, rows, group, gpt;   // gpt: groups that fit into 32 rows
    unsigned k1_magic;    // (as GaParams has it)
    float inv_sqrt_d;
    double log2_base;
    const char *q, *k_, *v, *d_out;
    const float *out, *lse;
    char *d_q, *d_k, *d_v;
    float2* table;        // [T + k][d / 2] cosines and sines
    char* k_rot;          // [seqs][nkv][rows][d], storage type
    char* q_rot;          // [parts][seqs][nq][rows][d], storage type: times log2(e) / sqrt(d); bf16: high parts, low parts
    float2* stats;        // [seqs][nq][rows]: -lse / ln 2, -delta
};
template <typename WT> struct GbTraits { static constexpr int PARTS = Traits<WT>::BF ? 2 : 1; };

__device__ __forceinline__ int gb_group(const GbParams& P, int row) { return P.k > 0 ? (int)__umulhi((unsigned)row, P.k1_magic) : row; }

// ---- the table, rotated q and k, and the rows' statistics; a workgroup takes one position (as ga_rope_kernel)
template <typename WT, int D>
__global__ void __launch_bounds__(256) gb_prep_kernel(const GbParams P) {
    constexpr int ESZ = Traits<WT>::ESZ, Q4 = D / 8;
    __shared__ float2 cs[D / 2];
    const int pos = blockIdx.x, tid = threadIdx.x;
    if (tid < D / 2) {
        const float2 t = ga_cos_sin((double)pos * ga_exp2(-2.0 * tid / D * P.log2_base));
        cs[tid] = t;
        if (blockIdx.y == 0) P.table[(size_t)pos * (D / 2) + tid] = t;
    }
    __syncthreads();
    const int s0 = max(0, pos - P.T + 1), slots = min(pos, P.k) - s0 + 1, g4 = tid % Q4;
    auto turn = [&](f32x4 a, f32x4 b, float scale, f32x4& ra, f32x4& rb) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 t = cs[4 * g4 + e];
            ra[e] = (a[e] * t.x - b[e] * t.y) * scale;
            rb[e] = (b[e] * t.x + a[e] * t.y) * scale;
        }
    };
    const long long nk = (long long)slots * P.seqs * P.nkv * Q4, nq = (long long)slots * P.seqs * P.nq * Q4;
    for (long long x = (long long)blockIdx.y * 256 + tid; x < nk; x += (long long)gridDim.y * 256) {
        const unsigned y = (unsigned)(x / Q4), z = y / P.nkv, head = y - z * P.nkv, slot = z / P.seqs, seq = z - slot * P.seqs;
        const int sl = s0 + (int)slot;
        const size_t row = (size_t)(pos - sl) * (P.k + 1) + sl;
        const char* p = P.k_ + ((((size_t)seq * P.rows + row) * P.nkv + head) * D + 4 * g4) * ESZ;
        f32x4 ra, rb;
        turn(load4_q<WT>(p), load4_q<WT>(p + D / 2 * ESZ), 1.f, ra, rb);
        char* o = P.k_rot + ((((size_t)seq * P.nkv + head) * P.rows + row) * D + 4 * g4) * ESZ;
        store4<WT>(o, ra);
        store4<WT>(o + D / 2 * ESZ, rb);
    }
    const size_t part = (size_t)P.seqs * P.nq * P.rows * D * ESZ;
    for (long long x = (long long)blockIdx.y * 256 + tid; x < nq; x += (long long)gridDim.y * 256) {
        const unsigned y = (unsigned)(x / Q4), z = y / P.nq, head = y - z * P.nq, slot = z / P.seqs, seq = z - slot * P.seqs;
        const int sl = s0 + (int)slot;
        const size_t row = (size_t)(pos - sl) * (P.k + 1) + sl;
        const size_t at = ((size_t)seq * P.rows + row) * P.nq + head, from = at * D + 4 * g4;
        f32x4 ra, rb;
        turn(load4_q<WT>(P.q + from * ESZ), load4_q<WT>(P.q + (from + D / 2) * ESZ), P.inv_sqrt_d * 1.4426950408889634f, ra, rb);
        const size_t to = ((size_t)seq * P.nq + head) * P.rows + row;
        char* o = P.q_rot + (to * D + 4 * g4) * ESZ;
        const f32x4 ha = store4<WT>(o, ra), hb = store4<WT>(o + D / 2 * ESZ, rb);
        if constexpr (Traits<WT>::BF) {
            store4<WT>(o + part, ra - ha);
            store4<WT>(o + part + D / 2 * ESZ, rb - hb);
        }
        const f32x4 oa = load4_q<float>(P.out + from), ob = load4_q<float>(P.out + from + D / 2);
        const f32x4 da = load4_q<WT>(P.d_out + from * ESZ), db = load4_q<WT>(P.d_out + (from + D / 2) * ESZ);
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += oa[e] * da[e] + ob[e] * db[e];
#pragma unroll
        for (int m = Q4 / 2; m >= 1; m >>= 1) sum += __shfl_xor(sum, m, 64);
        if (g4 == 0) P.stats[to] = make_float2(-P.lse[at] * 1.4426950408889634f, -sum);
    }
}

// ------------------------------------------------------------------------------------------
// Tiles of 32 rows in LDS, read as rows (16 bytes of lane c's row) and as columns.  Within a row, 32-byte chunks stand at
// chunk ^ f(row): rows read together, and the four or eight rows of a column read, fall into different banks.
// ------------------------------------------------------------------------------------------
template <typename WT, int D> struct GbTile {
    static constexpr int ESZ = Traits<WT>::ESZ, ROWB = D * ESZ, BYTES = 32 * ROWB, STEPS = ROWB / 32, NJ = D / 32;
    static constexpr bool BF = Traits<WT>::BF;
    static constexpr int U = BYTES / (GB_THREADS * 16), PPR = ROWB / 16;   // 16-byte pieces per thread, per row
    static constexpr int WU = BYTES / (64 * 16);                           // ... per lane of a single wavefront
    static __device__ __forceinline__ int f(int row) { return ROWB == 128 ? (row >> 1) & 3 : row & 7; }
    static __device__ __forceinline__ int at(int row, int piece) { return row * ROWB + (((piece >> 1) ^ f(row)) << 5) + (piece & 1) * 16; }

    int rd, cd;           // this lane's places: of its row (chunk 0), of its column (tile 0, keys 0 ..)
    __device__ __forceinline__ GbTile(int lane) {
        const int c = lane & 31, half = lane >> 5;
        rd = at(c, half);
        if constexpr (BF) {
            const int row = 4 * half + ((lane & 15) >> 2), vhi = (lane >> 4) & 1;
            cd = row * ROWB + ((vhi ^ f(row)) << 5) + (lane & 3) * 8;
        } else {
            cd = 4 * half * ROWB + (((c >> 3) ^ (4 * half)) << 5) + (c & 7) * 4;
        }
    }
    // 16 bytes of the lane's row: step st's operand
    __device__ __forceinline__ uint4 row(const char* tile, int st) const { return ld16(tile + (rd ^ (st << 5))); }
    // columns 32 j + c, rows 16 m + 4 half + {0..3, 8..11} (bf16); with clean, values that are not finite count as zero
    template <bool CLEAN> __device__ __forceinline__ bf16x8 column(const char* tile, int j, int m) const {
        const char* a = tile + m * 16 * ROWB + (cd ^ (j << 6));
        const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)a);
        const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(a + 8 * ROWB));
        u32x4 v = __builtin_bit_cast(u32x4, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
        if constexpr (CLEAN) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] = (v[e] & 0x7F80u) == 0x7F80u ? v[e] & 0xFFFF0000u : v[e];
                v[e] = (v[e] & 0x7F800000u) == 0x7F800000u ? v[e] & 0xFFFFu : v[e];
            }
        }
        return __builtin_bit_cast(bf16x8, v);
    }
    // column 32 j + c of row 8 (i / 4) + i % 4 + 4 half (float32)
    template <bool CLEAN> __device__ __forceinline__ float element(const char* tile, int j, int i) const {
        const float v = *reinterpret_cast<const float*>(tile + (8 * (i / 4) + i % 4) * ROWB + (cd ^ (j << 7) ^ ((i & 3) << 5)));
        return !CLEAN || fabsf(v) < INFINITY ? v : 0.f;
    }
};

// scores += rows . own: the lane's i-th is that of row 8 (i / 4) + i % 4 + 4 half and the lane's own query or key
template <typename WT, int D>
__device__ __forceinline__ void gb_scores(const GbTile<WT, D>& L, const char* tile, const uint4 (&own)[GbTile<WT, D>::STEPS], f32x16& x) {
#pragma unroll
    for (int st = 0; st < GbTile<WT, D>::STEPS; ++st) {
        const uint4 a = L.row(tile, st);
        if constexpr (Traits<WT>::BF) {
            x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, own[st]), x, 0, 0, 0);
        } else {
            const f32x4 u = __builtin_bit_cast(f32x4, a), w = __builtin_bit_cast(f32x4, own[st]);
#pragma unroll
            for (int e = 0; e < 4; ++e) x = __builtin_amdgcn_mfma_f32_32x32x2f32(u[e], w[e], x, 0, 0, 0);
        }
    }
}
// y^T += rows^T . p, p as gb_scores leaves it
template <typename WT, int D, bool CLEAN>
__device__ __forceinline__ void gb_products(const GbTile<WT, D>& L, const char* tile, const f32x16& p, f32x16 (&y)[D / 32]) {
    if constexpr (Traits<WT>::BF) {
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            uint4 b;
            b.x = pack_bf16x2(p[8 * m], p[8 * m + 1]);
            b.y = pack_bf16x2(p[8 * m + 2], p[8 * m + 3]);
            b.z = pack_bf16x2(p[8 * m + 4], p[8 * m + 5]);
            b.w = pack_bf16x2(p[8 * m + 6], p[8 * m + 7]);
#pragma unroll
            for (int j = 0; j < D / 32; ++j)
                y[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(L.template column<CLEAN>(tile, j, m), __builtin_bit_cast(bf16x8, b), y[j], 0, 0, 0);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
            for (int j = 0; j < D / 32; ++j) y[j] = __builtin_amdgcn_mfma_f32_32x32x2f32(L.template element<CLEAN>(tile, j, i), p[i], y[j], 0, 0, 0);
    }
}
// rows first + (own thread's) .. of a matrix with `stride` bytes between rows, rows beyond lo .. hi replaced by the nearest
template <typename WT, int D, int THREADS, int U>
__device__ __forceinline__ void gb_load(const char* base, size_t stride, int first, int step, int lo, int hi, int t, uint4 (&x)[U]) {
    constexpr int PPR = GbTile<WT, D>::PPR;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i = t + THREADS * u, row = min(max(first + i / PPR, lo), hi) * step;
        x[u] = ld16_q(base + (size_t)(unsigned)row * stride + (i % PPR) * 16);
    }
}
template <typename WT, int D, int THREADS, int U>
__device__ __forceinline__ void gb_store(char* tile, int t, const uint4 (&x)[U]) {
    constexpr int PPR = GbTile<WT, D>::PPR;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int i = t + THREADS * u;
        *reinterpret_cast<uint4*>(tile + GbTile<WT, D>::at(i / PPR, i % PPR)) = x[u];
    }
}
// a lane's row as operand, straight from memory
template <typename WT, int D> __device__ __forceinline__ void gb_own_rows(const char* row, int half, uint4 (&x)[GbTile<WT, D>::STEPS]) {
#pragma unroll
    for (int st = 0; st < GbTile<WT, D>::STEPS; ++st) x[st] = ld16_q(row + st * 32 + half * 16);
}
// the lane's row of a gradient, y[j][i] = column 32 j + 8 (i / 4) + 4 half + i % 4, times scale; with turn, rotated back
template <typename WT, int D>
__device__ __forceinline__ void gb_write(char* row, const float2* turn, float scale, int half, const f32x16 (&y)[D / 32]) {
    constexpr int ESZ = Traits<WT>::ESZ, NJ = D / 32;
#pragma unroll
    for (int j = 0; j < NJ / 2; ++j)
#pragma unroll
        for (int i4 = 0; i4 < 4; ++i4) {
            f32x4 a, b;
            const int col = 32 * j + 8 * i4 + 4 * half;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                a[e] = y[j][4 * i4 + e] * scale;
                b[e] = y[j + NJ / 2][4 * i4 + e] * scale;
            }
            if (turn) {
                const f32x4 t0 = *reinterpret_cast<const f32x4*>(turn + col), t1 = *reinterpret_cast<const f32x4*>(turn + col + 2);
                const float c[4] = {t0[0], t0[2], t1[0], t1[2]}, s[4] = {t0[1], t0[3], t1[1], t1[3]};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = a[e];
                    a[e] = x * c[e] + b[e] * s[e];
                    b[e] = b[e] * c[e] - x * s[e];
                }
            }
            if constexpr (Traits<WT>::BF) {
                *reinterpret_cast<u32x2_q*>(row + col * ESZ) = (u32x2_q)u32x2{pack_bf16x2(a[0], a[1]), pack_bf16x2(a[2], a[3])};
                *reinterpret_cast<u32x2_q*>(row + (col + D / 2) * ESZ) = (u32x2_q)u32x2{pack_bf16x2(b[0], b[1]), pack_bf16x2(b[2], b[3])};
            } else {
                *reinterpret_cast<f32x4_q*>(row + col * ESZ) = (f32x4_q)a;
                *reinterpret_cast<f32x4_q*>(row + (col + D / 2) * ESZ) = (f32x4_q)b;
            }
        }
}

// ------------------------------------------------------------------------------------------
// Gradients of the queries: 128 layout rows per workgroup, 32 per wavefront.  Key tiles: the layout rows R0 - 32 .. R0 + 127, among
// which the queries see their own groups' [MASK] rows, then the real tokens up to the last group.
// ------------------------------------------------------------------------------------------
template <typename WT, int D>
__global__ void __launch_bounds__(GB_THREADS) gb_dq_kernel(const GbParams P) {
    typedef GbTile<WT, D> Tile;
    constexpr int ESZ = Traits<WT>::ESZ, PARTS = GbTraits<WT>::PARTS, NJ = D / 32, BUF = 2 * Tile::BYTES;
    __shared__ __attribute__((aligned(16))) char smem[2 * BUF];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, half = lane >> 5;
    const int K1 = P.k + 1, blk = gridDim.x - 1 - blockIdx.x, h = blockIdx.y, seq = blockIdx.z, hk = h / P.group;
    const int R0 = GB_ROWS * blk, r0 = R0 + 32 * wave, r_last = min(R0 + GB_ROWS, P.rows) - 1, g_last = gb_group(P, r_last);
    const bool active = r0 < P.rows;
    const int n_own = P.k > 0 ? GB_WAVES + 1 : 0, n_tiles = n_own + g_last / 32 + 1;
    const int qrow = min(r0 + c, r_last), qg = gb_group(P, qrow), w_first = min(r0, r_last), wg0 = gb_group(P, w_first), wg1 = gb_group(P, min(r0 + 31, r_last));
    const Tile L(lane);
    const char* krows = P.k_rot + ((size_t)seq * P.nkv + hk) * P.rows * D * ESZ;
    const char* vrows = P.v + ((size_t)seq * P.rows * P.nkv + hk) * D * ESZ;
    const size_t vstride = (size_t)P.nkv * D * ESZ;
    uint4 sk[Tile::U], sv[Tile::U];
    auto load = [&](int t) __attribute__((always_inline)) {
        const bool own = t < n_own;
        const int first = own ? R0 - 32 + 32 * t : 32 * (t - n_own), hi = own ? r_last : g_last, step = own ? 1 : K1;
        gb_load<WT, D, GB_THREADS>(krows, (size_t)D * ESZ, first, step, 0, hi, tid, sk);
        gb_load<WT, D, GB_THREADS>(vrows, vstride, first, step, 0, hi, tid, sv);
    };
    auto store = [&](int t) __attribute__((always_inline)) {
        gb_store<WT, D, GB_THREADS>(smem + (t & 1) * BUF, tid, sk);
        gb_store<WT, D, GB_THREADS>(smem + (t & 1) * BUF + Tile::BYTES, tid, sv);
    };
    load(0);
    const size_t qat = ((size_t)seq * P.nq + h) * P.rows + qrow, part = (size_t)P.seqs * P.nq * P.rows * D * ESZ;
    uint4 q[PARTS][Tile::STEPS], d_o[Tile::STEPS];
#pragma unroll
    for (int p = 0; p < PARTS; ++p) gb_own_rows<WT, D>(P.q_rot + p * part + qat * D * ESZ, half, q[p]);
    gb_own_rows<WT, D>(P.d_out + (((size_t)seq * P.rows + qrow) * P.nq + h) * D * ESZ, half, d_o);
    const float2 st = P.stats[qat];
    f32x16 y[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i) y[j][i] = 0.f;
    store(0);
    if (n_tiles > 1) load(1);
    __syncthreads();
    for (int t = 0; t < n_tiles; ++t) {
        if (t + 1 < n_tiles) store(t + 1);
        if (t + 2 < n_tiles) load(t + 2);
        const char *kt = smem + (t & 1) * BUF, *vt = kt + Tile::BYTES;
        const bool own = t < n_own;
        const int first = own ? R0 - 32 + 32 * t : 32 * (t - n_own);
        // (own rows: the wavefront's own tile and, where its first row is not the first of its group, the one before)
        const bool busy = active && (own ? t == wave + 1 || (t == wave && wg0 * K1 != r0) : first <= wg1);
        if (busy) {
            f32x16 s, dp;
#pragma unroll
            for (int i = 0; i < 16; ++i) { s[i] = st.x; dp[i] = st.y; }
#pragma unroll
            for (int p = 0; p < PARTS; ++p) gb_scores<WT, D>(L, kt, q[p], s);
            gb_scores<WT, D>(L, vt, d_o, dp);
            if (!own && first + 31 <= wg0) {
#pragma unroll
                for (int i = 0; i < 16; ++i) s[i] = __builtin_amdgcn_exp2f(s[i]) * dp[i];
                gb_products<WT, D, false>(L, kt, s, y);
            } else {
                const int lo = (own ? qg * K1 + 1 : 0) - first - 4 * half, hi = (own ? qrow : qg) - first - 4 * half;
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int key = 8 * (i / 4) + i % 4;
                    s[i] = key >= lo && key <= hi ? __builtin_amdgcn_exp2f(s[i]) * dp[i] : 0.f;
                }
                gb_products<WT, D, true>(L, kt, s, y);
            }
        }
        __syncthreads();
    }
    if (r0 + c < P.rows)
        gb_write<WT, D>(P.d_q + (((size_t)seq * P.rows + qrow) * P.nq + h) * D * ESZ, P.table + (size_t)(qrow - qg * P.k) * (D / 2), P.inv_sqrt_d, half, y);
}

// ------------------------------------------------------------------------------------------
// A wavefront's 32 keys: their rows as operands, their gradients; one tile of 32 query rows at a time.
// ------------------------------------------------------------------------------------------
template <typename WT, int D> struct GbKeys {
    typedef GbTile<WT, D> Tile;
    static constexpr int PARTS = GbTraits<WT>::PARTS, NJ = D / 32;
    uint4 kf[Tile::STEPS], vf[Tile::STEPS];
    f32x16 dk[NJ], dv[NJ];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) { dk[j][i] = 0.f; dv[j][i] = 0.f; }
    }
    // buf: the tiles of the rotated queries' parts, then of d_out; stats: the rows' (-lse / ln 2, -delta); the lane's key is seen by
    // rows lo .. hi of the tile (counted from 4 half), all of them if not masked
    template <bool MASKED> __device__ __forceinline__ void step(const Tile& L, const char* buf, const float2* stats, int half, int lo, int hi) {
        f32x16 s, dp;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float2 x = stats[8 * (i / 4) + i % 4 + 4 * half];
            s[i] = x.x;
            dp[i] = x.y;
        }
#pragma unroll
        for (int p = 0; p < PARTS; ++p) gb_scores<WT, D>(L, buf + p * Tile::BYTES, kf, s);
        const char* dt = buf + PARTS * Tile::BYTES;
        gb_scores<WT, D>(L, dt, vf, dp);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int row = 8 * (i / 4) + i % 4;
            const bool in = !MASKED || (row >= lo && row <= hi);
            const float p = in ? __builtin_amdgcn_exp2f(s[i]) : 0.f;
            s[i] = p;
            dp[i] = in ? p * dp[i] : 0.f;
        }
        gb_products<WT, D, MASKED>(L, dt, s, dv);
#pragma unroll
        for (int p = 0; p < PARTS; ++p) gb_products<WT, D, MASKED>(L, buf + p * Tile::BYTES, dp, dk);
    }
    __device__ __forceinline__ void write(const GbParams& P, int seq, int hk, int row, int pos, int half) const {
        const size_t at = (((size_t)seq * P.rows + row) * P.nkv + hk) * D * Traits<WT>::ESZ;
        gb_write<WT, D>(P.d_k + at, P.table + (size_t)pos * (D / 2), 0.6931471805599453f, half, dk);   // (the queries carry log2(e) / sqrt(d))
        gb_write<WT, D>(P.d_v + at, nullptr, 1.f, half, dv);
    }
};

// Gradients of real tokens' keys and values: 128 tokens per workgroup, 32 per wavefront, and all rows from the first token's group on,
// of every query head that shares the kv head.
template <typename WT, int D>
__global__ void __launch_bounds__(GB_THREADS) gb_dkv_kernel(const GbParams P) {
    typedef GbTile<WT, D> Tile;
    constexpr int ESZ = Traits<WT>::ESZ, PARTS = GbTraits<WT>::PARTS, OFF_S = (PARTS + 1) * Tile::BYTES, BUF = OFF_S + 32 * 8;
    __shared__ __attribute__((aligned(16))) char smem[2 * BUF];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, half = lane >> 5;
    const int K1 = P.k + 1, hk = blockIdx.y, seq = blockIdx.z;
    const int t0 = GB_ROWS * blockIdx.x, w0 = t0 + 32 * wave, key = min(w0 + c, P.T - 1);
    const int first_row = t0 * K1, per_head = (P.rows - first_row + 31) / 32, n_tiles = per_head * P.group;
    const Tile L(lane);
    const size_t part = (size_t)P.seqs * P.nq * P.rows * D * ESZ, ostride = (size_t)P.nq * D * ESZ;
    uint4 sq[PARTS][Tile::U], so[Tile::U];
    float2 ss;
    int load_head = 0, load_tile = 0;
    auto load = [&]() __attribute__((always_inline)) {       // the next tile, head by head
        const int h = hk * P.group + load_head, first = first_row + 32 * load_tile;
        const size_t at = ((size_t)seq * P.nq + h) * P.rows;
#pragma unroll
        for (int p = 0; p < PARTS; ++p) gb_load<WT, D, GB_THREADS>(P.q_rot + p * part + at * D * ESZ, (size_t)D * ESZ, first, 1, 0, P.rows - 1, tid, sq[p]);
        gb_load<WT, D, GB_THREADS>(P.d_out + ((size_t)seq * P.rows * P.nq + h) * D * ESZ, ostride, first, 1, 0, P.rows - 1, tid, so);
        ss = P.stats[at + min(first + (tid & 31), P.rows - 1)];
        if (++load_tile == per_head) { load_tile = 0; ++load_head; }
    };
    auto store = [&](int t) __attribute__((always_inline)) {
        char* b = smem + (t & 1) * BUF;
#pragma unroll
        for (int p = 0; p < PARTS; ++p) gb_store<WT, D, GB_THREADS>(b + p * Tile::BYTES, tid, sq[p]);
        gb_store<WT, D, GB_THREADS>(b + PARTS * Tile::BYTES, tid, so);
        if (tid < 32) *reinterpret_cast<float2*>(b + OFF_S + tid * 8) = ss;
    };
    load();
    GbKeys<WT, D> keys;
    gb_own_rows<WT, D>(P.k_rot + (((size_t)seq * P.nkv + hk) * P.rows + (size_t)key * K1) * D * ESZ, half, keys.kf);
    gb_own_rows<WT, D>(P.v + (((size_t)seq * P.rows + (size_t)key * K1) * P.nkv + hk) * D * ESZ, half, keys.vf);
    keys.clear();
    store(0);
    if (n_tiles > 1) load();
    __syncthreads();
    int tile = 0;
    for (int t = 0; t < n_tiles; ++t) {
        if (t + 1 < n_tiles) store(t + 1);
        if (t + 2 < n_tiles) load();
        const char* buf = smem + (t & 1) * BUF;
        const int first = first_row + 32 * tile;
        if (w0 < P.T && first + 31 >= w0 * K1) {
            if (first >= (w0 + 31) * K1 && first + 31 < P.rows)
                keys.template step<false>(L, buf, reinterpret_cast<const float2*>(buf + OFF_S), half, 0, 31);
            else
                keys.template step<true>(L, buf, reinterpret_cast<const float2*>(buf + OFF_S), half, key * K1 - first - 4 * half, P.rows - 1 - first - 4 * half);
        }
        if (++tile == per_head) tile = 0;
        __syncthreads();
    }
    if (w0 + c < P.T) keys.write(P, seq, hk, key * K1, key, half);
}

// Gradients of [MASK] tokens' keys and values, which the later rows of their own group see: a wavefront takes as many whole groups as
// fit into 32 rows, every query head that shares the kv head in turn.
template <typename WT, int D>
__global__ void __launch_bounds__(64) gb_own_kernel(const GbParams P) {
    typedef GbTile<WT, D> Tile;
    constexpr int ESZ = Traits<WT>::ESZ, PARTS = GbTraits<WT>::PARTS, OFF_S = (PARTS + 1) * Tile::BYTES;
    __shared__ __attribute__((aligned(16))) char smem[OFF_S + 32 * 8];
    const int lane = threadIdx.x, c = lane & 31, half = lane >> 5;
    const int K1 = P.k + 1, hk = blockIdx.y, seq = blockIdx.z, first = blockIdx.x * P.gpt * K1, last = min(first + P.gpt * K1, P.rows) - 1;
    const int krow = min(first + c, last), g = gb_group(P, krow), slot = krow - g * K1;
    const Tile L(lane);
    const size_t part = (size_t)P.seqs * P.nq * P.rows * D * ESZ, ostride = (size_t)P.nq * D * ESZ;
    GbKeys<WT, D> keys;
    gb_own_rows<WT, D>(P.k_rot + (((size_t)seq * P.nkv + hk) * P.rows + krow) * D * ESZ, half, keys.kf);
    gb_own_rows<WT, D>(P.v + (((size_t)seq * P.rows + krow) * P.nkv + hk) * D * ESZ, half, keys.vf);
    keys.clear();
    for (int i = 0; i < P.group; ++i) {
        const int h = hk * P.group + i;
        const size_t at = ((size_t)seq * P.nq + h) * P.rows;
        uint4 x[Tile::WU];
        __syncthreads();
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            gb_load<WT, D, 64>(P.q_rot + p * part + at * D * ESZ, (size_t)D * ESZ, first, 1, 0, last, lane, x);
            gb_store<WT, D, 64>(smem + p * Tile::BYTES, lane, x);
        }
        gb_load<WT, D, 64>(P.d_out + ((size_t)seq * P.rows * P.nq + h) * D * ESZ, ostride, first, 1, 0, last, lane, x);
        gb_store<WT, D, 64>(smem + PARTS * Tile::BYTES, lane, x);
        if (lane < 32) *reinterpret_cast<float2*>(smem + OFF_S + lane * 8) = P.stats[at + krow];
        __syncthreads();
        keys.template step<true>(L, smem, reinterpret_cast<const float2*>(smem + OFF_S), half, slot > 0 ? krow - first - 4 * half : 99, g * K1 + P.k - first - 4 * half);
    }
    if (first + c <= last && slot > 0) keys.write(P, seq, hk, krow, krow - g * P.k, half);
}

// the checks are those of ps_group_attention
ps_group_attn_args forward_args(const ps_group_attn_grad_args* a) {
    ps_group_attn_args f = {};
    f.seqs = a->seqs; f.tokens = a->tokens; f.k = a->k; f.n_heads = a->n_heads; f.n_kv_heads = a->n_kv_heads;
    f.head_dim = a->head_dim; f.dtype = a->dtype; f.rope_base = a->rope_base;
    return f;
}
int check(const ps_group_attn_grad_args* a) {
    if (!a) return PS_ERR_NULL;
    const ps_group_attn_args f = forward_args(a);
    return ga_check(&f);
}

struct GbLayout { size_t table, k_rot, q_rot, stats, total; };
GbLayout layout(const ps_group_attn_grad_args* a) {
    GbLayout L;
    const bool bf = a->dtype == PS_BF16;
    const size_t rows = (size_t)a->seqs * a->tokens * (a->k + 1), row = (size_t)a->head_dim * (bf ? 2 : 4);
    L.table = 0;
    L.k_rot = a256((size_t)(a->tokens + a->k) * (a->head_dim / 2) * sizeof(float2));
    L.q_rot = L.k_rot + a256(rows * a->n_kv_heads * row);
    L.stats = L.q_rot + a256(rows * a->n_heads * row * (bf ? 2 : 1));
    L.total = L.stats + a256(rows * a->n_heads * sizeof(float2));
    return L;
}

template <typename WT, int D> int launch(const GbParams& P, hipStream_t s) {
    // (as ga_rope_kernel: where positions are few, several workgroups of at most one item per thread share one)
    const long long items = (long long)P.seqs * P.nq * (D / 8) * (P.k + 1);
    const unsigned share = (unsigned)std::max(1LL, std::min((items + 255) / 256, 4096LL / (P.T + P.k)));
    hipLaunchKernelGGL((gb_prep_kernel<WT, D>), dim3(P.T + P.k, share), dim3(256), 0, s, P);
    hipLaunchKernelGGL((gb_dq_kernel<WT, D>), dim3((P.rows + GB_ROWS - 1) / GB_ROWS, P.nq, P.seqs), dim3(GB_THREADS), 0, s, P);
    hipLaunchKernelGGL((gb_dkv_kernel<WT, D>), dim3((P.T + GB_ROWS - 1) / GB_ROWS, P.nkv, P.seqs), dim3(GB_THREADS), 0, s, P);
    if (P.k > 0) hipLaunchKernelGGL((gb_own_kernel<WT, D>), dim3((P.T + P.gpt - 1) / P.gpt, P.nkv, P.seqs), dim3(64), 0, s, P);
    return hipGetLastError() == hipSuccess ? PS_OK : PS_ERR_DEVICE;
}

}   // namespace

extern "C" size_t ps_group_attention_grad_workspace_bytes(const ps_group_attn_grad_args* a) { return check(a) == PS_OK ? layout(a).total : 0; }

extern "C" int ps_group_attention_grad(const ps_group_attn_grad_args* a, void* stream) {
    const int st = check(a);
    if (st != PS_OK) return st;
    if (!a->q || !a->k_ || !a->v || !a->out || !a->lse || !a->d_out || !a->d_q || !a->d_k || !a->d_v || !a->workspace) return PS_ERR_NULL;
    const GbLayout L = layout(a);
    if (a->workspace_bytes < L.total || ((uintptr_t)a->workspace & 255)) return PS_ERR_WORKSPACE;
    char* ws = (char*)a->workspace;
    GbParams P = {};
    P.seqs = a->seqs; P.T = a->tokens; P.k = a->k; P.nq = a->n_heads; P.nkv = a->n_kv_heads;
    P.rows = a->tokens * (a->k + 1);
    P.group = P.nq / P.nkv;
    P.gpt = 32 / (a->k + 1);
    P.k1_magic = (unsigned)((0x100000000ull + a->k) / (unsigned)(a->k + 1));
    P.inv_sqrt_d = (float)(1.0 / sqrt((double)a->head_dim));
    P.log2_base = log2((double)a->rope_base);
    P.q = (const char*)a->q; P.k_ = (const char*)a->k_; P.v = (const char*)a->v; P.d_out = (const char*)a->d_out;
    P.out = a->out; P.lse = a->lse;
    P.d_q = (char*)a->d_q; P.d_k = (char*)a->d_k; P.d_v = (char*)a->d_v;
    P.table = (float2*)(ws + L.table); P.k_rot = ws + L.k_rot; P.q_rot = ws + L.q_rot; P.stats = (float2*)(ws + L.stats);
    hipStream_t s = (hipStream_t)stream;
    if (a->dtype == PS_BF16) return a->head_dim == 128 ? launch<bf16_t, 128>(P, s) : launch<bf16_t, 64>(P, s);
    return a->head_dim == 128 ? launch<float, 128>(P, s) : launch<float, 64>(P, s);
}

// Backward pass of the attention of group-wise parallel training (see include/ps_train.h; Section 4.1).
//
// With q~, k~ rotated, s = q~ k~ / sqrt(d), P = exp(s - lse), delta_i = sum_d d_out_i out_i:
//   dP = d_out V^T;  dS = P (dP - delta);  dV = P^T d_out;  dK~ = dS^T q~ / sqrt(d);  dQ~ = dS k~ / sqrt(d), turned back.
// The probabilities are worked out again where they are needed, twice: by workgroups that own query rows (gb_dq_kernel) and by
// workgroups that own keys (gb_dkv_kernel: real tokens, and [MASK] tokens, which only their own group's rows see).
// Nobody adds to what another writes: no atomics, the same bits every time.  That is 7 products where one pass would do with 5, and 10 in bf16,
// where the rotated queries stand as two parts (scores twice, dK~), as in the forward pass whose lse they have to match.
//
// Bound by the matrix cores, by waits beside them and, for the [MASK] keys, by memory: T 2048, k 4, 32 heads x 128 takes 1036 .. 1063 us (5 products
// at the rate of a large library product: 327; the 10: 654), of which keys 640 .. 710 ([MASK] keys 110), queries 395 .. 430, rotated keys 30; 4 x T 1024,
// k 8, 32 / 8 heads 2320; T 203, k 5, 40 heads 104 (112 with other calls in between); float32 2 x T 300, k 3, 8 heads x 64 84.
//
// All products are 32 x 32 MFMA tiles, as in ga_attn_wide_kernel: what the wavefront owns (queries, or keys) lies along the lanes,
// so a score tile leaves the matrix core in the operand layout of the products that follow it (a lane holds 16 of the 32 rows of the other
// side for its own query or key; the contraction may take them in any order as long as both operands do).  -lse and
// -delta are the accumulators' initial values.  The other side's rows are staged in LDS once per workgroup and read both ways: as rows
// (scores) and as columns (gradients; bf16: transposed by the LDS unit).
#include "ps_train_device.h"
#include "ps_draft_debug.h"

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
    float *lse2, *delta;  // [seqs][nq][rows]: -lse / ln 2, -sum of d_out out
};
template <typename WT> struct GbTraits { static constexpr int PARTS = Traits<WT>::BF ? 2 : 1; };

__device__ __forceinline__ int gb_group(const GbParams& P, int row) { return P.k > 0 ? (int)__umulhi((unsigned)row, P.k1_magic) : row; }

// ---- the table and the rotated keys; a workgroup takes one position (as ga_rope_kernel, whose keys lie otherwise)
template <typename WT, int D>
__global__ void __launch_bounds__(256) gb_prep_kernel(const GbParams P) {
    constexpr int ESZ = Traits<WT>::ESZ, Q4 = D / 8;
    __shared__ float2 cs[D / 2];
    const int pos = blockIdx.x, tid = threadIdx.x, g4 = tid % Q4;
    const int s0 = max(0, pos - P.T + 1), slots = min(pos, P.k) - s0 + 1;
    const long long n = (long long)slots * P.seqs * P.nkv * Q4;
    char* to = nullptr;
    f32x4 a, b;
    auto request = [&](long long x) __attribute__((always_inline)) {
        const unsigned y = (unsigned)(x / Q4), z = y / P.nkv, head = y - z * P.nkv, slot = z / P.seqs, seq = z - slot * P.seqs;
        const int sl = s0 + (int)slot;
        const size_t row = (size_t)(pos - sl) * (P.k + 1) + sl;
        const char* p = P.k_ + ((((size_t)seq * P.rows + row) * P.nkv + head) * D + 4 * g4) * ESZ;
        to = P.k_rot + ((((size_t)seq * P.nkv + head) * P.rows + row) * D + 4 * g4) * ESZ;
        a = load4_q<WT>(p);
        b = load4_q<WT>(p + D / 2 * ESZ);
    };
    long long x = (long long)blockIdx.y * 256 + tid;
    if (x < n) request(x);                                  // (on its way while the table is worked out)
    if (tid < D / 2) {
        const float2 t = ga_cos_sin((double)pos * ga_exp2(-2.0 * tid / D * P.log2_base));
        cs[tid] = t;
        if (blockIdx.y == 0) P.table[(size_t)pos * (D / 2) + tid] = t;
    }
    __syncthreads();
    while (x < n) {
        f32x4 ra, rb;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float2 t = cs[4 * g4 + e];
            ra[e] = a[e] * t.x - b[e] * t.y;
            rb[e] = b[e] * t.x + a[e] * t.y;
        }
        store4<WT>(to, ra);
        store4<WT>(to + D / 2 * ESZ, rb);
        x += (long long)gridDim.y * 256;
        if (x < n) request(x);
    }
}

// ------------------------------------------------------------------------------------------
// Tiles of 32 rows in LDS, read as rows (16 bytes of lane c's row) and as columns.  A tile is cut into blocks of 64 bytes of
// every row, row behind row; 16-byte piece i of a row's 64 bytes stands at i ^ row / 4 % 4.  So the 16 rows that a quarter of a wavefront
// reads fall into different banks, as do the four rows of 64 bytes that half of one reads by columns, and a lane gets
// along with two addresses for rows and two for columns: everything else is a constant of the instruction.  (Rows whole, chunks
// exchanged by exclusive or with the row: an instruction for each address, and conflicts in up to 46 % of the LDS's busy cycles.)
// ------------------------------------------------------------------------------------------
template <typename WT, int D> struct GbTile {
    static constexpr int ESZ = Traits<WT>::ESZ, ROWB = D * ESZ, BYTES = 32 * ROWB, STEPS = ROWB / 32;
    static constexpr bool BF = Traits<WT>::BF;
    static __device__ __forceinline__ int swap(int row, int i) { return i ^ (row >> 2 & 3); }

    int rd[2], cd[2];     // this lane's places: of its row, pieces half and 2 + half; of its column, rows 4 half .. and 8 + 4 half ..
    __device__ __forceinline__ GbTile(int lane) {
        const int c = lane & 31, half = lane >> 5;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            rd[i] = c * 64 + swap(c, 2 * i + half) * 16;
            if constexpr (BF) {
                const int row = 8 * i + 4 * half + ((lane & 15) >> 2), piece = (lane >> 4 & 1) * 2 + (lane >> 1 & 1);
                cd[i] = row * 64 + swap(row, piece) * 16 + (lane & 1) * 8;
            } else {
                const int row = 8 * i + 4 * half;
                cd[i] = (c >> 4) * 2048 + row * 64 + swap(row, c >> 2 & 3) * 16 + (c & 3) * 4;
            }
        }
    }
    // 16 bytes of the lane's row: step st's operand
    __device__ __forceinline__ uint4 row(const char* tile, int st) const { return ld16(tile + rd[st & 1] + (st >> 1) * 2048); }
    // columns 32 j + c, rows 16 m + 4 half + {0..3, 8..11} (bf16)
    __device__ __forceinline__ bf16x8 column(const char* tile, int j, int m) const {
        const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(tile + cd[0] + j * 2048 + m * 1024));
        const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(tile + cd[1] + j * 2048 + m * 1024));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    // ... values that are not finite count as zero (gb_add_odd makes up for it)
    static __device__ __forceinline__ bf16x8 finite(bf16x8 x) {
        u32x4 v = __builtin_bit_cast(u32x4, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = (v[e] & 0x7F80u) == 0x7F80u ? v[e] & 0xFFFF0000u : v[e];
            v[e] = (v[e] & 0x7F800000u) == 0x7F800000u ? v[e] & 0xFFFFu : v[e];
        }
        return __builtin_bit_cast(bf16x8, v);
    }
    // column 32 j + c of row 8 (i / 4) + i % 4 + 4 half (float32; with clean, likewise)
    template <bool CLEAN> __device__ __forceinline__ float element(const char* tile, int j, int i) const {
        const float v = *reinterpret_cast<const float*>(tile + cd[i >> 2 & 1] + j * 4096 + (i >> 3) * 1024 + (i & 3) * 64);
        return !CLEAN || fabsf(v) < INFINITY ? v : 0.f;
    }
};

// float32: scores += rows . own: the lane's i-th is that of row 8 (i / 4) + i % 4 + 4 half and the lane's own query or key
template <typename WT, int D>
__device__ __forceinline__ void gb_scores(const GbTile<WT, D>& L, const char* tile, const uint4 (&own)[GbTile<WT, D>::STEPS], f32x16& x) {
#pragma unroll
    for (int st = 0; st < GbTile<WT, D>::STEPS; ++st) {
        const f32x4 u = __builtin_bit_cast(f32x4, L.row(tile, st)), w = __builtin_bit_cast(f32x4, own[st]);
#pragma unroll
        for (int e = 0; e < 4; ++e) x = __builtin_amdgcn_mfma_f32_32x32x2f32(u[e], w[e], x, 0, 0, 0);
    }
}
// float32: y^T += rows^T . p, p as gb_scores leaves it
template <typename WT, int D, bool CLEAN>
__device__ __forceinline__ void gb_products(const GbTile<WT, D>& L, const char* tile, const f32x16& p, f32x16 (&y)[D / 32]) {
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int j = 0; j < D / 32; ++j) y[j] = __builtin_amdgcn_mfma_f32_32x32x2f32(L.template element<CLEAN>(tile, j, i), p[i], y[j], 0, 0, 0);
}
// bf16: p (P, or dS) as operand of the two MFMAs over its 32 rows, rounded to bf16 once.  The forward pass holds P in two parts; here a second part
// would be 3 products more in the keys' kernel (dV, dK with either part of dS) and one in the queries', 14 in the place of 10, for an error of 0.0017 of the
// gradients' 2-norm, which the results' own rounding leaves, in the place of 0.0024: the rounding of P and dS weighs as much as that of the
// results.  The queries' low parts are another matter: they belong to the scores, whose lse the forward pass made with them.
template <typename WT> struct GbOperand {
    bf16x8 b[2];
    __device__ __forceinline__ GbOperand(const f32x16& p) {
#pragma unroll
        for (int m = 0; m < 2; ++m)
            b[m] = __builtin_bit_cast(bf16x8, make_uint4(pack_bf16x2(p[8 * m], p[8 * m + 1]), pack_bf16x2(p[8 * m + 2], p[8 * m + 3]),
                                                         pack_bf16x2(p[8 * m + 4], p[8 * m + 5]), pack_bf16x2(p[8 * m + 6], p[8 * m + 7])));
    }
};
typedef __attribute__((address_space(3))) void lds_void;
// 16 bytes per lane to the LDS, lane after lane from `to` on, by the memory unit itself
__device__ __forceinline__ void gb_copy(rsrc_t from, unsigned off, char* to) { __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lds_void*)to, 16, off, 0, 0, 0); }
// this wavefront's requests have arrived, and its own reads and writes of LDS are done
__device__ __forceinline__ void gb_wait() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" : : : "memory"); }
// ... the workgroup's
__device__ __forceinline__ void gb_arrived() {
    gb_wait();
    __syncthreads();
}
// A tile of 32 rows, `stride` bytes apart, rows beyond `most` replaced by it: its i-th KiB (64 bytes of 16 rows)
template <typename WT, int D> __device__ __forceinline__ void gb_request(const char* m, unsigned stride, int most, char* tile, int i, int lane) {
    const int row = 16 * (i & 1) + lane / 4, piece = GbTile<WT, D>::swap(row, lane & 3);
    gb_copy(make_rsrc(m), (unsigned)min(row, most) * stride + (i >> 1) * 64 + piece * 16, tile + i * 1024);
}
// ... this wavefront's share of WAVES
template <typename WT, int D, int WAVES>
__device__ __forceinline__ void gb_stage(const char* m, unsigned stride, int most, char* tile, int wave, int lane) {
    constexpr int N = GbTile<WT, D>::BYTES / 1024;
    static_assert(N % WAVES == 0, "");
#pragma unroll
    for (int u = 0; u < N / WAVES; ++u) gb_request<WT, D>(m, stride, most, tile, wave + u * WAVES, lane);
}
// bf16: a tile's work as N operands from LDS, one after the other, each with the MFMAs that take it (and the one before it).  Operands are
// asked for three ahead, and the compiler keeps that order: left alone it asks for one or two, and an MFMA waits for most of the LDS's
// latency.  (Two to six ahead take the same time; more spill.)  beside(): what is done at the start (the next stage's requests).
constexpr int GB_SLOTS = 5;
template <int N, typename LOAD, typename USE, typename BESIDE> __device__ __forceinline__ void gb_stream(LOAD load, USE use, BESIDE beside) {
    constexpr int AHEAD = GB_SLOTS - 2;
    bf16x8 x[GB_SLOTS];
    auto first = [&](auto self, auto n) __attribute__((always_inline)) {
        if constexpr (n < AHEAD && n < N) {
            x[n] = load(n);
            self(self, std::integral_constant<int, n + 1>{});
        }
    };
    first(first, std::integral_constant<int, 0>{});
    auto run = [&](auto self, auto n) __attribute__((always_inline)) {
        if constexpr (n < N) {
            if constexpr (n + AHEAD < N) x[(n + AHEAD) % GB_SLOTS] = load(std::integral_constant<int, n + AHEAD>{});
            __builtin_amdgcn_sched_barrier(0);
            use(n, x[n % GB_SLOTS], x[(n + GB_SLOTS - 1) % GB_SLOTS]);
            if constexpr (n == 0) beside();
            __builtin_amdgcn_sched_barrier(0);
            self(self, std::integral_constant<int, n + 1>{});
        }
    };
    run(run, std::integral_constant<int, 0>{});
}
// a lane's row as operand, straight from memory
template <typename WT, int D> __device__ __forceinline__ void gb_own_rows(const char* row, int half, uint4 (&x)[GbTile<WT, D>::STEPS]) {
#pragma unroll
    for (int st = 0; st < GbTile<WT, D>::STEPS; ++st) x[st] = ld16_q(row + st * 32 + half * 16);
}
constexpr float GB_LN2 = 0.6931471805599453f;
// In tiles that the mask cuts, what is not finite counts as zero in the products (a hidden row's 0 times Inf would be NaN).  For the queries or
// keys that do see such a row this makes up for it at the end, from memory: y[j][i], column 32 j + 8 (i / 4) + 4 half + i % 4 of the lane's sum,
// gets the row's values that are not finite.  PROBABILITY: as they are, which is what a probability makes of them; else NaN (the
// other factor, a dS, is NaN or Inf itself, or 0 where a key's score is -Inf).  A row may be added more than once.
template <typename WT, int D, bool PROBABILITY> __device__ __forceinline__ void gb_add_odd(const char* row, int half, f32x16 (&y)[D / 32]) {
#pragma unroll
    for (int j = 0; j < D / 32; ++j)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const f32x4 v = load4_q<WT>(row + (32 * j + 8 * u + 4 * half) * Traits<WT>::ESZ);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (!(fabsf(v[e]) < INFINITY)) y[j][4 * u + e] += PROBABILITY ? v[e] : NAN;
        }
}
// whether there is nothing left to add: a call whose values are all NaN would walk all rows for it (T 2048, k 4 3.3 ms in the place of 1.1)
template <int N> __device__ __forceinline__ bool gb_all_nan(const f32x16 (&y)[N]) {
    bool all = true;
#pragma unroll
    for (int j = 0; j < N; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i) all &= y[j][i] != y[j][i];
    return all;
}
// columns col .. col + 3 and col + D / 2 .. of a row of a gradient, times scale; with turn, rotated back
template <typename WT, int D> __device__ __forceinline__ void gb_write4(char* row, const float2* turn, int col, float scale, f32x4 a, f32x4 b) {
    constexpr int ESZ = Traits<WT>::ESZ;
    a *= scale;
    b *= scale;
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
// the lane's row, y[j][i] = column 32 j + 8 (i / 4) + 4 half + i % 4
template <typename WT, int D>
__device__ __forceinline__ void gb_write(char* row, const float2* turn, float scale, int half, const f32x16 (&y)[D / 32]) {
    constexpr int NJ = D / 32;
#pragma unroll
    for (int j = 0; j < NJ / 2; ++j)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            f32x4 a, b;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                a[e] = y[j][4 * u + e];
                b[e] = y[j + NJ / 2][4 * u + e];
            }
            gb_write4<WT, D>(row, turn, 32 * j + 8 * u + 4 * half, scale, a, b);
        }
}

// ------------------------------------------------------------------------------------------
// Gradients of the queries.  A wavefront owns 32 layout rows.  It rotates its queries (and leaves them, and the rows' statistics, for the
// kernel of the keys), looks at its own groups' [MASK] keys - among its own 32 rows and, where its first row is not the first of its
// group, the 32 before - and walks the real tokens up to its last group, 64 per stage, two buffers.  KW = 1: a workgroup is four wavefronts
// of 32 rows; 2 (few rows): two, each shared by two wavefronts that take every other key tile and meet in the LDS at the end.
// ------------------------------------------------------------------------------------------
template <typename WT, int D, int KW>
__global__ void __launch_bounds__(GB_THREADS, D * Traits<WT>::ESZ > 256 ? 1 : 2) gb_dq_kernel(const GbParams P) {
    typedef GbTile<WT, D> Tile;
    constexpr int ESZ = Traits<WT>::ESZ, GE = Traits<WT>::GE, PARTS = GbTraits<WT>::PARTS, NJ = D / 32, STEPS = Tile::STEPS, ROWS = GB_ROWS / KW;
    constexpr int BUF = 4 * Tile::BYTES;                    // two key tiles, K and V each
    static_assert(2 * BUF == GB_WAVES * 2 * Tile::BYTES, "a stage's buffers, or one key tile for each wavefront");
    __shared__ __attribute__((aligned(16))) char smem[2 * BUF];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, half = lane >> 5;
    const int rw = wave / KW, kw = wave % KW;
    // (the rows with the most keys start first; neighbours, which go to different XCDs, take different heads)
    const int K1 = P.k + 1, y_at = blockIdx.x / P.nq, h = blockIdx.x - y_at * P.nq, blk = gridDim.x / P.nq - 1 - y_at, seq = blockIdx.y, hk = h / P.group;
    const int R0 = ROWS * blk, r0 = R0 + 32 * rw, r_last = min(R0 + ROWS, P.rows) - 1, g_last = gb_group(P, r_last);
    const bool active = r0 < P.rows;
    const int n_stages = g_last / 64 + 1;
    const int qrow = min(r0 + c, r_last), qg = gb_group(P, qrow), w_first = min(r0, r_last), wg0 = gb_group(P, w_first), wg1 = gb_group(P, min(r0 + 31, r_last));
    const Tile L(lane);
    const char* krows = P.k_rot + ((size_t)seq * P.nkv + hk) * P.rows * D * ESZ;
    const char* vrows = P.v + ((size_t)seq * P.rows * P.nkv + hk) * D * ESZ;
    const unsigned vstride = (unsigned)(P.nkv * D * ESZ);
    auto stage_own = [&](int first) __attribute__((always_inline)) {   // layout rows first .. first + 31, to the wavefront's own tiles
        char* b = smem + wave * 2 * Tile::BYTES;
        const int from = min(max(first, 0), r_last);
        gb_stage<WT, D, 1>(krows + (size_t)from * D * ESZ, D * ESZ, r_last - from, b, 0, lane);
        gb_stage<WT, D, 1>(vrows + (size_t)from * vstride, vstride, r_last - from, b + Tile::BYTES, 0, lane);
    };
    auto stage = [&](int t, char* buf) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int first = min(64 * t + 32 * i, g_last);
            char* b = buf + i * 2 * Tile::BYTES;
            gb_stage<WT, D, GB_WAVES>(krows + (size_t)first * K1 * D * ESZ, K1 * D * ESZ, g_last - first, b, wave, lane);
            gb_stage<WT, D, GB_WAVES>(vrows + (size_t)first * K1 * vstride, K1 * vstride, g_last - first, b + Tile::BYTES, wave, lane);
        }
    };
    // own [MASK] keys: the wavefront's own tile and the one before (KW = 2: one of the two each)
    const bool before = wg0 * K1 != r0;
    if (P.k > 0) stage_own(r0 - 32 * kw);

    // ---- the lane's row: statistics, the rotated query as operand
    const size_t at = ((size_t)seq * P.rows + qrow) * P.nq + h, to = ((size_t)seq * P.nq + h) * P.rows + qrow, part = (size_t)P.seqs * P.nq * P.rows * D * ESZ;
    uint4 q[PARTS][STEPS], d_o[STEPS];
    gb_own_rows<WT, D>(P.q + at * D * ESZ, half, q[0]);
    gb_own_rows<WT, D>(P.d_out + at * D * ESZ, half, d_o);
    float delta0 = 0.f;
    {
        const float* o = P.out + at * D + half * GE;
#pragma unroll
        for (int t = 0; t < STEPS; ++t) {
            float x[GE];
            unpack_group<WT>(d_o[t], x);
#pragma unroll
            for (int e = 0; e < GE; e += 4) {
                const f32x4 y = load4_q<float>(o + 2 * GE * t + e);
                delta0 -= (x[e] * y[0] + x[e + 1] * y[1]) + (x[e + 2] * y[2] + x[e + 3] * y[3]);
            }
        }
        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(delta0), __float_as_uint(delta0), false, false);
        delta0 = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
    }
    const float lse0 = -P.lse[at] * 1.4426950408889634f, qscale = P.inv_sqrt_d * 1.4426950408889634f;
    const float2* turn = P.table + (size_t)(qrow - qg * P.k) * (D / 2);
    const bool owner = kw == 0 && r0 + c < P.rows;
    if (owner && half == 0) {
        P.lse2[to] = lse0;
        P.delta[to] = delta0;
    }
#pragma unroll
    for (int t = 0; t < STEPS / 2; ++t) {
        float a[GE], b[GE], ra[GE], rb[GE];
        unpack_group<WT>(q[0][t], a);
        unpack_group<WT>(q[0][t + STEPS / 2], b);
        const f32x4* cs = reinterpret_cast<const f32x4*>(turn + GE * (2 * t + half));
#pragma unroll
        for (int e = 0; e < GE; e += 2) {
            const f32x4 x = cs[e / 2];
            ra[e] = (a[e] * x[0] - b[e] * x[1]) * qscale;
            rb[e] = (b[e] * x[0] + a[e] * x[1]) * qscale;
            ra[e + 1] = (a[e + 1] * x[2] - b[e + 1] * x[3]) * qscale;
            rb[e + 1] = (b[e + 1] * x[2] + a[e + 1] * x[3]) * qscale;
        }
        if constexpr (Traits<WT>::BF) {
            unsigned hi[4];
            q[0][t] = __builtin_bit_cast(uint4, split_hi(ra, hi));
            q[1][t] = __builtin_bit_cast(uint4, split_lo(ra, hi));
            q[0][t + STEPS / 2] = __builtin_bit_cast(uint4, split_hi(rb, hi));
            q[1][t + STEPS / 2] = __builtin_bit_cast(uint4, split_lo(rb, hi));
        } else {
            q[0][t] = __builtin_bit_cast(uint4, f32x4{ra[0], ra[1], ra[2], ra[3]});
            q[0][t + STEPS / 2] = __builtin_bit_cast(uint4, f32x4{rb[0], rb[1], rb[2], rb[3]});
        }
    }
    if (owner) {
#pragma unroll
        for (int p = 0; p < PARTS; ++p)
#pragma unroll
            for (int t = 0; t < STEPS; ++t) *reinterpret_cast<uint4*>(P.q_rot + p * part + to * D * ESZ + t * 32 + half * 16) = q[p][t];
    }
    f32x16 y[NJ];
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i) y[j][i] = 0.f;

    // one key tile; masked: keys lo .. hi of it (counted from 4 half) are seen
    bool odd = false;                                        // a key in such a tile was not finite: nor were its scores
    auto work = [&](const char* kt, auto masked, int lo, int hi, auto beside) __attribute__((always_inline)) {
        const char* vt = kt + Tile::BYTES;
        float lse = lse0, delta = delta0;
        asm volatile("" : "+v"(lse), "+v"(delta));          // (32 copies of them would be kept in registers across the loop)
        f32x16 s, dp;
        auto probabilities = [&]() __attribute__((always_inline)) {   // dS in the place of s
            if constexpr (masked) {
                float m = 0.f;
#pragma unroll
                for (int i = 0; i < 16; i += 2) m = abs_max3(m, s[i], s[i + 1]);
                odd |= __any(!(m < INFINITY)) != 0;
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int key = 8 * (i / 4) + i % 4;
                const float x = __builtin_amdgcn_exp2f(s[i]) * dp[i];
                s[i] = !masked || (key >= lo && key <= hi) ? x : 0.f;
            }
        };
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            s[i] = lse;
            dp[i] = delta;
        }
        if constexpr (Traits<WT>::BF) {
            bf16x8 ds[2];
            constexpr int H = 2 * STEPS, N = H + 2 * NJ;     // a step's K and V rows in turn; K columns
            gb_stream<N>(
                [&](auto n) __attribute__((always_inline)) {
                    if constexpr (n < H) return __builtin_bit_cast(bf16x8, L.row(n % 2 ? vt : kt, n / 2));
                    else return L.column(kt, (n - H) % NJ, (n - H) / NJ);
                },
                [&](auto n, bf16x8 x, bf16x8 before) __attribute__((always_inline)) {
                    if constexpr (n < H) {                   // (scores and dP in turn: no MFMA takes what the one before it gives)
                        if constexpr (n % 2 == 0) {
                            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, __builtin_bit_cast(bf16x8, q[0][n / 2]), s, 0, 0, 0);
                        } else {
                            dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, __builtin_bit_cast(bf16x8, d_o[n / 2]), dp, 0, 0, 0);
                            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(before, __builtin_bit_cast(bf16x8, q[PARTS - 1][n / 2]), s, 0, 0, 0);
                        }
                    } else {
                        constexpr int j = (n - H) % NJ;
                        y[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(masked ? Tile::finite(x) : x, ds[(n - H) / NJ], y[j], 0, 0, 0);
                    }
                    if constexpr (n == H - 1) {
                        probabilities();
                        const GbOperand<WT> p(s);
                        ds[0] = p.b[0];
                        ds[1] = p.b[1];
                    }
                }, beside);
        } else {
            beside();
#pragma unroll
            for (int p = 0; p < PARTS; ++p) gb_scores<WT, D>(L, kt, q[p], s);
            gb_scores<WT, D>(L, vt, d_o, dp);
            probabilities();
            gb_products<WT, D, masked>(L, kt, s, y);
        }
    };
    if (P.k > 0) {
        const char* mine = smem + wave * 2 * Tile::BYTES;
        const int lo = qg * K1 + 1 - 4 * half, hi = qrow - 4 * half;
        for (int i = kw; i < 2; i += KW) {                   // 0: rows r0 .., 1: rows r0 - 32 ..
            if (KW == 1 && i == 1) {
                gb_wait();                                   // (nobody else reads these tiles)
                if (before) stage_own(r0 - 32);
            }
            gb_arrived();
            if (active && (i == 0 || before)) work(mine, std::true_type{}, lo - (r0 - 32 * i), hi - (r0 - 32 * i), [] {});
        }
        __syncthreads();
    }
    // real tokens: stages that all of the wavefront's queries see, some of them, none
    stage(0, smem);
    gb_arrived();
    int t = 0;
    // (restrict: a read of this stage need not wait for the next one's requests; to the compiler both are one array, and without it every
    // stage's first read waits for requests that have only just been made: T 2048, k 4, both kernels, 1066 us in the place of 1031)
    auto seen = [&](const char* __restrict mine, char* __restrict next) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 2 / KW; ++i)
            work(mine + (i * KW + kw) * 2 * Tile::BYTES, std::false_type{}, 0, 0,
                 [&]() __attribute__((always_inline)) { if (i == 0 && t + 1 < n_stages) stage(t + 1, next); });
    };
    for (const int end = active ? (wg0 + 1) / 64 : 0; t < end; ++t) {
        seen(smem + (t & 1) * BUF, smem + (1 - (t & 1)) * BUF);
        gb_arrived();
    }
    auto partly = [&](const char* __restrict mine, char* __restrict next) __attribute__((always_inline)) {
        if (t + 1 < n_stages) stage(t + 1, next);
#pragma unroll 1
        for (int i = kw; i < 2; i += KW) {
            const int first = 64 * t + 32 * i;
            if (active && first <= wg1) work(mine + i * 2 * Tile::BYTES, std::true_type{}, -first - 4 * half, qg - first - 4 * half, [] {});
        }
    };
    for (; t < n_stages; ++t) {
        partly(smem + (t & 1) * BUF, smem + (1 - (t & 1)) * BUF);
        gb_arrived();
    }
    if (__builtin_expect(odd, 0)) {                          // the lane's own [MASK] keys, the tokens behind the stages that are seen whole
#pragma unroll 1
        for (int r = qg * K1 + 1; r <= qrow && !gb_all_nan(y); ++r) gb_add_odd<WT, D, false>(krows + (size_t)r * D * ESZ, half, y);
#pragma unroll 1
        for (int n = (wg0 + 1) / 64 * 64; n <= qg && !gb_all_nan(y); ++n) gb_add_odd<WT, D, false>(krows + (size_t)n * K1 * D * ESZ, half, y);
    }
    if constexpr (KW == 2) {
        f32x4* area = reinterpret_cast<f32x4*>(smem) + rw * NJ * 4 * 64 + lane;
        if (kw) {
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int u = 0; u < 4; ++u) area[(j * 4 + u) * 64] = f32x4{y[j][4 * u], y[j][4 * u + 1], y[j][4 * u + 2], y[j][4 * u + 3]};
        }
        __syncthreads();
        if (kw) return;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const f32x4 v = area[(j * 4 + u) * 64];
#pragma unroll
                for (int e = 0; e < 4; ++e) y[j][4 * u + e] += v[e];
            }
    }
    if (r0 + c < P.rows) gb_write<WT, D>(P.d_q + at * D * ESZ, turn, P.inv_sqrt_d, half, y);
}

// ------------------------------------------------------------------------------------------
// Gradients of keys and values.  A wavefront owns 32 keys (rows as operands, gradients as accumulators) and takes a tile of 32 query rows
// at a time.  A workgroup is KW wavefronts of keys by two of rows: a stage holds two row tiles (rotated queries' parts, d_out,
// statistics), brought in by the memory unit itself; the two row wavefronts' sums meet in the LDS at the end.
// bf16, head_dim 128: the values' rows stay in LDS, so that two wavefronts per SIMD find room for everything else in their 256 registers.
// (64 keys per wavefront, which halves the LDS reads per product but leaves a SIMD one wavefront: 900 us in the place of 640 at T 2048.)
// A step takes 48 MFMAs, 88 LDS reads and 69 vector instructions; the matrix cores are busy 42 % of the time and the LDS 28 %.
// ------------------------------------------------------------------------------------------
template <typename WT, int D, bool V_LDS> struct GbKeys {
    typedef GbTile<WT, D> Tile;
    static constexpr int PARTS = GbTraits<WT>::PARTS, NJ = D / 32;
    uint4 kf[Tile::STEPS], vf[V_LDS ? 1 : Tile::STEPS];
    const char* v_tile;
    f32x16 dk[NJ], dv[NJ];
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) { dk[j][i] = 0.f; dv[j][i] = 0.f; }
    }
    // buf: the tiles of the rotated queries' parts, then of d_out; stats: the 32 rows' -lse / ln 2, then (behind `two` floats) -delta; the lane's
    // key is seen by rows lo .. hi of the tile (counted from 4 half), all of them if not masked
    template <bool MASKED, typename BESIDE>
    __device__ __forceinline__ void step(const Tile& L, const char* buf, const float* stats, int two, int half, int lo, int hi, BESIDE beside) {
        f32x16 s, dp;
        auto start = [&](const float* x, f32x16& y) __attribute__((always_inline)) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x4 v = *reinterpret_cast<const f32x4*>(x + 8 * q + 4 * half);
#pragma unroll
                for (int e = 0; e < 4; ++e) y[4 * q + e] = v[e];
            }
        };
        const char* dt = buf + PARTS * Tile::BYTES;
        auto probabilities = [&]() __attribute__((always_inline)) {   // P in the place of s, dS in that of dp
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int row = 8 * (i / 4) + i % 4;
                const bool in = !MASKED || (row >= lo && row <= hi);
                const float p = in ? __builtin_amdgcn_exp2f(s[i]) : 0.f;
                s[i] = p;
                dp[i] = in ? p * dp[i] : 0.f;
            }
        };
        start(stats, s);
        if constexpr (Traits<WT>::BF) {
            bf16x8 p[2], ds[2];
            // a step's rows of the queries' high part, (of the values, if they stand in LDS), of d_out and of the queries' low part; columns of d_out,
            // of the parts
            constexpr int U = V_LDS ? 4 : 3, B = U * Tile::STEPS, C = 2 * NJ, N = B + 3 * C;
            start(stats + two, dp);
            gb_stream<N>(
                [&](auto n) __attribute__((always_inline)) {
                    if constexpr (n < B) {
                        constexpr int u = n % U;
                        const char* from = u == U - 1 ? buf + Tile::BYTES : u == U - 2 ? dt : u == 0 ? buf : v_tile;
                        return __builtin_bit_cast(bf16x8, L.row(from, n / U));
                    } else {
                        constexpr int o = (n - B) % C;
                        return L.column((n - B) / C == 0 ? dt : buf + ((n - B) / C - 1) * Tile::BYTES, o % NJ, o / NJ);
                    }
                },
                [&](auto n, bf16x8 x, bf16x8 before) __attribute__((always_inline)) {
                    if constexpr (n < B) {                   // (scores and dP in turn: no MFMA takes what the one before it gives)
                        constexpr int u = n % U;
                        if constexpr (u == U - 2) {
                            if constexpr (!V_LDS) before = __builtin_bit_cast(bf16x8, vf[n / U]);
                            dp = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, before, dp, 0, 0, 0);
                        } else if constexpr (u == 0 || u == U - 1) {
                            s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, __builtin_bit_cast(bf16x8, kf[n / U]), s, 0, 0, 0);
                        }
                    } else {
                        constexpr int o = (n - B) % C, j = o % NJ;
                        const bf16x8 a = MASKED ? Tile::finite(x) : x;
                        if constexpr (n < B + C) dv[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, p[o / NJ], dv[j], 0, 0, 0);
                        else dk[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, ds[o / NJ], dk[j], 0, 0, 0);
                    }
                    if constexpr (n == B - 1) {
                        probabilities();
                        const GbOperand<WT> a(s), b(dp);
                        p[0] = a.b[0]; p[1] = a.b[1]; ds[0] = b.b[0]; ds[1] = b.b[1];
                    }
                }, beside);
        } else {
            start(stats + two, dp);
            beside();
            gb_scores<WT, D>(L, buf, kf, s);
            gb_scores<WT, D>(L, dt, vf, dp);
            probabilities();
            gb_products<WT, D, MASKED>(L, dt, s, dv);
            gb_products<WT, D, MASKED>(L, buf, dp, dk);
        }
    }
};
// A query or a gradient that is not finite makes every dS of its row so, and with it the d_k of every key that it sees (of one of the wavefront's)
template <int N> __device__ __forceinline__ bool gb_odd_rows(const f32x16 (&dk)[N]) { return __any(!(fabsf(dk[0][0]) < INFINITY)) != 0; }
// ... what rows first .. last of the layout, which the lane's key sees, have left out: query heads of the kv head in turn
template <typename WT, int D>
__device__ __forceinline__ void gb_add_odd_rows(const GbParams& P, int seq, int hk, int first, int last, int half, f32x16 (&dk)[D / 32], f32x16 (&dv)[D / 32]) {
    constexpr int ESZ = Traits<WT>::ESZ;
#pragma unroll 1
    for (int h = hk * P.group; h < (hk + 1) * P.group; ++h)
#pragma unroll 1
        for (int r = first; r <= last && !gb_all_nan(dv); ++r) {   // (a d_v of NaN alone: P or d_out was, and so is d_k)
            gb_add_odd<WT, D, true>(P.d_out + (((size_t)seq * P.rows + r) * P.nq + h) * D * ESZ, half, dv);
            gb_add_odd<WT, D, false>(P.q_rot + (((size_t)seq * P.nq + h) * P.rows + r) * D * ESZ, half, dk);
        }
}
template <typename WT, int D>
__device__ __forceinline__ void gb_write_keys(const GbParams& P, int seq, int hk, int row, int pos, int half, const f32x16 (&dk)[D / 32], const f32x16 (&dv)[D / 32]) {
    const size_t at = (((size_t)seq * P.rows + row) * P.nkv + hk) * D * Traits<WT>::ESZ;
    gb_write<WT, D>(P.d_k + at, P.table + (size_t)pos * (D / 2), GB_LN2, half, dk);   // (the queries carry log2(e) / sqrt(d))
    gb_write<WT, D>(P.d_v + at, nullptr, 1.f, half, dv);
}

// Work of a launch of gb_dkv_kernel.  Workgroups units * splits: (key tile, part, head), the tiles with the most rows first, neighbours
// different heads; `splits` workgroups share a key tile's rows and leave partial sums.  Then those of [MASK] keys (four tiles each).
struct GbWork { int heads, splits, units, own_tiles; float* partial; };

template <typename WT, int D, int KW> struct GbDkv {
    typedef GbTile<WT, D> Tile;
    static constexpr bool V_LDS = Traits<WT>::BF && D == 128;
    static constexpr int WAVES = 2 * KW, KEYS = 32 * KW, PER_SIMD = D * Traits<WT>::ESZ > 256 ? 1 : 2;
    static constexpr int PARTS = GbTraits<WT>::PARTS, SET = (PARTS + 1) * Tile::BYTES, OFF_S = 2 * SET, BUF = OFF_S + 2 * 32 * 8;
    static constexpr int OFF_V = 2 * BUF, STAGES = OFF_V + (V_LDS ? KW * Tile::BYTES : 0);
    static constexpr int OWNERS = V_LDS ? 4 : WAVES;         // wavefronts with tiles of [MASK] keys: one set of tiles each, and their values
    static constexpr int OWN = SET + (V_LDS ? Tile::BYTES : 0) + 32 * 8, SMEM = STAGES > OWNERS * OWN ? STAGES : OWNERS * OWN;
    static_assert(SMEM <= 160 * 1024 && KW * D / 32 * 16 * 64 * 4 <= SMEM, "");
};

template <typename WT, int D, int KW>
__global__ void __launch_bounds__((GbDkv<WT, D, KW>::WAVES * 64), (GbDkv<WT, D, KW>::PER_SIMD)) gb_dkv_kernel(const GbParams P, const GbWork W) {
    typedef GbTile<WT, D> Tile;
    typedef GbDkv<WT, D, KW> C;
    constexpr int ESZ = Traits<WT>::ESZ, PARTS = C::PARTS, NJ = D / 32;
    __shared__ __attribute__((aligned(16))) char smem[C::SMEM];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, half = lane >> 5;
    const int K1 = P.k + 1;
    const Tile L(lane);
    const size_t part = (size_t)P.seqs * P.nq * P.rows * D * ESZ;
    const unsigned ostride = (unsigned)(P.nq * D * ESZ), vstride = (unsigned)(P.nkv * D * ESZ);
    GbKeys<WT, D, C::V_LDS> keys;
    keys.clear();
    if ((int)blockIdx.x >= W.units * W.splits) {
        // ---- [MASK] keys, which the later rows of their own group see: a wavefront takes as many whole groups as fit into 32 rows, every
        // query head that shares the kv head in turn
        const int x = C::OWNERS * ((int)blockIdx.x - W.units * W.splits) + wave, tiles = (P.T + P.gpt - 1) / P.gpt;
        if (wave >= C::OWNERS || x >= W.own_tiles) return;
        const int head = x / tiles, first = (x - head * tiles) * P.gpt * K1, last = min(first + P.gpt * K1, P.rows) - 1, seq = head / P.nkv, hk = head - seq * P.nkv;
        const int krow = min(first + c, last), g = gb_group(P, krow), slot = krow - g * K1;
        char* const buf = smem + wave * C::OWN;
        gb_own_rows<WT, D>(P.k_rot + (((size_t)seq * P.nkv + hk) * P.rows + krow) * D * ESZ, half, keys.kf);
        const char* v = P.v + (((size_t)seq * P.rows + first) * P.nkv + hk) * D * ESZ;
        if constexpr (C::V_LDS) {
            gb_stage<WT, D, 1>(v, vstride, last - first, buf + C::SET, 0, lane);
            keys.v_tile = buf + C::SET;
        } else {
            gb_own_rows<WT, D>(v + (size_t)(krow - first) * vstride, half, keys.vf);
        }
        float* const stats = reinterpret_cast<float*>(buf + C::OWN - 32 * 8);
        for (int i = 0; i < P.group; ++i) {
            const int h = hk * P.group + i;
            const size_t at = ((size_t)seq * P.nq + h) * P.rows;
#pragma unroll
            for (int p = 0; p < PARTS; ++p) gb_stage<WT, D, 1>(P.q_rot + p * part + (at + first) * D * ESZ, D * ESZ, last - first, buf + p * Tile::BYTES, 0, lane);
            gb_stage<WT, D, 1>(P.d_out + (((size_t)seq * P.rows + first) * P.nq + h) * D * ESZ, ostride, last - first, buf + PARTS * Tile::BYTES, 0, lane);
            stats[lane] = (lane < 32 ? P.lse2 : P.delta)[at + krow];
            gb_wait();                                       // (for this wavefront's own reads)
            keys.template step<true>(L, buf, stats, 32, half, slot > 0 ? krow - first - 4 * half : 99, g * K1 + P.k - first - 4 * half, [] {});
            gb_wait();
        }
        if (__builtin_expect(gb_odd_rows(keys.dk), 0)) gb_add_odd_rows<WT, D>(P, seq, hk, krow, slot > 0 ? g * K1 + P.k : -1, half, keys.dk, keys.dv);
        if (first + c <= last && slot > 0) gb_write_keys<WT, D>(P, seq, hk, krow, krow - g * P.k, half, keys.dk, keys.dv);
        return;
    }
    const int y = blockIdx.x / W.heads, head = blockIdx.x - y * W.heads, kt = y / W.splits, split = y - kt * W.splits;
    const int seq = head / P.nkv, hk = head - seq * P.nkv, kw = wave % KW, rw = wave / KW;
    const int t0 = C::KEYS * kt, w0 = t0 + 32 * kw, key = min(w0 + c, P.T - 1);   // the workgroup's and the wavefront's first token, the lane's
    const int first_row = t0 * K1, per_head = (P.rows - first_row + 63) / 64, all = per_head * P.group;
    const int i0 = (int)((long long)all * split / W.splits), i1 = (int)((long long)all * (split + 1) / W.splits);
    // the next set of 64 rows to request: of query head hk * group + next_g, from its next_j-th on (behind the last: the last again; a branch
    // among the products would have the compiler spill)
    int next_g = i0 / per_head, next_j = i0 - next_g * per_head;
    const int next_j0 = next_j;
    float stat = 0.f;
    bool stat_in = false;
    auto stage = [&](int i, char* b) __attribute__((always_inline)) {   // set i, to a buffer
        const int h = hk * P.group + next_g, first = first_row + 64 * next_j, left = P.rows - 1 - first;
        const size_t at = ((size_t)seq * P.nq + h) * P.rows + first;
        constexpr int N = Tile::BYTES / 1024;
        static_assert(2 * N % C::WAVES == 0, "");
#pragma unroll
        for (int u = 0; u < 2 * N / C::WAVES; ++u) {         // the two tiles' requests together
            const int x = wave + u * C::WAVES, r = x / N, from = min(32 * r, left), most = left - from;
            char* to = b + r * C::SET;
#pragma unroll
            for (int p = 0; p < PARTS; ++p) gb_request<WT, D>(P.q_rot + p * part + (at + from) * D * ESZ, D * ESZ, most, to + p * Tile::BYTES, x % N, lane);
            gb_request<WT, D>(P.d_out + (((size_t)seq * P.rows + first + from) * P.nq + h) * D * ESZ, ostride, most, to + PARTS * Tile::BYTES, x % N, lane);
        }
        // (every second wavefront's is the same; a row beyond the last: probability 0, whatever the last row, which it repeats, holds)
        // (looked at where it is stored, a stage later)
        stat = (wave & 1 ? P.delta : P.lse2)[at + min(lane, left)];
        stat_in = wave & 1 || lane <= left;
        next_j += i + 1 < i1;
        const bool wrap = next_j == per_head;
        next_j = wrap ? 0 : next_j;
        next_g += wrap;
    };
    auto stage_stats = [&](int i) __attribute__((always_inline)) { reinterpret_cast<float*>(smem + (i & 1) * C::BUF + C::OFF_S)[64 * (wave & 1) + lane] = stat_in ? stat : -INFINITY; };
    if (i0 < i1) stage(i0, smem + (i0 & 1) * C::BUF);
    gb_own_rows<WT, D>(P.k_rot + (((size_t)seq * P.nkv + hk) * P.rows + (size_t)key * K1) * D * ESZ, half, keys.kf);
    if constexpr (C::V_LDS) {
        const int first = min(w0, P.T - 1);                  // (either row wavefront brings in half of the rows)
        gb_stage<WT, D, 2>(P.v + (((size_t)seq * P.rows + (size_t)first * K1) * P.nkv + hk) * D * ESZ, K1 * vstride, P.T - 1 - first, smem + C::OFF_V + kw * Tile::BYTES, rw, lane);
        keys.v_tile = smem + C::OFF_V + kw * Tile::BYTES;
    } else {
        gb_own_rows<WT, D>(P.v + (((size_t)seq * P.rows + (size_t)key * K1) * P.nkv + hk) * D * ESZ, half, keys.vf);
    }
    if (i0 < i1) stage_stats(i0);
    // (the compiler's own loads end here: it would wait for them in the loop, and with them for the requests that it does not know)
    for (uint4& x : keys.kf) asm volatile("" : "+v"(x.x), "+v"(x.y), "+v"(x.z), "+v"(x.w));
    if constexpr (!C::V_LDS)
        for (uint4& x : keys.vf) asm volatile("" : "+v"(x.x), "+v"(x.y), "+v"(x.z), "+v"(x.w));
    gb_arrived();
    // (restrict: as in gb_dq_kernel)
    auto products = [&](int i, int first, auto masked, const char* __restrict buf, char* __restrict next) __attribute__((always_inline)) {
        const float* stats = reinterpret_cast<const float*>(buf + C::OFF_S) + 32 * rw;
        if constexpr (masked) {
            stage(i + 1, next);
            if (w0 < P.T && first + 31 >= w0 * K1) keys.template step<true>(L, buf + rw * C::SET, stats, 64, half, key * K1 - first - 4 * half, 31, [] {});
        } else {
            keys.template step<false>(L, buf + rw * C::SET, stats, 64, half, 0, 31, [&]() __attribute__((always_inline)) { stage(i + 1, next); });
        }
    };
    auto step = [&](int i, int first, auto masked) __attribute__((always_inline)) {
        products(i, first, masked, smem + (i & 1) * C::BUF, smem + (1 - (i & 1)) * C::BUF);
        stage_stats(i + 1);
        gb_arrived();
    };
    // of every head the row tiles that see some of the wavefront's keys, then those that see all of them
    const int see_all = w0 < P.T ? min(max((w0 + 31) * K1 - first_row - 32 * rw + 63, 0) / 64, per_head) : per_head;
    for (int i = i0, j = next_j0; i < i1; j = 0) {
        const int head0 = i - j;
        for (const int end = min(i1, head0 + see_all); i < end; ++i) step(i, first_row + 64 * (i - head0) + 32 * rw, std::true_type{});
        for (const int end = min(i1, head0 + per_head); i < end; ++i) step(i, first_row + 64 * (i - head0) + 32 * rw, std::false_type{});
    }
    if (__builtin_expect(gb_odd_rows(keys.dk), 0)) gb_add_odd_rows<WT, D>(P, seq, hk, key * K1, min((w0 + 31) * K1 + 30, P.rows - 1), half, keys.dk, keys.dv);   // (the last row of a masked tile)
    // ---- the row wavefronts' sums, one gradient after the other by way of the LDS
    auto meet = [&](f32x16 (&y)[NJ]) __attribute__((always_inline)) {
        f32x4* area = reinterpret_cast<f32x4*>(smem) + kw * NJ * 4 * 64 + lane;
        if (rw) {
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) area[(j * 4 + q) * 64] = f32x4{y[j][4 * q], y[j][4 * q + 1], y[j][4 * q + 2], y[j][4 * q + 3]};
        }
        __syncthreads();
        if (!rw) {
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const f32x4 v = area[(j * 4 + q) * 64];
#pragma unroll
                    for (int e = 0; e < 4; ++e) y[j][4 * q + e] += v[e];
                }
        }
        __syncthreads();
    };
    meet(keys.dk);
    meet(keys.dv);
    if (rw) return;
    if (W.splits > 1) {
        // [tile of 32 keys][split][dk, dv][NJ * 4][64 lanes] of 16 bytes
        f32x4* to = reinterpret_cast<f32x4*>(W.partial) + (((size_t)(kt * W.heads + head) * KW + kw) * W.splits + split) * (2 * NJ * 4 * 64) + lane;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const f32x16 &a = keys.dk[j], &b = keys.dv[j];
                to[(j * 4 + q) * 64] = f32x4{a[4 * q], a[4 * q + 1], a[4 * q + 2], a[4 * q + 3]};
                to[((NJ + j) * 4 + q) * 64] = f32x4{b[4 * q], b[4 * q + 1], b[4 * q + 2], b[4 * q + 3]};
            }
        return;
    }
    if (w0 + c < P.T) gb_write_keys<WT, D>(P, seq, hk, key * K1, key, half, keys.dk, keys.dv);
}

// The parts' sums, added in order.  A workgroup takes a tile of 32 keys, a wavefront one gradient's column blocks j and j + NJ / 2, which
// the rotation mixes
template <typename WT, int D>
__global__ void __launch_bounds__(D * 2) gb_merge_kernel(const GbParams P, const GbWork W, int keys_wg) {
    constexpr int ESZ = Traits<WT>::ESZ, NJ = D / 32, PART = 2 * NJ * 4 * 64;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 31, half = lane >> 5, per_wg = keys_wg / 32;
    const int which = wave / (NJ / 2), j0 = wave % (NJ / 2);   // dk, dv
    const int sub = blockIdx.x % per_wg, unit = blockIdx.x / per_wg, kt = unit / W.heads, head = unit - kt * W.heads, seq = head / P.nkv, hk = head - seq * P.nkv;
    const int key = kt * keys_wg + 32 * sub + c;
    if (key >= P.T) return;
    const f32x4* from = reinterpret_cast<const f32x4*>(W.partial) + (size_t)blockIdx.x * W.splits * PART + (which * NJ + j0) * 4 * 64 + lane;
    f32x4 a[4], b[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) { a[u] = f32x4{0.f, 0.f, 0.f, 0.f}; b[u] = a[u]; }
#pragma unroll 2
    for (int i = 0; i < W.splits; ++i, from += PART)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            a[u] += from[u * 64];
            b[u] += from[(NJ / 2 * 4 + u) * 64];
        }
    char* row = (which ? P.d_v : P.d_k) + (((size_t)seq * P.rows + (size_t)key * (P.k + 1)) * P.nkv + hk) * D * ESZ;
#pragma unroll
    for (int u = 0; u < 4; ++u) gb_write4<WT, D>(row, which ? nullptr : P.table + (size_t)key * (D / 2), 32 * j0 + 8 * u + 4 * half, which ? 1.f : GB_LN2, a[u], b[u]);
}

// The checks are those of ps_group_attention; and a launch's threads (256 per 128 query rows, up to 512 per tile of keys) are counted in 32 bits:
// as many query rows fill the memory, and as many key tiles take tens of thousands of sequences of a few tokens with a hundred kv heads
int check(const ps_group_attn_grad_args* a) {
    if (!a) return PS_ERR_NULL;
    ps_group_attn_args f = {};
    f.seqs = a->seqs; f.tokens = a->tokens; f.k = a->k; f.n_heads = a->n_heads; f.n_kv_heads = a->n_kv_heads;
    f.head_dim = a->head_dim; f.dtype = a->dtype; f.rope_base = a->rope_base;
    const int st = ga_check(&f);
    if (st != PS_OK) return st;
    const long long rows = (long long)a->tokens * (a->k + 1), heads = (long long)a->seqs * a->n_kv_heads, gpt = 32 / (a->k + 1);
    const long long row_wgs = (rows + GB_ROWS - 1) / GB_ROWS * a->n_heads, key_wgs = heads * ((a->tokens + 63) / 64 + (a->tokens / gpt + 4) / 4) + 1024;
    return row_wgs >= 1 << 24 || key_wgs >= 1 << 23 ? PS_ERR_UNSUPPORTED : PS_OK;
}

// How a call is cut: wavefronts that share 32 query rows; keys of a workgroup, parts of their rows
struct GbPlan { int kw, keys, heads, tiles, splits; };
GbPlan plan(const ps_group_attn_grad_args* a) {
    GbPlan L;
    const bool bf = a->dtype == PS_BF16, d128 = a->head_dim == 128;
    // Two wavefronts for 32 query rows where four rows' workgroups would leave compute units without one.  Whole calls, us, one / two:
    // T 64, k 4, 8 heads x 64 (24 workgroups) 30 / 29, T 1000, k 2 (192) 63 / 56, float32 2 x T 300, k 3 (160) 89 / 85; but 8 x T 128, k 3, 8 heads x 128
    // (256) 64 / 68, T 203, k 5, 40 heads (400) 101 / 109
    const long long row_blocks = ((long long)a->tokens * (a->k + 1) + GB_ROWS - 1) / GB_ROWS * a->n_heads * a->seqs;
    L.kw = row_blocks < 256 ? 2 : 1;
    // 128 keys per workgroup at head_dim 128 in bf16; 64 where two wavefronts per SIMD do not fit (float32), or, at head_dim 64, where there are few
    // (64 / 128: T 1000, k 2, 8 heads 56 / 59, float32 2 x T 300 84 / 94)
    L.heads = a->n_kv_heads * a->seqs;
    L.keys = d128 ? (bf ? 128 : 64) : (long long)((a->tokens + 127) / 128) * L.heads >= 256 ? 128 : 64;
    L.tiles = (a->tokens + L.keys - 1) / L.keys;
    // Parts of a key tile's rows, for a workgroup on every compute unit (two where the LDS takes two) as long as a part has a few stages of 64
    // rows, for twice as many where parts stay long: a causal call's key tiles are unlike each other.  Whole calls, us, parts 1 / 2 / 3 / 4 / 8:
    // T 2048, k 4, 32 heads (512 tiles) 1042 / 1067 / 1123 / 1140 / 1283; 4 x T 1024, k 8, 32 / 8 heads (256) 2470 / 2311 / 2333 / 2351 / 2436; T 203, k 5,
    // 40 heads (80) 123 / 104 / 103 / 108 / 120; T 512, k 4, 32 / 8 heads (32) 455 / 270 / 223 / 181 / 156
    const long long units = (long long)L.tiles * L.heads, places = d128 || L.keys == 128 ? 256 : 512;
    const long long stages = ((long long)a->tokens * (a->k + 1) + 63) / 64 * (a->n_heads / a->n_kv_heads);
    L.splits = (int)std::max(1LL, std::max(std::min(places / units, stages / (bf && d128 ? 4 : 2)), std::min(2 * places / units, stages / 64)));
    return L;
}

struct GbLayout { size_t table, k_rot, q_rot, stats, partial, total; };
GbLayout layout(const ps_group_attn_grad_args* a) {
    GbLayout L;
    const bool bf = a->dtype == PS_BF16;
    const size_t rows = (size_t)a->seqs * a->tokens * (a->k + 1), row = (size_t)a->head_dim * (bf ? 2 : 4);
    const GbPlan G = plan(a);
    L.table = 0;
    L.k_rot = a256((size_t)(a->tokens + a->k) * (a->head_dim / 2) * sizeof(float2));
    L.q_rot = L.k_rot + a256(rows * a->n_kv_heads * row);
    L.stats = L.q_rot + a256(rows * a->n_heads * row * (bf ? 2 : 1));
    L.partial = L.stats + 2 * a256(rows * a->n_heads * sizeof(float));
    L.total = L.partial + (G.splits > 1 ? (size_t)G.tiles * G.heads * G.splits * G.keys * a->head_dim * 2 * sizeof(float) : 0);
    return L;
}

template <typename WT, int D, int KW> void launch_keys(const GbParams& P, const GbPlan& G, GbWork W, hipStream_t s) {
    typedef GbDkv<WT, D, KW> C;
    const unsigned own = (unsigned)((W.own_tiles + C::OWNERS - 1) / C::OWNERS);
    hipLaunchKernelGGL((gb_dkv_kernel<WT, D, KW>), dim3((unsigned)(W.units * W.splits) + own), dim3(C::WAVES * 64), 0, s, P, W);
    if (W.splits > 1) hipLaunchKernelGGL((gb_merge_kernel<WT, D>), dim3(W.units * KW), dim3(D * 2), 0, s, P, W, G.keys);
}

template <typename WT, int D> int launch(const GbParams& P, const GbPlan& G, float* partial, hipStream_t s) {
    // (as ga_rope_kernel: where positions are few, several workgroups of at most one item per thread share one)
    const long long items = (long long)P.seqs * P.nkv * (D / 8) * (P.k + 1);
    hipLaunchKernelGGL((gb_prep_kernel<WT, D>), dim3(P.T + P.k, (unsigned)std::max(1LL, std::min((items + 255) / 256, 2048LL / (P.T + P.k)))), dim3(256), 0, s, P);
    const dim3 grid(P.nq * ((P.rows + GB_ROWS / G.kw - 1) / (GB_ROWS / G.kw)), P.seqs);
    if (G.kw == 2) hipLaunchKernelGGL((gb_dq_kernel<WT, D, 2>), grid, dim3(GB_THREADS), 0, s, P);
    else hipLaunchKernelGGL((gb_dq_kernel<WT, D, 1>), grid, dim3(GB_THREADS), 0, s, P);
    const GbWork W = {G.heads, G.splits, G.tiles * G.heads, P.k > 0 ? (P.T + P.gpt - 1) / P.gpt * G.heads : 0, partial};
    if constexpr (D == 128) {
        launch_keys<WT, D, Traits<WT>::BF ? 4 : 2>(P, G, W, s);
    } else {
        if (G.keys == 64) launch_keys<WT, D, 2>(P, G, W, s);
        else launch_keys<WT, D, 4>(P, G, W, s);
    }
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
    P.table = (float2*)(ws + L.table); P.k_rot = ws + L.k_rot; P.q_rot = ws + L.q_rot; P.lse2 = (float*)(ws + L.stats);
    P.delta = (float*)(ws + L.stats + (L.partial - L.stats) / 2);
    hipStream_t s = (hipStream_t)stream;
    const GbPlan G = plan(a);
    float* partial = (float*)(ws + L.partial);
    if (a->dtype == PS_BF16) return a->head_dim == 128 ? launch<bf16_t, 128>(P, G, partial, s) : launch<bf16_t, 64>(P, G, partial, s);
    return a->head_dim == 128 ? launch<float, 128>(P, G, partial, s) : launch<float, 64>(P, G, partial, s);
}

// see ps_draft_debug.h
extern "C" int ps_train_debug_grad_plan(const ps_group_attn_grad_args* a, int* out) {
    const int st = check(a);
    if (st != PS_OK) return st;
    if (!out) return PS_ERR_NULL;
    const GbPlan L = plan(a);
    out[0] = L.kw; out[1] = L.keys; out[2] = L.splits;
    return PS_OK;
}

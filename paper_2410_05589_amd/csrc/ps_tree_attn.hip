// Attention of a draft tree's rows over the target's 8-bit cache and over the tree's own keys and values (see include/ps_verify.h).
//
//   S = scale q K^T,  P = exp(S - m),  out = P V / sum P,  K = k_scale code, V = v_scale code per block of 32 positions
//
// e4m3 codes are bf16 numbers, so both products run on v_mfma_f32_32x32x16_bf16 with exact keys and values; the scales are powers of two:
// the keys' join the scores' constant, the values' come in with the conversion of their codes.  Queries stand along the lanes: S^T = K Q^T leaves a lane (query c, half h) the
// scores of positions 8 a + 4 h + b, and out^T = V^T P^T takes them from there as its operand: the cache keeps values in just that order, so
// codes go from memory to the matrix cores through a conversion (two codes an instruction), with no exchange between lanes.
// The running maximum is raised only when a score passes it by 2^8 (sums stay far inside float32), so sums are rarely rescaled.
//
// Probabilities are rounded to bf16 for the second product (their sum is taken before that, in float32): a row's error is then that of many independent
// roundings, below its result's own.  (Of the 2-norm, with the result's rounding: 0.0020 ... 0.0023; with probabilities in two parts 0.00165, the result's rounding alone, at 137 us
// in the place of 107 for 8 x 61 nodes over 4099 ... 12288 positions, 46.8 / 45.8 for 4 x 32768.)  float32 calls have three bf16 parts of queries and probabilities, 24 bits of each.
//
// Work: a sequence's blocks are cut into splits of `per` blocks; a workgroup takes a split of one kv head for up to four tiles of 32 rows (a row is a node and one of
// the heads that share the kv head).  Its wavefronts divide tiles (WR) and blocks (WK); those that share a tile meet in LDS, splits in the workspace and a
// second kernel.  One and two tiles: eight wavefronts, each with its blocks on their way to its registers; more: four, which read the same blocks from LDS.
//
// What bounds it (bf16, head_dim 128).  One tile: reading the codes.  32 sequences of 2048 positions, 32 heads, a row each: 537 MB in 87 us, 6.2 TB/s; 4 of 32768
// positions, 8 heads, 4 rows each: 268 MB in 46.  Many tiles: a block of one tile is 16 matrix instructions (512 cycles), 64 conversions, 16 exponentials
// and some 100 more vector instructions, which overlap with the products less than the two wavefronts of a SIMD could make them: 1600 cycles.  8 x 4099 ...
// 12288 positions, 61 nodes, 32 heads that share 8: 89 us, 0.74 PFLOP/s.  Left out in probes of that: conversions -6 %, exponentials -12 %, barriers and requests
// -20 %, all of these -30 %.  Small calls: 2 us until the first operands are there, 2 for the tree's own rows, 2 for the meeting and the results, then the join (3).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ps_cache_device.h"

namespace {

constexpr int TA_TILE = 32;
// wavefronts of a workgroup.  bf16: two per SIMD, so that one's matrix instructions run beside the other's exponentials, of one workgroup or, where
// wavefronts wait for each other's requests (WR 4), of two; float32 has three parts of every query and one wavefront per SIMD.  (Two tiles and
// less, eight / twice four, us: 52 rows of 8 x 8192 positions, 8 heads 38 / 45, of 2048 positions 17 / 21; 61 rows, 32 heads, 8 x 2048 42 / 49; one row 15.5 / 15.1)
template <typename WT, int WR> constexpr int ta_waves() { return Traits<WT>::BF && WR < 4 ? 8 : 4; }
// How far (in powers of two) scores may pass the maximum that they are taken against: probabilities stay below 2^8, their sums over 2^30 positions below 2^38.  (A maximum
// that is raised with every score above it: 4 % of the time with many tiles)
constexpr float TA_LAZY = 8.f;
// Sums of values are held times this, so that probabilities of up to 2^8 of the largest floats stay floats (2^-12: sixteen of them): cached values by their scale
// (2^-100 and above: still exact), own ones by their probabilities
constexpr float TA_HELD = 0x1p-12f, TA_HELD_LOG = -12.f;

struct TaParams {
    const char *q, *k, *v;
    char* out;
    float *lse, *part;
    const uint8_t *k_codes, *v_codes;
    const float *k_scale, *v_scale;
    long long q_row, kv_row;        // bytes between rows
    int n_heads, heads, grp, nodes, rows, tiles;   // rows = nodes * grp; tiles of 32 of them
    int batch, per;                 // blocks per split
    int stream;                     // codes pass the caches by
    float c;                        // scale * log2(e)
    const int* len_dev;
    unsigned first[PC_SEQS];
    int len[PC_SEQS];
    int split0[PC_SEQS + 1];        // the sequence's first split
    u64 sees[PS_TREE_MAX_NODES];    // bit t: node t is the node itself or an ancestor
};

template <int D> struct Tile { uint4 k[D / 32], v[D / 32]; };

// 8 codes times a power of two as bf16 (exact for 2^-124 and above)
__device__ __forceinline__ bf16x8 widen8(unsigned lo, unsigned hi, float scale) {
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    const b2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const b2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ __forceinline__ unsigned word(uint4 v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// 8 floats as NP bf16 parts (three: all 24 bits)
template <int NP> __device__ __forceinline__ void split8(const float (&x)[8], bf16x8 (&out)[NP]) {
    float rest[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) rest[i] = x[i];
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        unsigned w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = pack_bf16x2(rest[2 * i], rest[2 * i + 1]);
            rest[2 * i] -= __uint_as_float(w[i] << 16);
            rest[2 * i + 1] -= __uint_as_float(w[i] & 0xFFFF0000u);
        }
        out[p] = __builtin_bit_cast(bf16x8, make_uint4(w[0], w[1], w[2], w[3]));
    }
}
// 8 consecutive elements of a row
template <typename WT, int NP> __device__ __forceinline__ void load_parts(const char* p, bool valid, bf16x8 (&out)[NP]) {
    if constexpr (Traits<WT>::BF) {
        out[0] = __builtin_bit_cast(bf16x8, valid ? ld16_q(p) : make_uint4(0, 0, 0, 0));
    } else {
        float x[8];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const f32x4 v = valid ? load4_q<WT>(p + 16 * i) : f32x4{0, 0, 0, 0};
#pragma unroll
            for (int e = 0; e < 4; ++e) x[4 * i + e] = v[e];
        }
        split8(x, out);
    }
}
template <typename WT> __device__ __forceinline__ float load1(const char* p) {
    if constexpr (Traits<WT>::BF) return bf16_to_f32(*reinterpret_cast<const uint16_t*>(p));
    else return *reinterpret_cast<const float*>(p);
}

// the other half's value (lane ^ 32)
__device__ __forceinline__ float other_half(float v) {
    const unsigned u = __float_as_uint(v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return __uint_as_float(threadIdx.x & 32 ? r[0] : r[1]);
}

// What a wavefront has of one tile of 32 rows: lane (row c, half h) has of every 32 dims the dims 8 a + 4 h + b as o[.][4 a + b] (times TA_HELD)
template <int D> struct RowState {
    f32x16 o[D / 32];
    float m, l;                     // maximum (in powers of two), this half's sum
};

// What makes a block's products powers of two; a float: keys above 2^100 and a scale above 1 would make it Inf, and a product of zero NaN
__device__ __forceinline__ float score_factor(float c, float k_scale) { return __builtin_fminf(c * k_scale, 3.4028234663852886e38f); }

// One tile of 32 keys: scores (raw products) to probabilities against the running maximum.  c: what makes products powers of two.  (The values' scale is no part of
// them: with a block's 2^-100, zeros' scale, those below 2^-26 would not be in the sum)
template <int D, int NB> __device__ __forceinline__ void raise_maximum(RowState<D>& R, const f32x16 (&s)[NB], const float (&c)[NB]) {
    float mx = -__builtin_inff();
#pragma unroll
    for (int n = 0; n < NB; ++n) {
        float x = s[n][0];
#pragma unroll
        for (int i = 1; i < 16; ++i) x = fmaxf(x, s[n][i]);
        mx = fmaxf(mx, x * c[n]);
    }
    mx = fmaxf(mx, other_half(mx));
    if (__ballot(mx > R.m + TA_LAZY)) {
        const float m = fmaxf(R.m, mx), alpha = m > R.m ? __builtin_amdgcn_exp2f(R.m - m) : 1.f;
        R.m = m;
        R.l *= alpha;
#pragma unroll
        for (int j = 0; j < D / 32; ++j) R.o[j] *= alpha;
    }
}
template <int D, bool OWN> __device__ __forceinline__ void exponentials(RowState<D>& R, f32x16& s, float c) {
    const float off = (R.m == -__builtin_inff() ? 0.f : R.m) - (OWN ? TA_HELD_LOG : 0.f);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        s[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], c, -off));
        sum += s[i];
    }
    R.l = OWN ? __builtin_fmaf(sum, 1.f / TA_HELD, R.l) : R.l + sum;
}
template <int NP> __device__ __forceinline__ void prob_parts(const f32x16& s, bf16x8 (&p)[2][NP]) {
#pragma unroll
    for (int st = 0; st < 2; ++st) {
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = s[8 * st + e];
        split8(x, p[st]);
    }
}

template <typename WT> __device__ __forceinline__ void store4_out(char* p, f32x4 x) {
    if constexpr (Traits<WT>::BF) *reinterpret_cast<u32x2_q*>(p) = u32x2{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
    else *reinterpret_cast<f32x4_q*>(p) = x;
}
__device__ __forceinline__ float log_sum(float m, float l) { return l == 0.f ? -__builtin_inff() : 0.69314718055994530942f * (m + __log2f(l)); }

// what a wavefront leaves in LDS of its tile: sums by row, maxima, row sums
template <int D> struct Meet {
    float o[TA_TILE][D + 4];
    float m[TA_TILE], l[TA_TILE];
};

// The parts of a block's attention: products with its keys, ...
template <int D, int NP> __device__ __forceinline__ void key_products(const bf16x8 (&q)[D / 16][NP], const uint4 (&k)[D / 32], f32x16& s) {
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const bf16x8 kf = widen8(word(k[c], 2 * u), word(k[c], 2 * u + 1), 1.f);
#pragma unroll
            for (int p = NP - 1; p >= 0; --p) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, q[2 * c + u][p], s, 0, 0, 0);
        }
}
// ... positions from `tail` on hidden, and their codes, which may be no numbers, zero, ...
template <int D> __device__ __forceinline__ void hide(f32x16& s, uint4 (&v)[D / 32], int tail) {
    const int half = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = 8 * (e >> 2) + 4 * half + (e & 3) < tail ? s[e] : -__builtin_inff();
    unsigned keep[4];
#pragma unroll
    for (int a = 0; a < 4; ++a) {
        const int n = min(max(tail - 8 * a - 4 * half, 0), 4);
        keep[a] = n == 4 ? 0xFFFFFFFFu : (1u << (8 * n)) - 1u;
    }
#pragma unroll
    for (int c = 0; c < D / 32; ++c) v[c] = make_uint4(v[c].x & keep[0], v[c].y & keep[1], v[c].z & keep[2], v[c].w & keep[3]);
}
// ... products with its values
template <int D, int NP> __device__ __forceinline__ void value_products(RowState<D>& R, const f32x16& s, const uint4 (&v)[D / 32], float scale) {
    bf16x8 p[2][NP];
    prob_parts<NP>(s, p);
#pragma unroll
    for (int j = 0; j < D / 32; ++j)
#pragma unroll
        for (int st = 0; st < 2; ++st) {
            const bf16x8 vf = widen8(word(v[j], 2 * st), word(v[j], 2 * st + 1), scale);
#pragma unroll
            for (int n = NP - 1; n >= 0; --n) R.o[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf, p[st][n], R.o[j], 0, 0, 0);
        }
}

// Four tiles of rows: four wavefronts read the same blocks, which come to LDS by way of the memory unit, 1 KiB per request, two steps of
// TA_STEP blocks ahead in three buffers (arrays of their own: a read from one need not wait for what is on its way into another).  A step's
// blocks are taken together: two chains of products, one look at the maximum.  Each wavefront asks for a quarter of a step
// (and, so that all wait for as many requests, for scales: those of the first two are read).
constexpr int TA_STEP = 2;
typedef __attribute__((address_space(3))) void lds_void;
template <int D> struct Stage {
    char codes[TA_STEP * 2 * PC_BLOCK * D];
    float scales[4][64];
};

template <typename WT, int D, int WR>
__global__ __launch_bounds__((64 * ta_waves<WT, WR>()), (Traits<WT>::BF ? 2 : 1)) void tree_attn_kernel(const TaParams P) {
    constexpr int W = ta_waves<WT, WR>(), WK = W / WR, NP = Traits<WT>::BF ? 1 : 3, C = D / 32, TILE = PC_BLOCK * D, ESZ = Traits<WT>::ESZ;
    constexpr bool STAGED = Traits<WT>::BF && WR == 4;
    // where wavefronts that share rows meet, and before that a wavefront's probabilities of its own rows (staged, where it is large enough: the
    // buffer that is requested last)
    constexpr bool OWN_IN_BUFFER = STAGED && sizeof(Stage<D>::codes) >= W * PC_BLOCK * TA_TILE * 4;
    __shared__ __attribute__((aligned(16))) Meet<(WK > 1 ? D : OWN_IN_BUFFER ? 0 : TA_TILE)> s_meet[W];
    __shared__ __attribute__((aligned(16))) Stage<STAGED ? D : 0> b0, b1, b2;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, lc = lane & 31;
    const int wr = wave % WR, wk = wave / WR, h = blockIdx.y;
    const int b = __popcll(__ballot(lane < P.batch && P.split0[lane + 1] <= (int)blockIdx.x));   // the sequence whose split this is
    const int split = blockIdx.x - P.split0[b], splits = P.split0[b + 1] - P.split0[b];
    const int len = pc_length(P.len_dev, b, P.len[b]), blocks = (len + 31) >> 5, tail = len & 31;
    const int tile = (int)blockIdx.z * WR + wr;              // this wavefront's rows
    const bool active = tile < P.tiles;
    const int begin = split * P.per, end = min(blocks, begin + P.per);
    const size_t seq0 = (size_t)P.first[b] * P.heads + h;
    const bool own = P.k && split == splits - 1;             // the tree's own rows are this workgroup's
    const int row = tile * TA_TILE + lc;
    const bool valid = row < P.rows;
    const int node = valid ? row / P.grp : 0, head = h * P.grp + (valid ? row % P.grp : 0);
    const u64 sees = own ? P.sees[node] : 0;

    // the tree's own values, where this workgroup takes them: in LDS by node, zeros in the place of Inf and NaN (s_odd: there were any)
    constexpr int OWN_PITCH = D * ESZ + 4 * ESZ;
    __shared__ __attribute__((aligned(16))) char s_own[PS_TREE_MAX_NODES * OWN_PITCH];
    __shared__ int s_odd[W];
    const char* own_k = P.k + (long long)b * P.nodes * P.kv_row + (long long)h * D * ESZ;
    const char* own_v = P.v + (long long)b * P.nodes * P.kv_row + (long long)h * D * ESZ;
    constexpr int OWN_PIECES = PS_TREE_MAX_NODES * (D / 8) / (64 * W);   // of 8 elements, per thread; nodes up to a tile's end: zeros
    f32x4 own_raw[OWN_PIECES][2];
    auto fetch_own = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < OWN_PIECES; ++n) {
            const int i = n * 64 * W + threadIdx.x, at = i / (D / 8), part = i % (D / 8);
            own_raw[n][0] = own_raw[n][1] = f32x4{0, 0, 0, 0};
            if (at < P.nodes) {
                const char* from = own_v + (long long)at * P.kv_row + part * 8 * ESZ;
                own_raw[n][0] = load4_q<WT>(from);
                own_raw[n][1] = load4_q<WT>(from + 4 * ESZ);
            }
        }
    };
    auto place_own = [&]() __attribute__((always_inline)) {
        bool odd = false;
#pragma unroll
        for (int n = 0; n < OWN_PIECES; ++n) {
            const int i = n * 64 * W + threadIdx.x, at = i / (D / 8), part = i % (D / 8);
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float v = own_raw[n][e >> 2][e & 3];
                const bool fine = __builtin_fabsf(v) < __builtin_inff();
                odd |= !fine;
                x[e] = fine ? v : 0.f;
            }
            char* to = s_own + at * OWN_PITCH + part * 8 * ESZ;
            if constexpr (Traits<WT>::BF) {
                *reinterpret_cast<u32x2*>(to) = u32x2{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])};
                *reinterpret_cast<u32x2*>(to + 8) = u32x2{pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
            } else {
                *reinterpret_cast<f32x4*>(to) = f32x4{x[0], x[1], x[2], x[3]};
                *reinterpret_cast<f32x4*>(to + 16) = f32x4{x[4], x[5], x[6], x[7]};
            }
        }
        odd = __ballot(odd) != 0;
        if (lane == 0) s_odd[wave] = odd;
    };

    bf16x8 q[2 * C][NP];
    RowState<D> R;
    auto load_rows = [&]() __attribute__((always_inline)) {
        const char* from = P.q + ((long long)b * P.nodes + node) * P.q_row + (long long)head * D * ESZ;
#pragma unroll
        for (int f = 0; f < 2 * C; ++f) load_parts<WT, NP>(from + (32 * (f >> 1) + 16 * half + 8 * (f & 1)) * ESZ, valid, q[f]);
        R.m = -__builtin_inff();
        R.l = 0.f;
#pragma unroll
        for (int j = 0; j < C; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) R.o[j][e] = 0.f;
    };
    // the tree's own rows, in the sequence's last split, while the first blocks are on their way: tiles of 32 nodes
    auto own_rows = [&]() __attribute__((always_inline)) {
        bf16x8 k0[2 * C][NP];
        auto load_keys = [&](int kt) __attribute__((always_inline)) {
            const int key = kt * 32 + lc;
#pragma unroll
            for (int f = 0; f < 2 * C; ++f)
                load_parts<WT, NP>(own_k + (long long)key * P.kv_row + (32 * (f >> 1) + 16 * half + 8 * (f & 1)) * ESZ, key < P.nodes, k0[f]);
        };
        const int first = wk;
        load_keys(first);
        place_own();
        __syncthreads();
        if (!active) return;
        const bool any_odd = __ballot(lane < W && s_odd[lane % W]) != 0;
        for (int kt = first; kt * 32 < P.nodes; kt += WK) {
            if (kt != first) load_keys(kt);
            {
                f32x16 s;
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
                for (int f = 0; f < 2 * C; ++f)
#pragma unroll
                    for (int x = NP - 1; x >= 0; --x)        // (parts whose product is below 2^-24 of the whole are left out)
#pragma unroll
                        for (int y = NP - 1 - x; y >= 0; --y) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k0[f][x], q[f][y], s, 0, 0, 0);
                const unsigned seen = (unsigned)(sees >> (32 * kt));
#pragma unroll
                for (int e = 0; e < 16; ++e) s[e] = (seen >> (8 * (e >> 2) + 4 * half + (e & 3))) & 1 ? s[e] : -__builtin_inff();
                f32x16 one[1] = {s};
                const float c1[1] = {P.c};
                raise_maximum<D, 1>(R, one, c1);
                exponentials<D, true>(R, s, P.c);
                bf16x8 p[2][NP];
                prob_parts<NP>(s, p);
#pragma unroll
                for (int j = 0; j < C; ++j)
#pragma unroll
                    for (int st = 0; st < 2; ++st) {
                        float x[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[e] = load1<WT>(s_own + (kt * 32 + 8 * (2 * st + (e >> 2)) + 4 * half + (e & 3)) * OWN_PITCH + (32 * j + lc) * ESZ);
                        bf16x8 vf[NP];
                        split8(x, vf);
#pragma unroll
                        for (int a = NP - 1; a >= 0; --a)
#pragma unroll
                            for (int c = NP - 1 - a; c >= 0; --c) R.o[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[a], p[st][c], R.o[j], 0, 0, 0);
                    }
                if (any_odd) {                               // what is Inf or NaN, for the rows that see it
                    float* sp = OWN_IN_BUFFER ? reinterpret_cast<float*>(b2.codes) + wave * PC_BLOCK * TA_TILE : reinterpret_cast<float*>(s_meet + wave);   // probabilities by node
#pragma unroll
                    for (int e = 0; e < 16; ++e) sp[(8 * (e >> 2) + 4 * half + (e & 3)) * TA_TILE + lc] = s[e];
                    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                    __builtin_amdgcn_wave_barrier();
                    for (int t = 0; t < 32 && kt * 32 + t < P.nodes; ++t) {
                        const float pt = sp[t * TA_TILE + lc];
                        const bool see = (seen >> t) & 1;
#pragma unroll
                        for (int j = 0; j < C; ++j)
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                const float v = load1<WT>(own_v + (long long)(kt * 32 + t) * P.kv_row + (32 * j + 8 * (e >> 2) + 4 * half + (e & 3)) * ESZ);
                                if (see && !(__builtin_fabsf(v) < __builtin_inff())) R.o[j][e] += pt * v;
                            }
                    }
                    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
                    __builtin_amdgcn_wave_barrier();
                }
            }
        }
    };
    if constexpr (STAGED) {
        constexpr int PIECES = TA_STEP * 2 * C / W;          // requests of 1 KiB per wavefront and step
        const int steps = (end - begin + TA_STEP - 1) / TA_STEP;
        // (offsets inside a split are 32 bits: the plan sees to that)
        const size_t at0 = seq0 + (size_t)begin * P.heads;
        const rsrc_t from_k = make_rsrc(P.k_codes + at0 * TILE), from_v = make_rsrc(P.v_codes + at0 * TILE);
        const rsrc_t from_ks = make_rsrc(P.k_scale + at0), from_vs = make_rsrc(P.v_scale + at0);
        auto request = [&](int step, Stage<D>& to) __attribute__((always_inline)) {
            const int first = step * TA_STEP, most = end - begin - 1;
#pragma unroll
            for (int r = 0; r < PIECES; ++r) {
                const int piece = wave * PIECES + r, block = min(first + piece / (2 * C), most), part = piece % (2 * C);   // keys' C pieces, then values'
                __builtin_amdgcn_raw_ptr_buffer_load_lds(part < C ? from_k : from_v, (lds_void*)(to.codes + piece * 1024), 16, lane * 16,
                                                         (unsigned)block * P.heads * TILE + (part % C) * 1024, 0, 0);
            }
            const unsigned off = (unsigned)min(first + lane, most) * P.heads * 4;   // (lane i: the step's block i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(wave & 1 ? from_vs : from_ks, (lds_void*)to.scales[wave], 4, off, 0, 0, 0);
        };
        auto step = [&](int k, Stage<D>& mine, Stage<D>& last) __attribute__((always_inline)) {
            // this step's requests have arrived (the step's behind it may be on their way), and everyone is done with the last one's buffer
            static_assert(PIECES == 2 || PIECES == 4, "one step of PIECES + 1 requests");
            if constexpr (PIECES == 4) asm volatile("s_waitcnt vmcnt(5) lgkmcnt(0)" ::: "memory");
            else asm volatile("s_waitcnt vmcnt(3) lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
            request(k + 2, last);
            const int i = begin + k * TA_STEP;
            if (!active) return;
            f32x16 x[2];
            uint4 t[2][C];
            float cs[2], vs[2];
#pragma unroll
            for (int n = 0; n < 2; ++n) {
#pragma unroll
                for (int c = 0; c < C; ++c) t[n][c] = ld16(mine.codes + (n * 2 * C + c) * 1024 + lane * 16);
                cs[n] = score_factor(P.c, mine.scales[0][n]);
                vs[n] = mine.scales[1][n] * TA_HELD;
            }
#pragma unroll
            for (int n = 0; n < 2; ++n) key_products<D, NP>(q, t[n], x[n]);
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int c = 0; c < C; ++c) t[n][c] = ld16(mine.codes + (n * 2 * C + C + c) * 1024 + lane * 16);
            if (i + 2 >= end) {                              // (the second one may be behind the split's end, either the sequence's last)
#pragma unroll
                for (int n = 0; n < 2; ++n)
                    if (i + n >= end) hide<D>(x[n], t[n], 0);
                    else if (tail && i + n == blocks - 1) hide<D>(x[n], t[n], tail);
            }
            raise_maximum<D, 2>(R, x, cs);
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                exponentials<D, false>(R, x[n], cs[n]);
                value_products<D, NP>(R, x[n], t[n], vs[n]);
            }
        };
        if (steps > 0) {
            request(0, b0);
            request(1, b1);
        }
        if (own) fetch_own();
        load_rows();
        if (own) own_rows();
        for (int k = 0; k < steps;) {
            step(k, b0, b2);
            if (++k >= steps) break;
            step(k, b1, b0);
            if (++k >= steps) break;
            step(k, b2, b1);
            ++k;
        }
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");   // (nothing is on its way to LDS any more)
    } else {
        // a wavefront's block after the current one is on its way to its registers
        auto fetch = [&](int i, Tile<D>& t) {
            const size_t at = (seq0 + (size_t)i * P.heads) * TILE + lane * 16;
            if (P.stream) {
#pragma unroll
                for (int c = 0; c < C; ++c) t.k[c] = ldg_stream16(P.k_codes + at + c * 1024);
#pragma unroll
                for (int c = 0; c < C; ++c) t.v[c] = ldg_stream16(P.v_codes + at + c * 1024);
            } else {
#pragma unroll
                for (int c = 0; c < C; ++c) t.k[c] = ld16(P.k_codes + at + c * 1024);
#pragma unroll
                for (int c = 0; c < C; ++c) t.v[c] = ld16(P.v_codes + at + c * 1024);
            }
        };
        // the scales of its next 64 blocks, one a lane
        float k_scales = 0.f, v_scales = 0.f;
        auto fetch_scales = [&](int i) {
            const int mine = i + lane * WK;
            if (mine < end) {
                const size_t at = seq0 + (size_t)mine * P.heads;
                k_scales = P.k_scale[at];
                v_scales = P.v_scale[at];
            }
        };
        Tile<D> next;
        // (blocks in turn; where there are own rows, behind the wavefronts that have those)
        int i = begin + (own ? (wk + WK - (P.nodes + 31) / 32 % WK) % WK : wk);
        const bool any = active && i < end;
        if (any) {
            fetch_scales(i);
            fetch(i, next);
        }
        if (own) fetch_own();
        load_rows();
        if (own) own_rows();
        if (any) {
            int turn = 0;
            for (; i < end; i += WK) {
                Tile<D> t = next;
                const float ks = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(k_scales), turn));
                const float vs = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v_scales), turn)) * TA_HELD;
                if (i + WK < end) {
                    fetch(i + WK, next);
                    turn = (turn + 1) & 63;
                    if (turn == 0) fetch_scales(i + WK);
                }
                f32x16 x[1];
                key_products<D, NP>(q, t.k, x[0]);
                if (tail && i == blocks - 1) hide<D>(x[0], t.v, tail);
                const float cs[1] = {score_factor(P.c, ks)};
                raise_maximum<D, 1>(R, x, cs);
                exponentials<D, false>(R, x[0], cs[0]);
                value_products<D, NP>(R, x[0], t.v, vs);
            }
        }
    }

    R.l += other_half(R.l);
    // wavefronts that share rows: each leaves its sums in LDS and takes some of the rows, a lane eight dims of one
    if constexpr (WK > 1) {
        auto& mine = s_meet[wave];
#pragma unroll
        for (int j = 0; j < C; ++j)
#pragma unroll
            for (int a = 0; a < 4; ++a)
                *reinterpret_cast<f32x4*>(&mine.o[lc][32 * j + 8 * a + 4 * half]) = f32x4{R.o[j][4 * a], R.o[j][4 * a + 1], R.o[j][4 * a + 2], R.o[j][4 * a + 3]};
        if (half == 0) { mine.m[lc] = R.m; mine.l[lc] = R.l; }
        __syncthreads();
        if (!active) return;
        constexpr int ROWS = TA_TILE / WK, PIECES = D / 8;
#pragma unroll
        for (int i = lane; i < ROWS * PIECES; i += 64) {
            const int r = wk * ROWS + i / PIECES, d0 = i % PIECES * 8, at_row = tile * TA_TILE + r;
            if (at_row >= P.rows) continue;
            float ms[WK], m = -__builtin_inff(), l = 0.f;
#pragma unroll
            for (int w = 0; w < WK; ++w) {
                ms[w] = s_meet[w * WR + wr].m[r];
                m = fmaxf(m, ms[w]);
            }
            const float base = m == -__builtin_inff() ? 0.f : m;
            f32x4 lo = {0, 0, 0, 0}, hi = {0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < WK; ++w) {
                const auto& from = s_meet[w * WR + wr];
                const float weight = __builtin_amdgcn_exp2f(ms[w] - base);
                l = __builtin_fmaf(from.l[r], weight, l);
                lo += *reinterpret_cast<const f32x4*>(&from.o[r][d0]) * weight;
                hi += *reinterpret_cast<const f32x4*>(&from.o[r][d0 + 4]) * weight;
            }
            if (splits == 1) {
                const size_t at = ((size_t)b * P.nodes + at_row / P.grp) * P.n_heads + h * P.grp + at_row % P.grp;
                const float inv = l == 0.f ? 0.f : 1.f / TA_HELD / l;
                lo *= inv;
                hi *= inv;
                char* to = P.out + (at * D + d0) * ESZ;
                if constexpr (Traits<WT>::BF) *reinterpret_cast<u32x4_q*>(to) = u32x4{pack_bf16x2(lo[0], lo[1]), pack_bf16x2(lo[2], lo[3]), pack_bf16x2(hi[0], hi[1]), pack_bf16x2(hi[2], hi[3])};
                else { *reinterpret_cast<f32x4_q*>(to) = lo; *reinterpret_cast<f32x4_q*>(to + 16) = hi; }
                if (P.lse && d0 == 0) P.lse[at] = log_sum(m, l);
            } else {
                float* to = P.part + (((size_t)blockIdx.x * P.heads + h) * P.rows + at_row) * (D + 4);
                *reinterpret_cast<f32x4*>(to + d0) = lo;
                *reinterpret_cast<f32x4*>(to + d0 + 4) = hi;
                if (d0 == 0) { to[D] = m; to[D + 1] = l; }
            }
        }
        return;
    }
    if (!valid) return;
    if (splits == 1) {
        const size_t at = ((size_t)b * P.nodes + node) * P.n_heads + head;
        const float inv = R.l == 0.f ? 0.f : 1.f / TA_HELD / R.l;
#pragma unroll
        for (int j = 0; j < C; ++j)
#pragma unroll
            for (int a = 0; a < 4; ++a)
                store4_out<WT>(P.out + (at * D + 32 * j + 8 * a + 4 * half) * ESZ, f32x4{R.o[j][4 * a], R.o[j][4 * a + 1], R.o[j][4 * a + 2], R.o[j][4 * a + 3]} * inv);
        if (P.lse && half == 0) P.lse[at] = log_sum(R.m, R.l);
    } else {
        float* to = P.part + (((size_t)blockIdx.x * P.heads + h) * P.rows + row) * (D + 4);
#pragma unroll
        for (int j = 0; j < C; ++j)
#pragma unroll
            for (int a = 0; a < 4; ++a)
                *reinterpret_cast<f32x4*>(to + 32 * j + 8 * a + 4 * half) = f32x4{R.o[j][4 * a], R.o[j][4 * a + 1], R.o[j][4 * a + 2], R.o[j][4 * a + 3]};
        if (half == 0) { to[D] = R.m; to[D + 1] = R.l; }
    }
}

// The splits of one row of one head: a lane has four dims, a wavefront 256 / D rows.  Bound by reading the parts (61 nodes, 32 heads, 32 splits of 8 sequences,
// 33 MB: 8.6 us, 4.7 TB/s with the results; a wavefront per row 10.2; few rows: 3 to 4 us, two reads one after the other).  Eight splits ahead: four are 0.4 us better there
// and 0.9 worse for 64 splits of 4 rows
template <typename WT, int D>
__global__ __launch_bounds__(256) void tree_attn_join_kernel(const TaParams P) {
    constexpr int LANES = D / 4, AHEAD = 8;
    const int lane = threadIdx.x % LANES, row = (blockIdx.x * 256 + threadIdx.x) / LANES, h = blockIdx.y, b = blockIdx.z;
    const int s0 = P.split0[b], splits = P.split0[b + 1] - s0;
    if (splits == 1 || row >= P.rows) return;
    const size_t step = (size_t)P.heads * P.rows * (D + 4);
    const float* from = P.part + (((size_t)s0 * P.heads + h) * P.rows + row) * (D + 4);
    float m = -__builtin_inff(), l = 0.f;
    f32x4 o = {0, 0, 0, 0};
    for (int s = 0; s < splits; s += AHEAD) {               // (as many splits' sums at a time: all asked for before the first is used)
        float ms[AHEAD], ls[AHEAD];
        f32x4 x[AHEAD];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const float* at = from + (size_t)min(s + u, splits - 1) * step;
            ms[u] = at[D];
            ls[u] = at[D + 1];
            x[u] = *reinterpret_cast<const f32x4*>(at + lane * 4);
        }
        float top = m;
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) top = fmaxf(top, ms[u]);
        const float base = top == -__builtin_inff() ? 0.f : top, w0 = __builtin_amdgcn_exp2f(m - base);
        m = top;
        l *= w0;
        o *= w0;
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const float w = s + u < splits ? __builtin_amdgcn_exp2f(ms[u] - base) : 0.f;
            l = __builtin_fmaf(ls[u], w, l);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(x[u][e], w, o[e]);
        }
    }
    const size_t at = ((size_t)b * P.nodes + row / P.grp) * P.n_heads + h * P.grp + row % P.grp;
    store4_out<WT>(P.out + (at * D + lane * 4) * Traits<WT>::ESZ, o * (l == 0.f ? 0.f : 1.f / TA_HELD / l));
    if (P.lse && lane == 0) P.lse[at] = log_sum(m, l);
}

// ------------------------------------------------------------------------------------------ host
struct TaPlan { int wr, waves, groups; size_t bytes; };

int plan(const ps_tree_shape* tree, const ps_tree_attn_args* a, TaParams& P, TaPlan& L) {
    if (!a || !tree || !tree->parent || !a->kv_len) return PS_ERR_NULL;
    const int st = pc_check(a->cache, a->batch);
    if (st != PS_OK) return st;
    const int N = tree->n_nodes, heads = a->cache->n_kv_heads, d = a->cache->head_dim;
    if (N < 1 || N > PS_TREE_MAX_NODES || tree->parent[0] != -1) return PS_ERR_SHAPE;
    P.sees[0] = 1;
    for (int s = 1; s < N; ++s) {
        const int pa = tree->parent[s];
        if (pa < 0 || pa >= s) return PS_ERR_SHAPE;
        P.sees[s] = P.sees[pa] | 1ull << s;
    }
    if (a->n_heads < 1 || a->n_heads % heads != 0) return PS_ERR_SHAPE;
    if (a->dtype != PS_F32 && a->dtype != PS_BF16) return PS_ERR_SHAPE;
    if (!(a->scale >= 0.f) || !(a->scale < __builtin_inff())) return PS_ERR_SHAPE;
    // (with a block's scale, 2^-100 and more, the scores' constant stays a normal number: a hidden key's -Inf times 0 would be NaN)
    if (a->n_heads > 1024 || (a->scale > 0.f && (a->scale < 0x1p-20f || a->scale > 0x1p20f))) return PS_ERR_UNSUPPORTED;
    P.batch = a->batch; P.n_heads = a->n_heads; P.heads = heads; P.grp = a->n_heads / heads; P.nodes = N; P.rows = N * P.grp;
    P.tiles = (P.rows + TA_TILE - 1) / TA_TILE;
    P.c = (float)((a->scale > 0.f ? (double)a->scale : 1.0 / __builtin_sqrt((double)d)) * 1.4426950408889634074);
    long long total = 0, blocks_of_longest = 0;
    for (int b = 0; b < a->batch; ++b) {
        P.first[b] = (unsigned)(a->cache->kv_offsets[b] / PC_BLOCK);
        P.len[b] = a->kv_len[b];
        if (P.len[b] < 0) return PS_ERR_SHAPE;
        if (P.len[b] > a->cache->kv_offsets[b + 1] - a->cache->kv_offsets[b]) return PS_ERR_KV_CAPACITY;
        if (P.len[b] > 1 << 30) return PS_ERR_UNSUPPORTED;
        const int blocks = (P.len[b] + PC_BLOCK - 1) / PC_BLOCK;
        total += blocks;
        blocks_of_longest = std::max<long long>(blocks_of_longest, blocks);
    }
    // codes that are read once and are more than the memory-side cache (256 MB) holds pass the caches by (one row tile, 32 x 2048 positions of 32 heads, 537 MB:
    // 114 -> 97 us; of 8 heads, 134 MB: 26.7 -> 28.1)
    P.stream = P.tiles == 1 && total * heads * PC_BLOCK * d * 2 > 192LL << 20;

    const bool bf = a->dtype == PS_BF16;
    // The cut is for the lengths that the host gives: a sequence whose length on the device is shorter has its blocks in the first splits only (one sequence, 2048 positions,
    // 32 heads, us, exact / a bound of 4096 / of 32768: one row 12.5 / 10.5 / 19.8, 61 nodes 16.7 / 17.7 / 29.4; eight sequences of 8 heads, 61 nodes 28 / 30 / 28).
    // How rows and blocks are cut: two or four tiles of rows per workgroup, about 256 workgroups or 512, whichever is estimated to take least time.  (bf16, us,
    // four tiles and 512 always / as estimated: 61 nodes, 32 heads that share 8, 2048 positions: 27.3 / 17.8, 8 x 2048: 44.1 / 29.5, 16 x 2048: 68.8 / 54.7 (two tiles:
    // 61), 32 x 2048: 93.6 / 89.3 (two tiles: 133), 64 x 1000: 105.5 / 107.9 (168); float32, four / two: 2048 33.3 / 26.7, 64 x 1000 298 / 312)
    auto cut = [&](int wr, int waves, long long at_once) {  // the least `per` that gives no more workgroups than that, where a split has two blocks per wavefront
        const long long units = (long long)heads * ((P.tiles + wr - 1) / wr);
        auto count = [&](long long per) {
            long long n = 0;
            for (int b = 0; b < a->batch; ++b) n += std::max<long long>(1, ((P.len[b] + PC_BLOCK - 1) / PC_BLOCK + per - 1) / per);
            return n * units;
        };
        // (a split's codes stay below 2 GiB)
        long long lo = 2 * (waves / wr), hi = std::max(lo, std::min(blocks_of_longest, (1LL << 31) / ((long long)heads * PC_BLOCK * d)));
        const long long most = std::max<long long>(at_once, count(hi));
        while (lo < hi) {
            const long long mid = (lo + hi) / 2;
            if (count(mid) <= most) hi = mid; else lo = mid + 1;
        }
        const long long groups = count(lo), splits = groups / units, longest = std::min<long long>(lo, blocks_of_longest);
        // us: 10 for what comes before and after a workgroup's blocks, 0.17 per block and tile of rows on a compute unit (float32: 0.5), rounds of 256
        // workgroups; two staged ones are on a compute unit, which shares its matrix cores among them; the join, at 4.5 TB/s
        const double block = (bf ? 0.17 : 0.5) * wr;
        const long long rounds = (groups + 255) / 256;
        double t = (bf && wr == 4 ? (groups + 511) / 512 : rounds) * 10 + rounds * longest * block;
        if (splits > a->batch) t += 4 + (double)splits * heads * P.rows * (d + 4) * 8 / 4.5e6;
        return std::pair<double, long long>(t, lo);
    };
    double best = 0;
    for (int wr = std::min(P.tiles, 2); wr <= (P.tiles >= 3 ? 4 : std::min(P.tiles, 2)); wr *= 2)
        for (int at_once = 256; at_once <= (wr == 1 ? 256 : 512); at_once *= 2) {
            const int waves = bf && wr < 4 ? 8 : 4;
            const auto c = cut(wr, waves, at_once);
            if (best > 0 && !(c.first < best)) continue;
            best = c.first;
            L.wr = wr; L.waves = waves;
            P.per = (int)c.second;
        }
    L.groups = (P.tiles + L.wr - 1) / L.wr;
    P.split0[0] = 0;
    bool one = true;
    for (int b = 0; b < a->batch; ++b) {
        const int n = std::max(1, ((P.len[b] + PC_BLOCK - 1) / PC_BLOCK + P.per - 1) / P.per);
        P.split0[b + 1] = P.split0[b] + n;
        one &= n == 1;
    }
    L.bytes = one ? 0 : a256((size_t)P.split0[a->batch] * heads * P.rows * (d + 4) * sizeof(float));
    return PS_OK;
}

template <typename WT, int D> void go(const TaParams& P, const TaPlan& L, hipStream_t s) {
    const dim3 grid(P.split0[P.batch], P.heads, L.groups), block(64 * L.waves);
    if (L.wr == 1) hipLaunchKernelGGL((tree_attn_kernel<WT, D, 1>), grid, block, 0, s, P);
    else if (L.wr == 2) hipLaunchKernelGGL((tree_attn_kernel<WT, D, 2>), grid, block, 0, s, P);
    else hipLaunchKernelGGL((tree_attn_kernel<WT, D, 4>), grid, block, 0, s, P);
    if (L.bytes) hipLaunchKernelGGL((tree_attn_join_kernel<WT, D>), dim3((P.rows + 1024 / D - 1) / (1024 / D), P.heads, P.batch), dim3(256), 0, s, P);
}

}   // namespace

extern "C" size_t ps_tree_attention_workspace_bytes(const ps_tree_shape* tree, const ps_tree_attn_args* a) {
    TaParams P = {};
    TaPlan L = {};
    return plan(tree, a, P, L) == PS_OK ? L.bytes : 0;
}

extern "C" int ps_tree_attention(const ps_tree_shape* tree, const ps_tree_attn_args* a, void* stream) {
    if (!a || !a->q || !a->out || !a->k_rows != !a->v_rows) return PS_ERR_NULL;
    TaParams P = {};
    TaPlan L = {};
    const int st = plan(tree, a, P, L);
    if (st != PS_OK) return st;
    if (!aligned4(a->q) || !aligned4(a->k_rows) || !aligned4(a->v_rows) || !aligned4(a->out) || !aligned4(a->lse) || !aligned4(a->kv_len_dev))
        return PS_ERR_UNSUPPORTED;
    int64_t bytes = 0;
    const int d = a->cache->head_dim;
    int sst = pc_stride(a->q_stride, (int64_t)a->n_heads * d, a->dtype, &bytes);
    P.q_row = bytes;
    if (sst == PS_OK && a->k_rows) {
        sst = pc_stride(a->kv_stride, (int64_t)P.heads * d, a->dtype, &bytes);
        P.kv_row = bytes;
    }
    if (sst != PS_OK) return sst;
    if (L.bytes && (!a->workspace || a->workspace_bytes < L.bytes || ((uintptr_t)a->workspace & 255))) return a->workspace ? PS_ERR_WORKSPACE : PS_ERR_NULL;
    P.q = (const char*)a->q; P.k = (const char*)a->k_rows; P.v = (const char*)a->v_rows;
    P.out = (char*)a->out; P.lse = a->lse; P.part = (float*)a->workspace;
    P.k_codes = a->cache->k_codes; P.v_codes = a->cache->v_codes; P.k_scale = a->cache->k_scale; P.v_scale = a->cache->v_scale;
    P.len_dev = a->kv_len_dev;
    const hipStream_t s = (hipStream_t)stream;
    if (a->dtype == PS_BF16) { if (d == 128) go<bf16_t, 128>(P, L, s); else go<bf16_t, 64>(P, L, s); }
    else if (d == 128) go<float, 128>(P, L, s);
    else go<float, 64>(P, L, s);
    return hipGetLastError() == hipSuccess ? PS_OK : PS_ERR_DEVICE;
}

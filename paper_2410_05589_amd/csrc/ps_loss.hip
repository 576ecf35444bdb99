// Cross entropy of rows against the LM head and its gradient with respect to the rows (see include/ps_train.h; Section 4.3, Eq. 3),
// without the logits: attention's scheme with h as queries and the LM head as keys and values.
//
//   l_v = h . W_v;  x_v = exp(l_v - l_t) / 2^64 for v != t, 0 for v = t;  S = sum_v x_v
//   loss = w log(1 + 2^64 S);   d_h = w (sum_v x_v W_v / (S + 2^-64) - W_t 2^64 S / (1 + 2^64 S))
//
// The exponentials are taken against the target's own logit, which is known beforehand (a dot product per row): no maximum has to be
// found first, one pass over the vocabulary does, and the target's column, left out, comes in at the end in float32: nothing
// cancels for a row that is sure of its target (1 - p_t is the sum of the others, not a difference).  A row with a logit more
// than 144 ln 2 = 99 above its target's would leave the float range; such rows (their loss is over 99) are marked and worked
// out again one by one, against their maximum.
//
// The vocabulary is gone through in pieces; two products for each, the floor being their 4 V H operations a row:
//   vl_score_kernel   W h^T, one tile per workgroup: exponentials to the workspace, sums of rows (of the unrounded) beside them.  In bf16 they are
//                     rounded once, half a step 2^-8 each: they are operands of the next product's MFMAs, and a gradient adds up many, so that its
//                     error stays that of its own rounding (relative 2-norm 0.0017 with them and with float32 exponentials)
//   vl_grad_kernel    exponentials . W, added to what the pieces before left, in float32
// The rows' sums make their losses and the gradients' factors: in vl_join_kernel, which adds up the parts of the products, or, where the last
// product's tiles become gradients at once, in vl_rows_kernel before it.
//
// Bound by the matrix cores: 10240 rows, H 4096, V 32000 take 4240 .. 4440 us, 1.21 .. 1.27 PFLOP/s of a large library product's 1.32 (4070 us); 9216 rows,
// V 128256 15650 .. 15990 (14700); 1218 rows, H 5120, V 32000 800 (605); the cores are busy 74 % of the scores' time and 84 % of the gradients'.  Small calls
// are a chain of four launches: 200 rows, H 256, V 1024 in float32 25 us.
#include <math.h>

#include "ps_train_device.h"
#include "ps_draft_debug.h"

namespace {

constexpr int VL_THREADS = 256, VL_AHEAD = 4;             // stages that are requested ahead of the one in LDS
enum { VL_NEAR = 0, VL_FAR_APART = 1, VL_DONE = 2, VL_ZERO = 3 };
constexpr float VL_SHIFT = 64.f, VL_FAR = 0x1p80f, VL_LOG2E = 1.4426950408889634f, VL_LN2 = 0.6931471805599453f;

struct VlParams {
    int rows, H, V, row0, rows_c;     // this chunk: rows row0 .. row0 + rows_c - 1
    int v0, nv, ldx;                  // this piece: tokens v0 .. v0 + nv - 1; elements between rows of x
    int nsum;                         // partial sums of a row: one for every 64 tokens
    int splits, split_n, first;       // parts of a piece's tokens, tokens of a part, first piece
    const char *h, *w;
    const int* targets;
    const float* weights;
    float* loss;
    char* d_hidden;
    float *tl, *sums, *acc, *alone;   // target logits; sums [rows_c][nsum]; products [splits][rows_c][H]; those of rows by themselves [rows_c][H]
    int* state;                       // rows: VL_NEAR, VL_FAR_APART (set by the scores), from vl_rows_kernel on also VL_DONE, VL_ZERO
    float2* factor;                   // of a row's products, of its target's row of the LM head
    char* x;                          // exponentials [rows_c][ldx], storage type
};

__device__ __forceinline__ bool vl_counts(const VlParams& P, int row) {
    return (unsigned)P.targets[row] < (unsigned)P.V && (!P.weights || P.weights[row] != 0.f);
}

// a row's dot product with row v of the LM head, all lanes of the wavefront get it
template <typename WT> __device__ __forceinline__ float vl_dot(const VlParams& P, int row, int v, int lane) {
    constexpr int GE = Traits<WT>::GE;
    const char *a = P.h + (size_t)row * P.H * Traits<WT>::ESZ, *b = P.w + (size_t)v * P.H * Traits<WT>::ESZ;
    float s[2] = {0.f, 0.f};
    for (int i = lane; i < P.H / GE; i += 64) {
        float x[GE], y[GE];
        load_group<WT>(a + (size_t)i * 16, x);
        load_group<WT>(b + (size_t)i * 16, y);
#pragma unroll
        for (int e = 0; e < GE; ++e) s[e & 1] += x[e] * y[e];
    }
    return wave_sum(s[0] + s[1]);
}

template <typename WT> __global__ void __launch_bounds__(VL_THREADS) vl_target_kernel(const VlParams P) {
    const int row = blockIdx.x * (VL_THREADS / 64) + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (row >= P.rows) return;
    const bool counts = vl_counts(P, row);
    const float t = counts ? vl_dot<WT>(P, row, P.targets[row], lane) : 0.f;
    if (lane == 0) {
        P.tl[row] = t;
        P.state[row] = VL_NEAR;
    }
}

// 16 bytes of a row of each operand (chunk 2 t + half of a 64-byte step): one MFMA of bf16, four of float32, in which both operands
// take the contraction in the same order (float32: element 4 half + e of the step's 8 in the e-th)
template <typename WT> __device__ __forceinline__ void vl_mma(uint4 a, uint4 b, f32x16& c) {
    if constexpr (Traits<WT>::BF) {
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    } else {
        const f32x4 x = __builtin_bit_cast(f32x4, a), y = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], y[e], c, 0, 0, 0);
    }
}
// place of 16-byte chunk j of a 64-byte row (16 rows' chunks of one number fill the banks)
__device__ __forceinline__ int vl_at(int row, int j) { return row * 64 + ((j ^ ((row >> 2) & 3)) << 4); }

// steps first .. end - 1: load(step, x) requests a stage into registers, store(buffer, x) puts it into LDS, multiply(buffer)
template <typename STAGE, typename LOAD, typename STORE, typename MULTIPLY>
__device__ __forceinline__ void vl_pipeline(int first, int end, char* smem, int buf, LOAD load, STORE store, MULTIPLY multiply) {
    if (first >= end) return;
    STAGE x[VL_AHEAD];
#pragma unroll
    for (int u = 0; u < VL_AHEAD; ++u)
        if (first + u < end) load(first + u, x[u]);
    store(smem, x[0]);
    if (first + VL_AHEAD < end) load(first + VL_AHEAD, x[0]);
    __syncthreads();
    for (int k0 = first; k0 < end; k0 += VL_AHEAD) {
#pragma unroll
        for (int u = 0; u < VL_AHEAD; ++u) {
            const int k = k0 + u;
            if (k >= end) break;
            STAGE& y = x[(u + 1) % VL_AHEAD];
            if (k + 1 < end) store(smem + ((u + 1) & 1) * buf, y);
            if (k + 1 + VL_AHEAD < end) load(k + 1 + VL_AHEAD, y);
            multiply(smem + (u & 1) * buf);
            __syncthreads();
        }
    }
}
static_assert(VL_AHEAD % 2 == 0, "a stage's buffer follows from its number");

// Tiles of TILE x TILE (64, where 128 would leave compute units without one), four wavefronts of half the side each
template <typename WT, int TILE>
__global__ void __launch_bounds__(VL_THREADS, 2) vl_score_kernel(const VlParams P) {
    constexpr int ESZ = Traits<WT>::ESZ, HALF = TILE / 2, N = TILE / 64, SIDE = TILE * 64, BUF = 2 * SIDE;
    __shared__ __attribute__((aligned(16))) char smem[2 * BUF];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, half = lane >> 5;
    const int vt = blockIdx.x * TILE, rt = blockIdx.y * TILE;   // in the piece, in the chunk
    const int wv = (wave & 1) * HALF, wr = (wave >> 1) * HALF;
    const size_t rb = (size_t)P.H * ESZ;
    const char *wsrc[N], *hsrc[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        wsrc[i] = P.w + (size_t)min(P.v0 + vt + tid / 4 + 64 * i, P.V - 1) * rb + (tid & 3) * 16;
        hsrc[i] = P.h + (size_t)(P.row0 + min(rt + tid / 4 + 64 * i, P.rows_c - 1)) * rb + (tid & 3) * 16;
    }
    f32x16 acc[N][N];
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    struct Stage { uint4 w[N], h[N]; };
    vl_pipeline<Stage>(0, P.H * ESZ / 64, smem, BUF,
        [&](int k, Stage& x) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < N; ++i) { x.w[i] = ld16(wsrc[i] + (size_t)k * 64); x.h[i] = ld16(hsrc[i] + (size_t)k * 64); }
        },
        [&](char* b, const Stage& x) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                *reinterpret_cast<uint4*>(b + vl_at(tid / 4 + 64 * i, tid & 3)) = x.w[i];
                *reinterpret_cast<uint4*>(b + SIDE + vl_at(tid / 4 + 64 * i, tid & 3)) = x.h[i];
            }
        },
        [&](const char* b) __attribute__((always_inline)) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                uint4 a[N], q[N];
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    a[i] = ld16(b + vl_at(wv + 32 * i + c, 2 * t + half));
                    q[i] = ld16(b + SIDE + vl_at(wr + 32 * i + c, 2 * t + half));
                }
#pragma unroll
                for (int i = 0; i < N; ++i)
#pragma unroll
                    for (int j = 0; j < N; ++j) vl_mma<WT>(a[i], q[j], acc[i][j]);
            }
        });
    // ---- lane (c, half) holds of row 32 j + c the tokens 32 i + 8 (e / 4) + 4 half + e % 4
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int r = rt + wr + 32 * j + c, row = P.row0 + min(r, P.rows_c - 1);
        const int t = P.targets[row] - P.v0 - vt - wv - 4 * half, end = P.V - P.v0 - vt - wv - 4 * half;
        const float ref = -P.tl[row] * VL_LOG2E - VL_SHIFT;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                f32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int at = 32 * i + 8 * q + e;
                    const float y = fmaf(acc[i][j][4 * q + e], VL_LOG2E, ref);
                    const bool in = at != t && at < end;
                    v[e] = in ? __builtin_amdgcn_exp2f(y) : 0.f;
                    sum += v[e];
                }
                if (P.x && r < P.rows_c) store4<WT>(P.x + ((size_t)r * P.ldx + vt + wv + 32 * i + 8 * q + 4 * half) * ESZ, v);
            }
        const auto sw2 = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum), __float_as_uint(sum), false, false);
        sum = __uint_as_float(sw2[0]) + __uint_as_float(sw2[1]);
        if (r < P.rows_c) {
            if (sum > VL_FAR) P.state[row] = VL_FAR_APART;   // (infinite among them)
            if (half == 0) P.sums[(size_t)r * P.nsum + (P.v0 + vt + wv) / HALF] = sum;
        }
    }
}

template <typename WT, int TILE>
__global__ void __launch_bounds__(VL_THREADS, 2) vl_grad_kernel(const VlParams P) {
    constexpr int ESZ = Traits<WT>::ESZ, KV = 64 / ESZ, HALF = TILE / 2, N = TILE / 64;   // KV: tokens of a step
    constexpr int ABUF = TILE * 64, WSTR = TILE * ESZ + (Traits<WT>::BF ? 64 : 32), WBUF = KV * WSTR, BUF = ABUF + WBUF;
    __shared__ __attribute__((aligned(16))) char smem[2 * BUF];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, half = lane >> 5;
    const int ct = blockIdx.x * TILE, rt = blockIdx.y * TILE, split = blockIdx.z;
    const int wc = (wave & 1) * HALF, wr = (wave >> 1) * HALF;
    const int k0 = split * (P.split_n / KV), k1 = min((split + 1) * P.split_n, (P.nv + KV - 1) / KV * KV) / KV;
    constexpr int TPV = TILE * ESZ / 16;                     // 16-byte pieces of a staged row of W
    const char* xsrc[N];
#pragma unroll
    for (int i = 0; i < N; ++i) xsrc[i] = P.x + (size_t)min(rt + tid / 4 + 64 * i, P.rows_c - 1) * P.ldx * ESZ + (tid & 3) * 16;
    const int wk = tid / TPV, wp = tid % TPV;                // this thread's tokens wk + (256 / TPV) i, its piece (beyond H: the last)
    const size_t wcol = (size_t)min(ct * ESZ + wp * 16, P.H * ESZ - 16);
    f32x16 acc[N][N];
    float* out = P.acc + (size_t)split * P.rows_c * P.H;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int r = rt + wr + 32 * i + 8 * (e / 4) + 4 * half + e % 4, col = ct + wc + 32 * j + c;
                acc[i][j][e] = P.first ? 0.f : out[(size_t)min(r, P.rows_c - 1) * P.H + min(col, P.H - 1)];
            }
    const int vkey = (lane & 15) >> 2, vhi = (lane >> 4) & 1;
    auto column = [&](const char* b, int t, int j) __attribute__((always_inline)) {   // W^T: columns wc + 32 j + c, 16 bytes' worth of tokens
        const char* p = b + ABUF;
        if constexpr (Traits<WT>::BF) {
            const char* a = p + (16 * t + 8 * half + vkey) * WSTR + (wc + 32 * j) * 2 + vhi * 32 + (lane & 3) * 8;
            const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)a);
            const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(a + 4 * WSTR));
            return __builtin_bit_cast(uint4, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            f32x4 r;
#pragma unroll
            for (int e = 0; e < 4; ++e) r[e] = *reinterpret_cast<const float*>(p + (8 * t + 4 * half + e) * WSTR + (wc + 32 * j + c) * 4);
            return __builtin_bit_cast(uint4, r);
        }
    };
    struct Stage { uint4 x[N], w[N]; };
    vl_pipeline<Stage>(k0, k1, smem, BUF,
        [&](int k, Stage& s) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                s.x[i] = ld16(xsrc[i] + (size_t)k * 64);
                s.w[i] = ld16(P.w + (size_t)min(P.v0 + k * KV + wk + VL_THREADS / TPV * i, P.V - 1) * P.H * ESZ + wcol);
            }
        },
        [&](char* b, const Stage& s) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                *reinterpret_cast<uint4*>(b + vl_at(tid / 4 + 64 * i, tid & 3)) = s.x[i];
                *reinterpret_cast<uint4*>(b + ABUF + (wk + VL_THREADS / TPV * i) * WSTR + wp * 16) = s.w[i];
            }
        },
        [&](const char* b) __attribute__((always_inline)) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                uint4 a[N], q[N];
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    a[i] = ld16(b + vl_at(wr + 32 * i + c, 2 * t + half));
                    q[i] = column(b, t, i);
                }
#pragma unroll
                for (int i = 0; i < N; ++i)
#pragma unroll
                    for (int j = 0; j < N; ++j) vl_mma<WT>(a[i], q[j], acc[i][j]);
            }
        });
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < N; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int r = rt + wr + 32 * i + 8 * (e / 4) + 4 * half + e % 4, col = ct + wc + 32 * j + c;
                if (r < P.rows_c && col < P.H) out[(size_t)r * P.H + col] = acc[i][j][e];
            }
}

// ------------------------------------------------------------------------------------------
// bf16, many rows: tiles of 256 x 256, eight wavefronts (two per SIMD) of 128 x 64 each, 32 elements of the contraction per stage.
// A stage (32 KiB) is brought in by the memory unit itself (no registers): 1 KiB per request, lanes in the order of the LDS,
// their source addresses permuted so that rows read together fall into different banks.  Four buffers: while a stage is multiplied from
// registers, the next is read from LDS, two more are on their way and the one that has just been read is filled anew.  The wait at
// a stage's barrier leaves the youngest two stages in flight.  The buffers are arrays of their own: the compiler then knows that a
// read from one need not wait for what is on its way into another.
// ------------------------------------------------------------------------------------------
constexpr int VW_THREADS = 512, VW_TILE = 256, VW_A = VW_TILE * 64, VW_BUF = 2 * VW_A;
typedef __attribute__((address_space(3))) void lds_void;
__device__ __forceinline__ void vw_copy(rsrc_t from, unsigned off, unsigned soff, char* to) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lds_void*)to, 16, off, soff, 0, 0);
}
// the workgroup's requests have arrived, and its reads and writes of LDS are done
__device__ __forceinline__ void vw_arrived() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __syncthreads();
}
// 256 rows of 64 bytes, as vl_at places them
struct VwRows {
    rsrc_t src;
    unsigned off[2];
    // rows first .. first + 255 of a matrix (rows beyond last: the last), wavefront w's 32 of them
    __device__ __forceinline__ VwRows(const char* m, size_t first, size_t last, unsigned stride, int wave, int lane) {
        src = make_rsrc(m + first * stride);
        const unsigned most = (unsigned)min((size_t)VW_TILE, last - first + 1) - 1;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const unsigned row = 32 * wave + 16 * i + lane / 4;
            off[i] = min(row, most) * stride + ((lane & 3) ^ ((row >> 2) & 3)) * 16;
        }
    }
    __device__ __forceinline__ void stage(int k, char* lds, int wave) const {
#pragma unroll
        for (int i = 0; i < 2; ++i) vw_copy(src, off[i], k * 64, lds + (32 * wave + 16 * i) * 64);
    }
};
struct VwOperands { bf16x8 a[4][2], b[2][2]; };
// steps stages from `first` on: stage(k, buffer) requests (four requests per wavefront), read(buffer, operands), then the products
template <int READS, typename STAGE, typename READ>
__device__ __forceinline__ void vw_pipeline(int first, int steps, char* b0, char* b1, char* b2, char* b3, STAGE stage, READ read, f32x16 (&acc)[4][2]) {
    const int last = first + steps - 1;
    stage(first, b0);
    stage(min(first + 1, last), b1);
    stage(min(first + 2, last), b2);
    stage(min(first + 3, last), b3);
    VwOperands x[2];
    asm volatile("s_waitcnt vmcnt(12)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    read(b0, x[0]);
    auto step = [&](int k, char* mine, char* next, const VwOperands& now, VwOperands& then) __attribute__((always_inline)) {
        // stage k is in registers (now); every wavefront has read it once all have come here, so that its buffer may be filled again
        asm volatile("s_waitcnt vmcnt(8) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_sched_barrier(0);
        stage(min(k + 4, last), mine);
        read(next, then);
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(now.a[i][t], now.b[j][t], acc[i][j], 0, 0, 0);
        // (requests and reads between the MFMAs, none of the latter beyond the barriers)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, (READS + 7) / 8, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
        __builtin_amdgcn_sched_barrier(0);
    };
    int k = first;
    for (; k + 3 <= last; k += 4) {
        step(k, b0, b1, x[0], x[1]);
        step(k + 1, b1, b2, x[1], x[0]);
        step(k + 2, b2, b3, x[0], x[1]);
        step(k + 3, b3, b0, x[1], x[0]);
    }
    if (k <= last) step(k, b0, b1, x[0], x[1]);
    if (k + 1 <= last) step(k + 1, b1, b2, x[1], x[0]);
    if (k + 2 <= last) step(k + 2, b2, b3, x[0], x[1]);
    vw_arrived();                                           // (nothing is on its way into the buffers any more)
}

// A tile's workgroup number -> the tile: workgroups go to the XCDs in turn; an XCD gets a stretch of the order, in which
// 32 neighbours (its compute units) share four rows' and eight columns' operands
__device__ __forceinline__ void vw_tile(unsigned id, unsigned nx, unsigned ny, unsigned& x, unsigned& y) {
    const unsigned n = nx * ny, q = n / 8, r = n % 8, xcd = id % 8;
    id = xcd * q + min(xcd, r) + id / 8;
    const unsigned g = id / (4 * nx), h = min(ny - 4 * g, 4u);
    id -= g * 4 * nx;
    x = id / h;
    y = 4 * g + id % h;
}

__global__ void __launch_bounds__(VW_THREADS, 2) vl_score_wide_kernel(const VlParams P, int nx, int ny) {
    __shared__ __attribute__((aligned(16))) char b0[VW_BUF], b1[VW_BUF], b2[VW_BUF], b3[VW_BUF];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, half = lane >> 5;
    unsigned tx, ty;
    vw_tile(blockIdx.x, nx, ny, tx, ty);
    const int vt = tx * VW_TILE, rt = ty * VW_TILE, wm = wave & 1, wn = wave >> 1;
    const unsigned rb = P.H * 2;
    const VwRows A(P.w, P.v0 + vt, P.V - 1, rb, wave, lane), B(P.h, P.row0 + rt, P.row0 + P.rows_c - 1, rb, wave, lane);
    f32x16 acc[4][2];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    const int at = vl_at(c, half), a0 = 128 * wm * 64 + at, w0 = VW_A + 64 * wn * 64 + at;
    vw_pipeline<12>(0, P.H / 32, b0, b1, b2, b3,
                [&](int k, char* b) __attribute__((always_inline)) { A.stage(k, b, wave); B.stage(k, b + VW_A, wave); },
                [&](const char* b, VwOperands& x) __attribute__((always_inline)) {
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
#pragma unroll
                        for (int j = 0; j < 2; ++j) x.b[j][t] = __builtin_bit_cast(bf16x8, ld16(b + (w0 ^ (t << 5)) + j * 2048));
#pragma unroll
                        for (int i = 0; i < 4; ++i) x.a[i][t] = __builtin_bit_cast(bf16x8, ld16(b + (a0 ^ (t << 5)) + i * 2048));
                    }
                }, acc);
    // ---- lane (c, half) holds of row 64 wn + 32 j + c the tokens 128 wm + 32 i + 8 (e / 4) + 4 half + e % 4; they leave by way of the LDS,
    // rows of 512 bytes, 16-byte piece p at p ^ row % 32 (64 rows to a buffer)
    char* const mine = wn < 2 ? wn ? b1 : b0 : wn == 2 ? b2 : b3;   // (also the one of the rows that the wavefront stores)
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int rr = 64 * wn + 32 * j + c, r = rt + rr, row = P.row0 + min(r, P.rows_c - 1);
        const int base = P.v0 + vt + 128 * wm, t = P.targets[row] - base - 4 * half, end = P.V - base - 4 * half;
        const float ref = -P.tl[row] * VL_LOG2E - VL_SHIFT;
        float sum[2] = {0.f, 0.f};
        // (a target among the wavefront's tokens, or the vocabulary's end: those count nothing)
        if (__any(((unsigned)(t + 4) < 132u) | (end < 128))) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int tok = 32 * i + 8 * (e / 4) + e % 4;
                    acc[i][j][e] = tok != t && tok < end ? acc[i][j][e] : -INFINITY;
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                f32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float y = fmaf(acc[i][j][4 * q + e], VL_LOG2E, ref);
                    v[e] = __builtin_amdgcn_exp2f(y);
                    sum[e & 1] += v[e];
                }
                if (P.x) {
                    const int piece = 16 * wm + 4 * i + q;
                    *reinterpret_cast<u32x2*>(mine + (rr & 63) * 512 + ((piece ^ (rr & 31)) << 4) + 8 * half) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
                }
            }
        const float mine = sum[0] + sum[1];
        const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mine), __float_as_uint(mine), false, false);
        if (r < P.rows_c) {
            const float both = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
            if (both > VL_FAR) P.state[row] = VL_FAR_APART;
            if (half == 0) P.sums[(size_t)r * P.nsum + (P.v0 + vt) / 128 + wm] = both;
        }
    }
    if (!P.x) return;
    __syncthreads();
#pragma unroll 4
    for (int i = 0; i < 16; ++i) {
        const int rr = 32 * wave + 2 * i + (lane >> 5), r = rt + rr, p = lane & 31;
        const uint4 v = ld16(mine + (rr & 63) * 512 + ((p ^ (rr & 31)) << 4));
        if (r < P.rows_c) *reinterpret_cast<uint4*>(P.x + ((size_t)r * P.ldx + vt + 8 * p) * 2) = v;
    }
}

// (LAST: of a whole row's products the gradient is made at once)
template <bool LAST>
__global__ void __launch_bounds__(VW_THREADS, 2) vl_grad_wide_kernel(const VlParams P, int nx, int ny) {
    __shared__ __attribute__((aligned(16))) char b0[VW_BUF], b1[VW_BUF], b2[VW_BUF], b3[VW_BUF];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, half = lane >> 5;
    unsigned tx, ty;
    vw_tile(blockIdx.x, nx, ny, tx, ty);
    const int split = blockIdx.y, ct = tx * VW_TILE, rt = ty * VW_TILE, wm = wave & 1, wn = wave >> 1;
    const unsigned rb = P.H * 2;
    const VwRows A(P.x, rt, P.rows_c - 1, P.ldx * 2, wave, lane);
    const int k0 = split * (P.split_n / 32), k1 = min((split + 1) * P.split_n, (P.nv + 31) / 32 * 32) / 32;
    // W: 32 rows of 512 bytes (columns beyond H: the last), wavefront w's 4 of them; 32-byte chunk j stands at j ^ 2 f(row),
    // f = row % 4 + 4 (row / 8 % 2), so that the eight rows of a transposed read fall into different banks
    unsigned col[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const unsigned row = 4 * wave + 2 * i + (lane >> 5), f = (row & 3) | ((row >> 3 & 1) << 2), chunk = ((lane & 31) >> 1) ^ (f << 1);
        col[i] = min((unsigned)ct * 2 + chunk * 32 + (lane & 1) * 16, rb - 16);
    }
    __shared__ float4 info[LAST ? VW_TILE : 1];              // the rows' factors, state, target
    if (LAST && tid < VW_TILE) {
        const int r = min(rt + tid, P.rows_c - 1), state = P.state[P.row0 + r];
        const float2 f = P.factor[r];
        info[tid] = make_float4(f.x, f.y, (float)state, __int_as_float(state == VL_NEAR ? P.targets[P.row0 + r] : 0));
    }
    f32x16 acc[4][2];
    float* out = P.acc + (size_t)split * P.rows_c * P.H;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int r = rt + 128 * wm + 32 * i + 8 * (e / 4) + 4 * half + e % 4, x = ct + 64 * wn + 32 * j + c;
                acc[i][j][e] = P.first ? 0.f : out[(size_t)min(r, P.rows_c - 1) * P.H + min(x, P.H - 1)];
            }
    const int a0 = 128 * wm * 64 + vl_at(c, half);
    const int vkey = (lane & 15) >> 2, vhi = (lane >> 4) & 1, f = vkey | half << 2;
    const int w0 = (VW_A + (8 * half + vkey) * 512 + ((vhi ^ (f << 1)) << 5) + (lane & 3) * 8) ^ (4 * wn << 5);
    if (k0 < k1)
        vw_pipeline<16>(k0, k1 - k0, b0, b1, b2, b3,
                    [&](int k, char* b) __attribute__((always_inline)) {
                        A.stage(k, b, wave);
                        const int v = P.v0 + 32 * k;
                        const rsrc_t src = make_rsrc(P.w + (size_t)v * rb);
#pragma unroll
                        for (int i = 0; i < 2; ++i) vw_copy(src, (unsigned)min(4 * wave + 2 * i + (lane >> 5), P.V - 1 - v) * rb + col[i], 0, b + VW_A + (4 * wave + 2 * i) * 512);
                    },
                    [&](const char* b, VwOperands& x) __attribute__((always_inline)) {
#pragma unroll
                        for (int t = 0; t < 2; ++t) {
#pragma unroll
                            for (int j = 0; j < 2; ++j) {
                                const char* a = b + (w0 ^ (2 * j << 5)) + t * 16 * 512;
                                const s16x4 u = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)a), w = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(a + 4 * 512));
                                x.b[j][t] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(u, w, 0, 1, 2, 3, 4, 5, 6, 7));
                            }
#pragma unroll
                            for (int i = 0; i < 4; ++i) x.a[i][t] = __builtin_bit_cast(bf16x8, ld16(b + (a0 ^ (t << 5)) + i * 2048));
                        }
                    }, acc);
    // ---- lane (c, half) holds columns 64 wn + 32 j + c of rows 128 wm + 32 i + 8 (e / 4) + 4 half + e % 4
    if constexpr (LAST) {
        // the targets' rows come into the LDS (rows of 512 bytes, 64 to a buffer, 64-byte blocks 2 m and 2 m + 1 exchanged in every second
        // four rows: the halves' rows fall into different banks), turn into the gradient there and leave in whole lines
        auto buffer = [&](int row) __attribute__((always_inline)) { return row < 128 ? row < 64 ? b0 : b1 : row < 192 ? b2 : b3; };
        char* const mine = buffer(32 * wave);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int rr = 32 * wave + 2 * i + (lane >> 5), piece = (lane & 31) ^ ((rr & 4) ? 4 : 0);
            const char* from = P.w + (size_t)(unsigned)__float_as_int(info[rr].w) * rb + min((unsigned)ct * 2 + piece * 16, rb - 16);
            __builtin_amdgcn_global_load_lds((__attribute__((address_space(1))) void*)from, (lds_void*)(mine + ((32 * wave + 2 * i) & 63) * 512), 16, 0, 0);
        }
        vw_arrived();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            char* const at = buffer(128 * wm + 32 * i) + 32 * (i & 1) * 512 + (64 * wn + c) * 2;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int rr = 8 * (e / 4) + 4 * half + e % 4;   // of the 32
                const f32x4 f = *reinterpret_cast<const f32x4*>(info + 128 * wm + 32 * i + rr);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    uint16_t* p = reinterpret_cast<uint16_t*>(at + rr * 512 + 64 * (j ^ half));
                    const float v = acc[i][j][e] * f[0] + bf16_to_f32(*p) * f[1];
                    *p = (uint16_t)pack_bf16x2(f[2] != 0.f ? 0.f : v, 0.f);
                }
            }
        }
        __syncthreads();
#pragma unroll 4
        for (int i = 0; i < 16; ++i) {
            const int rr = 32 * wave + 2 * i + (lane >> 5), piece = (lane & 31) ^ ((rr & 4) ? 4 : 0);
            const uint4 v = ld16(mine + (rr & 63) * 512 + (lane & 31) * 16);
            if (rt + rr < P.rows_c && ct + 8 * piece < P.H && info[rr].z != (float)VL_DONE)
                *reinterpret_cast<uint4*>(P.d_hidden + ((size_t)(P.row0 + rt + rr) * P.H + ct + 8 * piece) * 2) = v;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const int r = rt + 128 * wm + 32 * i + 8 * (e / 4) + 4 * half + e % 4, x = ct + 64 * wn + 32 * j + c;
                    if (r < P.rows_c && x < P.H) out[(size_t)r * P.H + x] = acc[i][j][e];
                }
    }
}

template <typename WT> __device__ __forceinline__ void vl_store_group(char* p, const float* v) {
    u32x4 r;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        if constexpr (Traits<WT>::BF) r[u] = pack_bf16x2(v[2 * u], v[2 * u + 1]);
        else r[u] = __float_as_uint(v[u]);
    }
    *reinterpret_cast<u32x4*>(p) = r;
}

// A row whose logits lie too far above its target's: its maximum, then sums against it, 256 tokens at a time.  Returns log2 of
// sum_{v != t} exp(l_v - l_t); acc (of the row, float32) becomes sum_{v != t} p_v W_v.  One workgroup reads the
// whole LM head, three times if the gradient is wanted, once if not: 37 ms at H 5120, V 32000 without, 93 with it, for one row or a thousand.
template <typename WT>
__device__ __forceinline__ float vl_row_alone(const VlParams& P, int row, int target, float* acc, float* s, int tid) {
    constexpr int GE = Traits<WT>::GE, ESZ = Traits<WT>::ESZ;
    const int lane = tid & 63, wave = tid >> 6;
    float m = -INFINITY, total = 0.f;
    for (int v = wave; v < P.V; v += 4) {
        const float l = vl_dot<WT>(P, row, v, lane) * VL_LOG2E;
        if (v == target) continue;
        const float top = fmaxf(m, l), ref = top > -INFINITY ? top : 0.f;
        total = total * __builtin_amdgcn_exp2f(m - ref) + __builtin_amdgcn_exp2f(l - ref);
        m = top;
    }
    __syncthreads();
    if (lane == 0) {
        s[2 * wave] = m;
        s[2 * wave + 1] = total;
    }
    __syncthreads();
    const float top = fmaxf(fmaxf(s[0], s[2]), fmaxf(s[4], s[6]));
    total = 0.f;
    for (int i = 0; i < 4; ++i) total += s[2 * i + 1] * __builtin_amdgcn_exp2f(s[2 * i] - top);
    const float z = top < INFINITY ? top + __builtin_amdgcn_logf(total) - P.tl[row] * VL_LOG2E : top;   // (an infinite logit: NaN among the probabilities)
    if (!P.d_hidden) return z;
    const float lse = top + __builtin_amdgcn_logf(total + __builtin_amdgcn_exp2f(P.tl[row] * VL_LOG2E - top));
    for (int v0 = 0; v0 < P.V; v0 += 256) {
        __syncthreads();
        for (int i = wave; i < 256; i += 4) {
            const int v = v0 + i;
            const float l = v < P.V ? vl_dot<WT>(P, row, v, lane) * VL_LOG2E : 0.f;
            if (lane == 0) s[i] = v < P.V && v != target ? __builtin_amdgcn_exp2f(l - lse) : 0.f;
        }
        __syncthreads();
        for (int c = tid; c < P.H / GE; c += VL_THREADS) {
            float sum[GE];
#pragma unroll
            for (int e = 0; e < GE; ++e) sum[e] = v0 == 0 ? 0.f : acc[c * GE + e];
            for (int i = 0; i < min(256, P.V - v0); ++i) {
                float x[GE];
                load_group<WT>(P.w + ((size_t)(v0 + i) * P.H + c * GE) * ESZ, x);
#pragma unroll
                for (int e = 0; e < GE; ++e) sum[e] += s[i] * x[e];
            }
#pragma unroll
            for (int e = 0; e < GE; ++e) acc[c * GE + e] = sum[e];
        }
    }
    __syncthreads();
    return z;
}

// What a row's sums make (a wavefront): its loss, written, and the factors of its products and of its target's row of the LM head, if it
// counts and is not far apart.  sum: of its exponentials.
struct VlRow { int state; float2 f; };
template <typename WT> __device__ __forceinline__ float2 vl_finish(const VlParams& P, int row, float z, float scale, bool write) {
    // z: log2 of sum_{v != t} exp(l_v - l_t); the loss is log(1 + 2^z), the others' probability 2^z / (1 + 2^z)
    // (a target's logit of Inf or NaN leaves no sum to compare it with: NaN; of -Inf, an infinite loss)
    if (!(fabsf(P.tl[row]) < INFINITY) && z != INFINITY) z = NAN;
    const float weight = P.weights ? P.weights[row] : 1.f, e = __builtin_amdgcn_exp2f(-fabsf(z));
    const float loss = z > 0.f ? z * VL_LN2 + log1pf(e) : log1pf(e), others = z > 0.f ? 1.f / (1.f + e) : e / (1.f + e);
    if (write) P.loss[row] = weight * (z == z ? loss : z);
    return make_float2(scale * weight, -weight * others);
}
template <typename WT> __device__ __forceinline__ VlRow vl_row(const VlParams& P, int r, int lane, bool write) {
    const int row = P.row0 + r, state = P.state[row];
    const bool counts = vl_counts(P, row);
    float sum = 0.f;
    for (int i = lane; i < P.nsum; i += 64) sum += P.sums[(size_t)r * P.nsum + i];
    sum = wave_sum(sum);
    VlRow y = {counts ? state : VL_ZERO, make_float2(0.f, 0.f)};
    if (y.state == VL_NEAR) y.f = vl_finish<WT>(P, row, __builtin_amdgcn_logf(sum) + VL_SHIFT, 1.f / (sum + 0x1p-64f), write && lane == 0);
    else if (y.state == VL_ZERO && write && lane == 0) P.loss[row] = 0.f;
    return y;
}
// ... a row that is far apart (the workgroup)
template <typename WT> __device__ __forceinline__ void vl_far_row(const VlParams& P, int r, float* s, int tid) {
    constexpr int GE = Traits<WT>::GE, ESZ = Traits<WT>::ESZ;
    const int row = P.row0 + r, target = P.targets[row];
    float* acc = P.alone + (size_t)r * P.H;
    const float2 f = vl_finish<WT>(P, row, vl_row_alone<WT>(P, row, target, acc, s, tid), 1.f, tid == 0);
    if (!P.d_hidden) return;
    for (int c = tid; c < P.H / GE; c += VL_THREADS) {
        float sum[GE], wt[GE];
        load_group<WT>(P.w + ((size_t)target * P.H + c * GE) * ESZ, wt);
#pragma unroll
        for (int u = 0; u < GE; ++u) sum[u] = acc[c * GE + u] * f.x + wt[u] * f.y;
        vl_store_group<WT>(P.d_hidden + ((size_t)row * P.H + c * GE) * ESZ, sum);
    }
}

// Before products that become gradients at once, and where none are wanted: the rows' losses and factors, a workgroup per row, because
// one that is far apart is worked out there (a wavefront per row: 7 us in the place of 12 for 4096 rows, but neighbours that are far apart wait
// for each other: four of them make 10240 rows, H 4096, V 32000 take 240 ms in the place of 68)
template <typename WT>
__global__ void __launch_bounds__(VL_THREADS) vl_rows_kernel(const VlParams P) {
    __shared__ float s[VL_THREADS];
    const int r = blockIdx.x, tid = threadIdx.x;
    const VlRow y = vl_row<WT>(P, r, tid & 63, tid < 64);   // (every wavefront adds the sums up: the same bits)
    __syncthreads();                                        // (... having read the row's state)
    if (tid == 0) {
        P.factor[r] = y.f;
        P.state[P.row0 + r] = y.state == VL_FAR_APART ? VL_DONE : y.state;
    }
    if (y.state == VL_FAR_APART) vl_far_row<WT>(P, r, s, tid);
}

// The loss and the gradient of rows whose products are in parts: a workgroup per row
template <typename WT>
__global__ void __launch_bounds__(VL_THREADS) vl_join_kernel(const VlParams P) {
    constexpr int GE = Traits<WT>::GE, ESZ = Traits<WT>::ESZ;
    __shared__ float s[VL_THREADS];
    const int r = blockIdx.x, row = P.row0 + r, tid = threadIdx.x;
    const VlRow y = vl_row<WT>(P, r, tid & 63, tid < 64);   // (every wavefront adds the sums up: the same bits)
    if (y.state == VL_FAR_APART) {
        vl_far_row<WT>(P, r, s, tid);
        return;
    }
    const char* wt = P.w + (size_t)(y.state == VL_NEAR ? P.targets[row] : 0) * P.H * ESZ;
    for (int c = tid; c < P.H / GE; c += VL_THREADS) {
        float sum[GE], w[GE];
#pragma unroll
        for (int u = 0; u < GE; ++u) sum[u] = 0.f;
        const float* acc = P.acc + (size_t)r * P.H + c * GE;
        for (int i = 0; i < P.splits; ++i, acc += (size_t)P.rows_c * P.H)
#pragma unroll
            for (int q = 0; q < GE; q += 4) {
                const f32x4 v = *reinterpret_cast<const f32x4*>(acc + q);
#pragma unroll
                for (int u = 0; u < 4; ++u) sum[q + u] += v[u];
            }
        load_group<WT>(wt + (size_t)c * 16, w);
#pragma unroll
        for (int u = 0; u < GE; ++u) sum[u] = y.state == VL_NEAR ? sum[u] * y.f.x + w[u] * y.f.y : 0.f;
        vl_store_group<WT>(P.d_hidden + ((size_t)row * P.H + c * GE) * ESZ, sum);
    }
}

int check(const ps_vocab_loss_args* a) {
    if (!a) return PS_ERR_NULL;
    if (a->rows < 1 || a->hidden < 1 || a->vocab < 1 || (a->dtype != PS_F32 && a->dtype != PS_BF16)) return PS_ERR_SHAPE;
    if (a->hidden % (a->dtype == PS_BF16 ? 32 : 16) != 0 || a->hidden > 1 << 16) return PS_ERR_UNSUPPORTED;
    if (a->rows > 1 << 22 || a->vocab > 1 << 23) return PS_ERR_UNSUPPORTED;
    return PS_OK;
}

// How a call is cut: chunks of rows, pieces of the vocabulary, parts of a piece's tokens in the second product
constexpr long long VL_PIECE_BYTES = 288ll << 20;            // of exponentials at a time
constexpr long long VL_PIECE_TILES = 1ll << 22;              // a launch of scores has at most
struct VlPlan {
    int tile, slots;      // 256 (the wide kernels), 128 or 64; workgroups of such tiles that run at a time
    int rows_c, piece, nsum;
    size_t tl, state, factor, sums, acc, alone, x, total;
};
// Where a chunk's tiles of the second product leave workgroups idle, several share a tile's tokens: the fewest that leave the
// least time, counted in rounds of all workgroups over the share of the tokens.  A part costs about as much as more tokens would: its sums
// are written, read and added.  (Counting 1000, 2000 or 5000 in the place of 3000: within 2 %.  500 rows, V 32000: 713 us in one part, 445 in 2, 317 in 4, 263 in 8.)
int splits_of(const VlPlan& L, int hidden, int rows) {
    const int tiles = (rows + L.tile - 1) / L.tile * ((hidden + L.tile - 1) / L.tile), part = L.tile == VW_TILE ? 3000 : 64;
    const int fewest = L.tile == VW_TILE ? 512 : 128;
    int best = 1;
    double least = 0.;
    for (int n = 1; n <= 32 && n * fewest <= std::max(L.piece, fewest); ++n) {
        const double t = (double)((tiles * n + L.slots - 1) / L.slots) * L.piece / n + (double)part * (n > 1 ? n : 0) * (L.tile == VW_TILE ? (double)tiles / L.slots : std::max(1., (double)tiles / L.slots));
        if (n == 1 || t < least) {
            least = t;
            best = n;
        }
    }
    return best;
}
VlPlan plan(const ps_vocab_loss_args* a) {
    const int esz = a->dtype == PS_BF16 ? 2 : 4;
    const bool grad = a->d_hidden != nullptr;
    VlPlan L;
    // Tiles.  The wide kernels where they have a tile for about half of the compute units: us, wide / 128 at H 4096, V 32000: 130 rows (125
    // tiles) 184 / 217, 300 rows 239 / 307; V 128256, 130 rows 512 / 889; H 512, V 2064: 5000 rows (180 tiles) 67 / 71, 1500 (54) 50 / 44.
    // But a tile of few rows: 65 rows 166 / 148 (V 128256, 501 tiles: 489 / 546, 30 rows 483 / 498).
    // 64 / 128: 30 rows 124 / 136 (V 128256 550 / 498), 130 rows 277 / 217; H 512, V 2064: 500 rows 28 / 38.  float32, which is
    // bound by its matrix rate and by few workgroups: 64 always (64 / 128 with kernels as they first were, the latter no longer built: H 256, V 1024: 30
    // rows 29 / 56, 5000 88 / 116; H 512, V 2064, 2000 rows 112 / 153; the first and the last now 25 and 105).
    const bool bf = a->dtype == PS_BF16;
    const long long tiles128 = (long long)((a->vocab + 127) / 128) * ((a->rows + 127) / 128), tiles256 = (long long)((a->vocab + 255) / 256) * ((a->rows + 255) / 256);
    if (bf && tiles256 >= 120 && (a->rows > 96 || tiles256 >= 400)) L.tile = VW_TILE, L.slots = 256;
    else if (!bf || tiles128 < 200 || (a->rows <= 64 && tiles128 < 512)) L.tile = 64, L.slots = 1024;
    else L.tile = 128, L.slots = 512;
    // rows at a time: as many as give the second product one tile for every workgroup that can run
    L.rows_c = std::min(a->rows, std::max(1, L.slots / ((a->hidden + L.tile - 1) / L.tile)) * L.tile);
    const int vocab = (a->vocab + L.tile - 1) / L.tile * L.tile;
    // (losses only: nothing is kept of a piece but sums; its tiles are one launch, whose threads are counted in 32 bits)
    const long long tiles = (long long)(vocab / L.tile) * ((L.rows_c + L.tile - 1) / L.tile);
    const int pieces = (int)(grad ? ((long long)L.rows_c * vocab * esz + VL_PIECE_BYTES - 1) / VL_PIECE_BYTES : (tiles + VL_PIECE_TILES - 1) / VL_PIECE_TILES);
    L.piece = ((vocab + pieces - 1) / pieces + L.tile - 1) / L.tile * L.tile;
    L.nsum = vocab / (L.tile / 2);
    size_t acc = 0;                                          // of all chunks (whole ones, the last)
    if (grad)
        for (const int rows : {L.rows_c, a->rows % L.rows_c})
            if (rows > 0) acc = std::max(acc, (size_t)splits_of(L, a->hidden, rows) * rows * a->hidden * 4);
    L.tl = 0;
    L.state = L.tl + a256((size_t)a->rows * 4);
    L.factor = L.state + a256((size_t)a->rows * 4);
    L.sums = L.factor + a256((size_t)L.rows_c * sizeof(float2));
    L.acc = L.sums + a256((size_t)L.rows_c * L.nsum * 4);
    L.alone = L.acc + a256(acc);
    L.x = L.alone + (grad ? a256((size_t)L.rows_c * a->hidden * 4) : 0);
    L.total = L.x + (grad ? a256((size_t)L.rows_c * L.piece * esz) : 0);
    return L;
}

template <typename WT, int TILE> void launch_score(const VlParams& P, hipStream_t s) {
    hipLaunchKernelGGL((vl_score_kernel<WT, TILE>), dim3((P.nv + TILE - 1) / TILE, (P.rows_c + TILE - 1) / TILE), dim3(VL_THREADS), 0, s, P);
}
template <typename WT, int TILE> void launch_grad(const VlParams& P, hipStream_t s) {
    hipLaunchKernelGGL((vl_grad_kernel<WT, TILE>), dim3((P.H + TILE - 1) / TILE, (P.rows_c + TILE - 1) / TILE, P.splits), dim3(VL_THREADS), 0, s, P);
}

template <typename WT> int run(VlParams P, const VlPlan& L, hipStream_t s) {
    hipLaunchKernelGGL((vl_target_kernel<WT>), dim3((P.rows + 3) / 4), dim3(VL_THREADS), 0, s, P);
    const bool wide = L.tile == VW_TILE;
    const int cols = (P.H + VW_TILE - 1) / VW_TILE;
    for (P.row0 = 0; P.row0 < P.rows; P.row0 += L.rows_c) {
        P.rows_c = std::min(L.rows_c, P.rows - P.row0);
        const int row_tiles = (P.rows_c + VW_TILE - 1) / VW_TILE;
        P.splits = splits_of(L, P.H, P.rows_c);
        P.split_n = ((L.piece + P.splits - 1) / P.splits + L.tile - 1) / L.tile * L.tile;
        const bool at_once = wide && P.splits == 1;          // the last piece's products become gradients
        for (P.v0 = 0; P.v0 < P.V; P.v0 += L.piece) {
            P.nv = std::min(L.piece, P.V - P.v0);
            P.first = P.v0 == 0;
            const int tokens = (P.nv + VW_TILE - 1) / VW_TILE;
            const bool last = P.v0 + L.piece >= P.V;
            if (wide) hipLaunchKernelGGL(vl_score_wide_kernel, dim3(tokens * row_tiles), dim3(VW_THREADS), 0, s, P, tokens, row_tiles);
            else if (L.tile == 64) launch_score<WT, 64>(P, s);
            else if constexpr (Traits<WT>::BF) launch_score<WT, 128>(P, s);
            if (last && (at_once || !P.d_hidden)) hipLaunchKernelGGL((vl_rows_kernel<WT>), dim3(P.rows_c), dim3(VL_THREADS), 0, s, P);
            if (!P.d_hidden) continue;
            if (last && at_once) hipLaunchKernelGGL(vl_grad_wide_kernel<true>, dim3(cols * row_tiles), dim3(VW_THREADS), 0, s, P, cols, row_tiles);
            else if (wide) hipLaunchKernelGGL(vl_grad_wide_kernel<false>, dim3(cols * row_tiles, P.splits), dim3(VW_THREADS), 0, s, P, cols, row_tiles);
            else if (L.tile == 64) launch_grad<WT, 64>(P, s);
            else if constexpr (Traits<WT>::BF) launch_grad<WT, 128>(P, s);
        }
        if (P.d_hidden && !at_once) hipLaunchKernelGGL((vl_join_kernel<WT>), dim3(P.rows_c), dim3(VL_THREADS), 0, s, P);
    }
    return hipGetLastError() == hipSuccess ? PS_OK : PS_ERR_DEVICE;
}

}   // namespace

extern "C" size_t ps_vocab_loss_workspace_bytes(const ps_vocab_loss_args* a) { return check(a) == PS_OK ? plan(a).total : 0; }

extern "C" int ps_vocab_loss(const ps_vocab_loss_args* a, void* stream) {
    const int st = check(a);
    if (st != PS_OK) return st;
    if (!a->h || !a->w_lm || !a->targets || !a->loss || !a->workspace) return PS_ERR_NULL;
    if (((uintptr_t)a->h | (uintptr_t)a->w_lm | (uintptr_t)a->d_hidden) & 15) return PS_ERR_UNSUPPORTED;
    if (((uintptr_t)a->targets | (uintptr_t)a->weights | (uintptr_t)a->loss) & 3) return PS_ERR_UNSUPPORTED;
    const VlPlan L = plan(a);
    if (a->workspace_bytes < L.total || ((uintptr_t)a->workspace & 255)) return PS_ERR_WORKSPACE;
    char* ws = (char*)a->workspace;
    VlParams P = {};
    P.rows = a->rows; P.H = a->hidden; P.V = a->vocab;
    P.ldx = L.piece; P.nsum = L.nsum;
    P.h = (const char*)a->h; P.w = (const char*)a->w_lm; P.targets = a->targets; P.weights = a->weights;
    P.loss = a->loss; P.d_hidden = (char*)a->d_hidden;
    P.tl = (float*)(ws + L.tl); P.state = (int*)(ws + L.state); P.factor = (float2*)(ws + L.factor); P.sums = (float*)(ws + L.sums);
    P.acc = (float*)(ws + L.acc); P.alone = (float*)(ws + L.alone); P.x = a->d_hidden ? ws + L.x : nullptr;
    return a->dtype == PS_BF16 ? run<bf16_t>(P, L, (hipStream_t)stream) : run<float>(P, L, (hipStream_t)stream);
}

// see ps_draft_debug.h
extern "C" int ps_train_debug_loss_plan(const ps_vocab_loss_args* a, int* out) {
    const int st = check(a);
    if (st != PS_OK) return st;
    if (!out) return PS_ERR_NULL;
    const VlPlan L = plan(a);
    const int rest = a->rows % L.rows_c;
    out[0] = L.tile; out[1] = L.rows_c; out[2] = L.piece;
    out[3] = splits_of(L, a->hidden, L.rows_c);
    out[4] = rest ? splits_of(L, a->hidden, rest) : out[3];
    out[5] = (std::min(L.piece, a->vocab) + L.tile - 1) / L.tile * ((L.rows_c + L.tile - 1) / L.tile);
    return PS_OK;
}

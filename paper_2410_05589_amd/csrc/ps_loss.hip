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
//   vl_score_kernel   W h^T, one tile of 128 x 128 per workgroup: exponentials to the workspace (storage type), sums of rows beside them
//   vl_grad_kernel    exponentials . W, added to what the pieces before left, in float32
// then vl_finish_kernel adds up the rows' sums and makes losses and gradients of them.
#include <math.h>

#include "ps_train_device.h"

namespace {

constexpr int VL_THREADS = 256, VL_TILE = 128;
constexpr float VL_SHIFT = 64.f, VL_FAR = 80.f, VL_LOG2E = 1.4426950408889634f, VL_LN2 = 0.6931471805599453f;

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
    float *tl, *sums, *acc;           // target logits; sums [rows_c][nsum]; products [splits][rows_c][H]
    int* far;                         // rows whose logits lie too far apart
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
        P.far[row] = 0;
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

template <typename WT>
__global__ void __launch_bounds__(VL_THREADS, 2) vl_score_kernel(const VlParams P) {
    constexpr int ESZ = Traits<WT>::ESZ, BUF = VL_TILE * 64;
    __shared__ __attribute__((aligned(16))) char smem[4 * BUF];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, half = lane >> 5;
    const int vt = blockIdx.x * VL_TILE, rt = blockIdx.y * VL_TILE;   // in the piece, in the chunk
    const int wv = (wave & 1) * 64, wr = (wave >> 1) * 64;
    const size_t rb = (size_t)P.H * ESZ;
    const char *wsrc[2], *hsrc[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        wsrc[i] = P.w + (size_t)min(P.v0 + vt + tid / 4 + 64 * i, P.V - 1) * rb + (tid & 3) * 16;
        hsrc[i] = P.h + (size_t)(P.row0 + min(rt + tid / 4 + 64 * i, P.rows_c - 1)) * rb + (tid & 3) * 16;
    }
    uint4 sw[2], sh[2];
    auto load = [&](int k) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 2; ++i) { sw[i] = ld16(wsrc[i] + (size_t)k * 64); sh[i] = ld16(hsrc[i] + (size_t)k * 64); }
    };
    auto store = [&](int k) __attribute__((always_inline)) {
        char* b = smem + (k & 1) * 2 * BUF;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            *reinterpret_cast<uint4*>(b + vl_at(tid / 4 + 64 * i, tid & 3)) = sw[i];
            *reinterpret_cast<uint4*>(b + BUF + vl_at(tid / 4 + 64 * i, tid & 3)) = sh[i];
        }
    };
    f32x16 acc[2][2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    const int steps = P.H * ESZ / 64;
    load(0);
    store(0);
    if (steps > 1) load(1);
    __syncthreads();
    for (int k = 0; k < steps; ++k) {
        if (k + 1 < steps) store(k + 1);
        if (k + 2 < steps) load(k + 2);
        const char* b = smem + (k & 1) * 2 * BUF;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            uint4 a[2], q[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                a[i] = ld16(b + vl_at(wv + 32 * i + c, 2 * t + half));
                q[i] = ld16(b + BUF + vl_at(wr + 32 * i + c, 2 * t + half));
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) vl_mma<WT>(a[i], q[j], acc[i][j]);
        }
        __syncthreads();
    }
    // ---- lane (c, half) holds of row 32 j + c the tokens 32 i + 8 (e / 4) + 4 half + e % 4
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int r = rt + wr + 32 * j + c, row = P.row0 + min(r, P.rows_c - 1);
        const int t = P.targets[row] - P.v0 - vt - wv - 4 * half, end = P.V - P.v0 - vt - wv - 4 * half;
        const float ref = -P.tl[row] * VL_LOG2E - VL_SHIFT;
        float sum = 0.f;
        bool far = false;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                f32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int at = 32 * i + 8 * q + e;
                    const float y = fmaf(acc[i][j][4 * q + e], VL_LOG2E, ref);
                    const bool in = at != t && at < end;
                    far |= in && y > VL_FAR && y < INFINITY;
                    v[e] = in ? __builtin_amdgcn_exp2f(y) : 0.f;
                    sum += v[e];
                }
                if (P.x && r < P.rows_c) store4<WT>(P.x + ((size_t)r * P.ldx + vt + wv + 32 * i + 8 * q + 4 * half) * ESZ, v);
            }
        const auto sw2 = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum), __float_as_uint(sum), false, false);
        sum = __uint_as_float(sw2[0]) + __uint_as_float(sw2[1]);
        if (r < P.rows_c) {
            if (far) P.far[row] = 1;
            if (half == 0) P.sums[(size_t)r * P.nsum + (P.v0 + vt + wv) / 64] = sum;
        }
    }
}

template <typename WT>
__global__ void __launch_bounds__(VL_THREADS, 2) vl_grad_kernel(const VlParams P) {
    constexpr int ESZ = Traits<WT>::ESZ, KV = 64 / ESZ;      // tokens of a step
    constexpr int ABUF = VL_TILE * 64, WSTR = VL_TILE * ESZ + (Traits<WT>::BF ? 64 : 32), WBUF = KV * WSTR, BUF = ABUF + WBUF;
    __shared__ __attribute__((aligned(16))) char smem[2 * BUF];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 31, half = lane >> 5;
    const int ct = blockIdx.x * VL_TILE, rt = blockIdx.y * VL_TILE, split = blockIdx.z;
    const int wc = (wave & 1) * 64, wr = (wave >> 1) * 64;
    const int k0 = split * (P.split_n / KV), k1 = min((split + 1) * P.split_n, (P.nv + KV - 1) / KV * KV) / KV;
    constexpr int TPV = VL_TILE * ESZ / 16;                  // 16-byte pieces of a staged row of W
    const char* xsrc[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) xsrc[i] = P.x + (size_t)min(rt + tid / 4 + 64 * i, P.rows_c - 1) * P.ldx * ESZ + (tid & 3) * 16;
    const int wk = tid / TPV, wp = tid % TPV;                // this thread's tokens wk + (256 / TPV) i, its piece (beyond H: the last)
    const size_t wcol = (size_t)min(ct * ESZ + wp * 16, P.H * ESZ - 16);
    uint4 sx[2], sw[2];
    auto load = [&](int k) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            sx[i] = ld16(xsrc[i] + (size_t)k * 64);
            sw[i] = ld16(P.w + (size_t)min(P.v0 + k * KV + wk + VL_THREADS / TPV * i, P.V - 1) * P.H * ESZ + wcol);
        }
    };
    auto store = [&](int k) __attribute__((always_inline)) {
        char* b = smem + (k & 1) * BUF;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            *reinterpret_cast<uint4*>(b + vl_at(tid / 4 + 64 * i, tid & 3)) = sx[i];
            *reinterpret_cast<uint4*>(b + ABUF + (wk + VL_THREADS / TPV * i) * WSTR + wp * 16) = sw[i];
        }
    };
    f32x16 acc[2][2];
    float* out = P.acc + (size_t)split * P.rows_c * P.H;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
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
    if (k0 < k1) {
        load(k0);
        store(k0);
        if (k0 + 1 < k1) load(k0 + 1);
        __syncthreads();
        for (int k = k0; k < k1; ++k) {
            if (k + 1 < k1) store(k + 1);
            if (k + 2 < k1) load(k + 2);
            const char* b = smem + (k & 1) * BUF;
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                uint4 a[2], q[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    a[i] = ld16(b + vl_at(wr + 32 * i + c, 2 * t + half));
                    q[i] = column(b, t, i);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) vl_mma<WT>(a[i], q[j], acc[i][j]);
            }
            __syncthreads();
        }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int r = rt + wr + 32 * i + 8 * (e / 4) + 4 * half + e % 4, col = ct + wc + 32 * j + c;
                if (r < P.rows_c && col < P.H) out[(size_t)r * P.H + col] = acc[i][j][e];
            }
}

// sum over the workgroup in a fixed order, for every thread
__device__ __forceinline__ float vl_block_sum(float v, float* s, int tid) {
    v = wave_sum(v);
    __syncthreads();
    if ((tid & 63) == 0) s[tid >> 6] = v;
    __syncthreads();
    return (s[0] + s[1]) + (s[2] + s[3]);
}

// A row whose logits lie too far above its target's: its maximum, then sums against it, 256 tokens at a time.  Returns log2 of
// sum_{v != t} exp(l_v - l_t); acc (of the row, float32) becomes sum_{v != t} p_v W_v.  One workgroup reads the whole LM head twice.
template <typename WT>
__device__ __attribute__((noinline)) float vl_row_alone(const VlParams& P, int row, int target, float* acc, float* s, int tid) {
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
    const float z = top + __builtin_amdgcn_logf(total) - P.tl[row] * VL_LOG2E;
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

template <typename WT>
__global__ void __launch_bounds__(VL_THREADS) vl_finish_kernel(const VlParams P) {
    constexpr int GE = Traits<WT>::GE, ESZ = Traits<WT>::ESZ;
    __shared__ float s[VL_THREADS];
    const int tid = threadIdx.x, r = blockIdx.x, row = P.row0 + r;
    char* out = P.d_hidden ? P.d_hidden + (size_t)row * P.H * ESZ : nullptr;
    if (!vl_counts(P, row)) {
        if (tid == 0) P.loss[row] = 0.f;
        for (int c = tid; out && c < P.H / GE; c += VL_THREADS) *reinterpret_cast<uint4*>(out + (size_t)c * 16) = make_uint4(0u, 0u, 0u, 0u);
        return;
    }
    const int target = P.targets[row];
    const float weight = P.weights ? P.weights[row] : 1.f;
    float* acc = P.acc + (size_t)r * P.H;
    float z, scale = 1.f;                                    // log2 of sum_{v != t} exp(l_v - l_t)
    int splits = P.splits;
    if (P.far[row]) {
        z = vl_row_alone<WT>(P, row, target, acc, s, tid);
        splits = 1;
    } else {
        float sum = 0.f;
        for (int i = tid; i < P.nsum; i += VL_THREADS) sum += P.sums[(size_t)r * P.nsum + i];
        sum = vl_block_sum(sum, s, tid);
        z = __builtin_amdgcn_logf(sum) + VL_SHIFT;
        scale = 1.f / (sum + 0x1p-64f);
    }
    // log(1 + 2^z) and 2^z / (1 + 2^z)
    const float e = __builtin_amdgcn_exp2f(-fabsf(z));
    const float loss = z > 0.f ? z * VL_LN2 + log1pf(e) : log1pf(e), others = z > 0.f ? 1.f / (1.f + e) : e / (1.f + e);
    if (tid == 0) P.loss[row] = weight * (z == z ? loss : z);
    if (!out) return;
    scale *= weight;
    const float back = -weight * others;
    for (int c = tid; c < P.H / GE; c += VL_THREADS) {
        float sum[GE], wt[GE];
#pragma unroll
        for (int e4 = 0; e4 < GE; e4 += 4) *reinterpret_cast<f32x4*>(sum + e4) = *reinterpret_cast<const f32x4*>(acc + c * GE + e4);
        for (int i = 1; i < splits; ++i)
#pragma unroll
            for (int e4 = 0; e4 < GE; e4 += 4) {
                const f32x4 v = *reinterpret_cast<const f32x4*>(acc + (size_t)i * P.rows_c * P.H + c * GE + e4);
#pragma unroll
                for (int u = 0; u < 4; ++u) sum[e4 + u] += v[u];
            }
        load_group<WT>(P.w + ((size_t)target * P.H + c * GE) * ESZ, wt);
        uint4 v;
        unsigned* o = &v.x;
#pragma unroll
        for (int u = 0; u < GE; ++u) sum[u] = sum[u] * scale + wt[u] * back;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            if constexpr (Traits<WT>::BF) o[u] = pack_bf16x2(sum[2 * u], sum[2 * u + 1]);
            else o[u] = __float_as_uint(sum[u]);
        }
        *reinterpret_cast<uint4*>(out + (size_t)c * 16) = v;
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
struct VlPlan {
    int rows_c, piece, splits, split_n, nsum;
    size_t tl, far, sums, acc, x, total;
};
VlPlan plan(const ps_vocab_loss_args* a) {
    const int esz = a->dtype == PS_BF16 ? 2 : 4, tile = VL_TILE;
    const bool grad = a->d_hidden != nullptr;
    VlPlan L;
    const int chunks = (a->rows + 4095) / 4096;
    L.rows_c = std::min(a->rows, ((a->rows + chunks - 1) / chunks + tile - 1) / tile * tile);
    const int row_tiles = (L.rows_c + tile - 1) / tile, vocab = (a->vocab + tile - 1) / tile * tile;
    const int pieces = grad ? (int)(((long long)L.rows_c * vocab * esz + (128 << 20) - 1) / (128 << 20)) : 1;
    L.piece = ((vocab + pieces - 1) / pieces + tile - 1) / tile * tile;
    // few tiles of the second product: several workgroups share a tile's tokens, of which each keeps at least 512
    const int tiles = row_tiles * ((a->hidden + tile - 1) / tile);
    L.splits = grad ? std::max(1, std::min(512 / tiles, L.piece / 512)) : 1;
    L.split_n = ((L.piece + L.splits - 1) / L.splits + tile - 1) / tile * tile;
    L.splits = (L.piece + L.split_n - 1) / L.split_n;
    L.nsum = vocab / 64;
    L.tl = 0;
    L.far = L.tl + a256((size_t)a->rows * 4);
    L.sums = L.far + a256((size_t)a->rows * 4);
    L.acc = L.sums + a256((size_t)L.rows_c * L.nsum * 4);
    L.x = L.acc + (grad ? a256((size_t)L.splits * L.rows_c * a->hidden * 4) : 0);
    L.total = L.x + (grad ? a256((size_t)L.rows_c * L.piece * esz) : 0);
    return L;
}

template <typename WT> int run(VlParams P, const VlPlan& L, hipStream_t s) {
    hipLaunchKernelGGL((vl_target_kernel<WT>), dim3((P.rows + 3) / 4), dim3(VL_THREADS), 0, s, P);
    for (P.row0 = 0; P.row0 < P.rows; P.row0 += L.rows_c) {
        P.rows_c = std::min(L.rows_c, P.rows - P.row0);
        const unsigned row_tiles = (P.rows_c + VL_TILE - 1) / VL_TILE;
        for (P.v0 = 0; P.v0 < P.V; P.v0 += L.piece) {
            P.nv = std::min(L.piece, P.V - P.v0);
            P.first = P.v0 == 0;
            hipLaunchKernelGGL((vl_score_kernel<WT>), dim3((P.nv + VL_TILE - 1) / VL_TILE, row_tiles), dim3(VL_THREADS), 0, s, P);
            if (P.d_hidden)
                hipLaunchKernelGGL((vl_grad_kernel<WT>), dim3((P.H + VL_TILE - 1) / VL_TILE, row_tiles, L.splits), dim3(VL_THREADS), 0, s, P);
        }
        hipLaunchKernelGGL((vl_finish_kernel<WT>), dim3(P.rows_c), dim3(VL_THREADS), 0, s, P);
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
    P.ldx = L.piece; P.nsum = L.nsum; P.splits = L.splits; P.split_n = L.split_n;
    P.h = (const char*)a->h; P.w = (const char*)a->w_lm; P.targets = a->targets; P.weights = a->weights;
    P.loss = a->loss; P.d_hidden = (char*)a->d_hidden;
    P.tl = (float*)(ws + L.tl); P.far = (int*)(ws + L.far); P.sums = (float*)(ws + L.sums);
    P.acc = (float*)(ws + L.acc); P.x = a->d_hidden ? ws + L.x : nullptr;
    return a->dtype == PS_BF16 ? run<bf16_t>(P, L, (hipStream_t)stream) : run<float>(P, L, (hipStream_t)stream);
}

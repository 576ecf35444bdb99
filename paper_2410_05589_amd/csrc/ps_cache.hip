// The target's KV cache in 8 bits: rows of keys and values to blocks of e4m3 codes with a scale each, and back (see include/ps_verify.h).
//
//   s = 2^e, the least e >= -100 with max |x| <= 448 2^e;  code = e4m3(x / s);  value = code * s
//
// Both are memory-bound: a block of 32 positions of one head is 32 rows of the caller's (64 ... 512 bytes each, a row of all heads apart)
// and one contiguous piece of codes (2 or 4 KiB).  One wavefront takes one block of one head's keys or values: rows are read and
// written by whole lines, the bytes meet in LDS by row, codes leave and arrive 16 bytes a lane in the attention's order.  Values lie
// transposed in that order (a lane of the attention has 16 positions of one dim), so they pass 4 x 4 byte exchanges.
//
// Measured (bf16, 8 heads of 128): 8 x 2048 rows written 22 to 25 us (67 MB read, 34 MB written, 4.0 to 4.5 TB/s), 4 x 4096 read back 19.6 (5.1 TB/s, a copy's rate); a path of up to 6
// rows for 8 sequences, 32 heads 6.8, a launch and three reads one after the other (length, path, rows).  Writing is behind reading for the two looks at each
// row (largest magnitude, then codes; they wait in registers) and the codes' turn through LDS; loads that pass the caches by change nothing.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ps_cache_device.h"

namespace {

// blocks a workgroup takes (us, one / four / sixteen: 8 x 2048 rows of 8 heads written 21.1 / 23.3 / 23.4, read 20.3 / 19.7 / 17.6; 8192 rows of 32 heads written 48 / 50 / 56,
// read 39 / 37 / 41; 40 heads written 60 / 60 / 58, read 49 / 47 / 50): writing, whose wavefronts take different times, leaves each its own
constexpr int PC_WRITERS = 1, PC_WAVES = 4;

struct PcParams {
    const char *k, *v;        // rows (write: read; read: written)
    uint8_t *k_codes, *v_codes;
    float *k_scale, *v_scale;
    long long row_bytes;      // between rows
    int rows, heads;          // rows per sequence in k and v
    const int *len_dev, *n_accepted, *path;
    int path_rows;
    int* len_out;
    unsigned first[PC_SEQS];  // the sequence's first block
    int len[PC_SEQS];         // write: its length (bound); read: first position
    int n[PC_SEQS];           // rows to write or read (at most)
};

__device__ __forceinline__ void wave_sync() {   // LDS written by a wavefront's lanes for its others
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// 8 elements of a row as they are, and as floats
template <typename WT> struct Eight;
template <> struct Eight<bf16_t> {
    uint4 v;
    __device__ __forceinline__ void load(const char* p) { v = ld16_q(p); }
    __device__ __forceinline__ void keep() { asm volatile("" : "+v"(v.x), "+v"(v.y), "+v"(v.z), "+v"(v.w)); }   // (its floats are made again, not kept: registers)
    __device__ __forceinline__ unsigned word(int i) const { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }
    __device__ __forceinline__ float get(int e) const { return __uint_as_float(e & 1 ? word(e >> 1) & 0xFFFF0000u : word(e >> 1) << 16); }
};
template <> struct Eight<float> {
    f32x4 lo, hi;
    __device__ __forceinline__ void load(const char* p) { lo = load4_q<float>(p); hi = load4_q<float>(p + 16); }
    __device__ __forceinline__ void keep() {}
    __device__ __forceinline__ float get(int e) const { return e < 4 ? lo[e & 3] : hi[e & 3]; }
};
template <typename WT> __device__ __forceinline__ void store8(char* p, const float (&x)[8]) {
    if constexpr (Traits<WT>::BF) {
        *reinterpret_cast<u32x4_q*>(p) = u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
    } else {
        *reinterpret_cast<f32x4_q*>(p) = f32x4{x[0], x[1], x[2], x[3]};
        *reinterpret_cast<f32x4_q*>(p + 16) = f32x4{x[4], x[5], x[6], x[7]};
    }
}

// old codes at a scale that has grown: c * ratio, rounded again
__device__ __forceinline__ unsigned again(unsigned v, float ratio) {
    const f32x4 x = unpack_e4m3x4(v) * ratio;
    return pack_e4m3x4(x[0], x[1], x[2], x[3]);
}

// the scale for a largest magnitude (its bits): the least power of two, 2^-100 or more, that brings it to 448 = 1.75 * 2^8 or below
__device__ __forceinline__ float scale_for(unsigned amax) {
    const int e = (int)(amax >> 23) - 8 + ((amax & 0x7FFFFF) > 0x600000);
    return __uint_as_float((unsigned)max(e, 127 - 100) << 23);
}

template <typename WT, int D>
__global__ __launch_bounds__(64 * PC_WRITERS) void cache_write_kernel(const PcParams P) {
    constexpr int PITCH = D + 16, LR = D / 8, RP = 64 / LR, PASSES = PC_BLOCK / RP, TILE = PC_BLOCK * D;
    __shared__ __attribute__((aligned(16))) unsigned char s_tile[PC_WRITERS][PC_BLOCK * PITCH];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int task = blockIdx.x * PC_WRITERS + wave, b = blockIdx.z;
    const int len = pc_length(P.len_dev, b, P.len[b]);
    int count = P.n[b], node = 0;
    if (P.n_accepted) {                                     // lane i + 1: the path's entry i; lane 0: node 0
        node = lane > 0 && lane <= P.path_rows ? P.path[(size_t)b * P.path_rows + lane - 1] : 0;
        const int acc = min(P.n_accepted[b], P.path_rows);
        const u64 good = __ballot(lane <= acc && (unsigned)node < (unsigned)P.rows);
        count = ~good ? __builtin_ctzll(~good) : 64;
    }
    if (P.len_out && task == 0 && blockIdx.y == 0 && lane == 0) P.len_out[b] = len + count;
    if (task >= 2 * P.heads) return;
    const bool value = task >= P.heads;
    const int h = value ? task - P.heads : task;
    const int block = (len >> 5) + (int)blockIdx.y;         // block of the sequence
    const int t0 = blockIdx.y == 0 ? len & 31 : 0;          // positions it has already
    const int from = (int)blockIdx.y * 32 + t0 - (len & 31);  // the first row that goes there
    const int n = min(count - from, 32 - t0);
    if (n <= 0) return;

    const char* rows = (value ? P.v : P.k) + (long long)b * P.rows * P.row_bytes + (long long)h * D * Traits<WT>::ESZ;
    const size_t at = (size_t)(P.first[b] + (unsigned)block) * P.heads + h;
    unsigned char* tile = (value ? P.v_codes : P.k_codes) + at * TILE;
    float* scale = (value ? P.v_scale : P.k_scale) + at;
    const float was = t0 ? *scale : 0.f;
    uint4 old[D / 32];                                      // the codes that are there (asked for together with the rows)
    if (t0)
#pragma unroll
        for (int c = 0; c < D / 32; ++c) old[c] = ld16(tile + c * 1024 + lane * 16);
    const int li = lane % LR, lr = lane / LR;

    Eight<WT> x[PASSES] = {};
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int t = i * RP + lr, row = from + t - t0;
        const int src = P.n_accepted ? __shfl(node, row & 63) : row;
        if (t >= t0 && t < t0 + n) x[i].load(rows + (long long)src * P.row_bytes + li * 8 * Traits<WT>::ESZ);
    }
    unsigned amax = 0;
#pragma unroll
    for (int i = 0; i < PASSES; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) amax = max(amax, __float_as_uint(x[i].get(e)) & 0x7FFFFFFFu);
    amax = wave_max_u32(amax);
    const bool odd = amax >= 0x7F800000u;                   // Inf or NaN among them: they do not count for the scale
    if (odd) {
#pragma unroll
        for (int i = 0; i < PASSES; ++i) x[i].keep();
        amax = 0;
#pragma unroll
        for (int i = 0; i < PASSES; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const unsigned m = __float_as_uint(x[i].get(e)) & 0x7FFFFFFFu;
                amax = max(amax, m < 0x7F800000u ? m : 0u);
            }
        amax = wave_max_u32(amax);
    }
    const float s = fmaxf(scale_for(amax), was), inv = 1.f / s;   // (powers of two: exact)

    unsigned char* mem = s_tile[wave];
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int t = i * RP + lr;
        float y[8];
        x[i].keep();
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = x[i].get(e) * inv;
        if (odd)
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = __builtin_fabsf(x[i].get(e)) < __builtin_inff() ? y[e] : __uint_as_float(0x7FC00000u);
        if (t >= t0) *reinterpret_cast<uint2*>(mem + t * PITCH + li * 8) = make_uint2(pack_e4m3x4(y[0], y[1], y[2], y[3]), pack_e4m3x4(y[4], y[5], y[6], y[7]));
    }
    if (t0) {
        const bool grown = s > was;
        const float ratio = was * inv;
        const int r = lane & 31, half = lane >> 5;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
            uint4 v = old[c];
            if (grown) v = make_uint4(again(v.x, ratio), again(v.y, ratio), again(v.z, ratio), again(v.w, ratio));
            if (!value) {
                if (r < t0) *reinterpret_cast<uint4*>(mem + r * PITCH + c * 32 + half * 16) = v;
            } else {
                const unsigned w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int t = 8 * (i >> 2) + 4 * half + (i & 3);
                    if (t < t0) mem[t * PITCH + c * 32 + r] = (unsigned char)(w[i >> 2] >> (8 * (i & 3)));
                }
            }
        }
    }
    wave_sync();
    if (!value) {
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
            *reinterpret_cast<uint4*>(tile + c * 1024 + lane * 16) = *reinterpret_cast<const uint4*>(mem + (lane & 31) * PITCH + c * 32 + (lane >> 5) * 16);
    } else if (lane < 2 * (D / 4)) {
        const int q = lane % (D / 4), half = lane / (D / 4);   // dims 4 q .. 4 q + 3
        unsigned o[4][4];
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            unsigned w[4], y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = *reinterpret_cast<const unsigned*>(mem + (8 * a + 4 * half + i) * PITCH + 4 * q);
            turn4x4(w, y);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e][a] = y[e];
        }
        unsigned char* to = tile + ((q / 8 * 2 + half) * 32 + q % 8 * 4) * 16;
#pragma unroll
        for (int e = 0; e < 4; ++e) *reinterpret_cast<uint4*>(to + e * 16) = make_uint4(o[e][0], o[e][1], o[e][2], o[e][3]);
    }
    if (lane == 0) *scale = s;
}

// the new lengths, where they take the place of the ones that the write reads
__global__ void cache_length_kernel(const PcParams P) {
    const int b = threadIdx.x;
    int count = P.n[b];
    if (P.n_accepted) {
        const int acc = min(P.n_accepted[b], P.path_rows);
        count = acc < 0 ? 0 : 1;
        while (count > 0 && count <= acc && (unsigned)P.path[(size_t)b * P.path_rows + count - 1] < (unsigned)P.rows) ++count;
    }
    P.len_out[b] = pc_length(P.len_dev, b, P.len[b]) + count;
}

template <typename WT, int D>
__global__ __launch_bounds__(64 * PC_WAVES) void cache_read_kernel(const PcParams P) {
    constexpr int PITCH = D + 16, LR = D / 8, RP = 64 / LR, PASSES = PC_BLOCK / RP, TILE = PC_BLOCK * D;
    __shared__ __attribute__((aligned(16))) unsigned char s_tile[PC_WAVES][PC_BLOCK * PITCH];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int task = blockIdx.x * PC_WAVES + wave, b = blockIdx.z;
    if (task >= 2 * P.heads) return;
    const bool value = task >= P.heads;
    char* out = const_cast<char*>(value ? P.v : P.k);
    if (!out) return;
    const int h = value ? task - P.heads : task;
    const int start = P.len[b], block = (start >> 5) + (int)blockIdx.y;
    const int t0 = blockIdx.y == 0 ? start & 31 : 0, from = (int)blockIdx.y * 32 + t0 - (start & 31);
    const int n = min(P.n[b] - from, 32 - t0);
    if (n <= 0) return;
    out += ((long long)b * P.rows + from) * P.row_bytes + (long long)h * D * Traits<WT>::ESZ;
    const size_t at = (size_t)(P.first[b] + (unsigned)block) * P.heads + h;
    const unsigned char* tile = (value ? P.v_codes : P.k_codes) + at * TILE;
    const float scale = (value ? P.v_scale : P.k_scale)[at];

    unsigned char* mem = s_tile[wave];
    if (!value) {
#pragma unroll
        for (int c = 0; c < D / 32; ++c)
            *reinterpret_cast<uint4*>(mem + (lane & 31) * PITCH + c * 32 + (lane >> 5) * 16) = ldg_stream16(tile + c * 1024 + lane * 16);
    } else if (lane < 2 * (D / 4)) {
        const int q = lane % (D / 4), half = lane / (D / 4);
        const unsigned char* src = tile + ((q / 8 * 2 + half) * 32 + q % 8 * 4) * 16;
        uint4 v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = ld16(src + e * 16);
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            unsigned w[4], y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = a == 0 ? v[e].x : a == 1 ? v[e].y : a == 2 ? v[e].z : v[e].w;
            turn4x4(w, y);
#pragma unroll
            for (int i = 0; i < 4; ++i) *reinterpret_cast<unsigned*>(mem + (8 * a + 4 * half + i) * PITCH + 4 * q) = y[i];
        }
    }
    wave_sync();
    const int li = lane % LR, lr = lane / LR;
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int t = i * RP + lr;
        const uint2 v = *reinterpret_cast<const uint2*>(mem + t * PITCH + li * 8);
        const f32x4 lo = unpack_e4m3x4(v.x) * scale, hi = unpack_e4m3x4(v.y) * scale;
        const float x[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        if (t >= t0 && t < t0 + n) store8<WT>(out + (long long)(t - t0) * P.row_bytes + li * 8 * Traits<WT>::ESZ, x);
    }
}

// what write and read check alike; n: the most rows per sequence
template <typename A> int check(const A* a, PcParams& P) {
    if (a->rows < 1) return PS_ERR_SHAPE;
    if (a->dtype != PS_F32 && a->dtype != PS_BF16) return PS_ERR_SHAPE;
    const int st = pc_check(a->cache, a->batch);
    if (st != PS_OK) return st;
    if (!aligned4(a->k_rows) || !aligned4(a->v_rows)) return PS_ERR_UNSUPPORTED;
    int64_t bytes = 0;
    const int sst = pc_stride(a->row_stride, (int64_t)a->cache->n_kv_heads * a->cache->head_dim, a->dtype, &bytes);
    if (sst != PS_OK) return sst;
    P.k = (const char*)a->k_rows; P.v = (const char*)a->v_rows;
    P.k_codes = a->cache->k_codes; P.v_codes = a->cache->v_codes; P.k_scale = a->cache->k_scale; P.v_scale = a->cache->v_scale;
    P.row_bytes = bytes; P.rows = a->rows; P.heads = a->cache->n_kv_heads;
    for (int b = 0; b < a->batch; ++b) {
        P.first[b] = (unsigned)(a->cache->kv_offsets[b] / PC_BLOCK);
        P.n[b] = a->n_seq ? a->n_seq[b] : a->rows;
        if (P.n[b] < 0 || P.n[b] > a->rows) return PS_ERR_SHAPE;
    }
    return PS_OK;
}
// positions 0 .. tokens - 1 of a sequence: its blocks have them, and the kernels' 32-bit lengths
int fits(const ps_cache* c, int b, long long tokens) {
    return tokens > c->kv_offsets[b + 1] - c->kv_offsets[b] ? PS_ERR_KV_CAPACITY : tokens > INT32_MAX ? PS_ERR_UNSUPPORTED : PS_OK;
}

template <typename F> int launch(int dtype, int d, F go) {
    if (dtype == PS_BF16) { if (d == 128) go(bf16_t{}, std::integral_constant<int, 128>{}); else go(bf16_t{}, std::integral_constant<int, 64>{}); }
    else if (d == 128) go(float{}, std::integral_constant<int, 128>{});
    else go(float{}, std::integral_constant<int, 64>{});
    return hipGetLastError() == hipSuccess ? PS_OK : PS_ERR_DEVICE;
}

}   // namespace

extern "C" int ps_cache_write(const ps_cache_write_args* a, void* stream) {
    if (!a || !a->k_rows || !a->v_rows || !a->kv_len || !a->n_accepted != !a->path) return PS_ERR_NULL;
    PcParams P = {};
    const int st = check(a, P);
    if (st != PS_OK) return st;
    if (a->path && (a->n_seq || a->path_rows < 1 || a->path_rows >= PS_TREE_MAX_NODES)) return PS_ERR_SHAPE;
    if (!aligned4(a->kv_len_dev) || !aligned4(a->n_accepted) || !aligned4(a->path) || !aligned4(a->len_out)) return PS_ERR_UNSUPPORTED;
    P.len_dev = a->kv_len_dev; P.n_accepted = a->n_accepted; P.path = a->path; P.path_rows = a->path ? a->path_rows : 0;
    int most = 0;
    for (int b = 0; b < a->batch; ++b) {
        P.len[b] = a->kv_len[b];
        if (P.len[b] < 0) return PS_ERR_SHAPE;
        if (a->path) P.n[b] = 1 + a->path_rows;
        const int fit = fits(a->cache, b, (long long)P.len[b] + P.n[b]);
        if (fit != PS_OK) return fit;
        // blocks that this many positions can touch (where the device has the length: wherever they start)
        const int start = a->kv_len_dev ? PC_BLOCK - 1 : P.len[b] % PC_BLOCK;
        most = std::max(most, P.n[b] ? (int)(((long long)start + P.n[b] + PC_BLOCK - 1) / PC_BLOCK) : 0);
    }
    if (most > 65535) return PS_ERR_UNSUPPORTED;
    const bool in_place = a->len_out && a->len_out == a->kv_len_dev;
    P.len_out = in_place ? nullptr : a->len_out;
    const dim3 grid((2 * P.heads + PC_WRITERS - 1) / PC_WRITERS, std::max(most, 1), a->batch);
    const int launched = launch(a->dtype, a->cache->head_dim, [&](auto wt, auto d) {
        hipLaunchKernelGGL((cache_write_kernel<decltype(wt), decltype(d)::value>), grid, dim3(64 * PC_WRITERS), 0, (hipStream_t)stream, P);
    });
    if (launched != PS_OK || !in_place) return launched;
    P.len_out = a->len_out;
    hipLaunchKernelGGL(cache_length_kernel, dim3(1), dim3(a->batch), 0, (hipStream_t)stream, P);
    return hipGetLastError() == hipSuccess ? PS_OK : PS_ERR_DEVICE;
}

extern "C" int ps_cache_read(const ps_cache_read_args* a, void* stream) {
    if (!a || (!a->k_rows && !a->v_rows)) return PS_ERR_NULL;
    PcParams P = {};
    const int st = check(a, P);
    if (st != PS_OK) return st;
    int most = 0;
    for (int b = 0; b < a->batch; ++b) {
        P.len[b] = a->start ? a->start[b] : 0;
        if (P.len[b] < 0) return PS_ERR_SHAPE;
        const int fit = fits(a->cache, b, (long long)P.len[b] + P.n[b]);
        if (fit != PS_OK) return fit;
        most = std::max(most, P.n[b] ? (int)(((long long)P.len[b] % PC_BLOCK + P.n[b] + PC_BLOCK - 1) / PC_BLOCK) : 0);
    }
    if (most > 65535) return PS_ERR_UNSUPPORTED;
    if (most == 0) return PS_OK;
    const dim3 grid((2 * P.heads + PC_WAVES - 1) / PC_WAVES, most, a->batch);
    return launch(a->dtype, a->cache->head_dim, [&](auto wt, auto d) {
        hipLaunchKernelGGL((cache_read_kernel<decltype(wt), decltype(d)::value>), grid, dim3(64 * PC_WAVES), 0, (hipStream_t)stream, P);
    });
}

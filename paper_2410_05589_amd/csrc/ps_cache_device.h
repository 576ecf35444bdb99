// What the kernels on the target's 8-bit cache share (ps_cache.hip: write and read; ps_tree_attn.hip): e4m3 numbers, the checks of a cache.
// The layout of a block is stated in include/ps_verify.h.
#pragma once
#include "ps_train_device.h"   // (accesses aligned to 4 bytes)
#include "ps_verify.h"

namespace {

constexpr int PC_BLOCK = PS_CACHE_BLOCK, PC_SEQS = PS_CACHE_MAX_BATCH;
static_assert(PC_BLOCK == 32, "the layout is that of 32 x 32 matrix tiles");

// two / four floats to e4m3, ties to even; magnitudes up to 448 or NaN
__device__ __forceinline__ unsigned pack_e4m3x4(float a, float b, float c, float d) {
    return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}
__device__ __forceinline__ f32x4 unpack_e4m3x4(unsigned v) {
    return f32x4{__builtin_amdgcn_cvt_f32_fp8((int)v, 0), __builtin_amdgcn_cvt_f32_fp8((int)v, 1),
                 __builtin_amdgcn_cvt_f32_fp8((int)v, 2), __builtin_amdgcn_cvt_f32_fp8((int)v, 3)};
}

// 4 x 4 bytes turned: out[e] byte b = w[b] byte e
__device__ __forceinline__ void turn4x4(const unsigned (&w)[4], unsigned (&out)[4]) {
    const unsigned t0 = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), t1 = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u);
    const unsigned u0 = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u), u1 = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
    out[0] = __builtin_amdgcn_perm(u0, t0, 0x05040100u);
    out[1] = __builtin_amdgcn_perm(u0, t0, 0x07060302u);
    out[2] = __builtin_amdgcn_perm(u1, t1, 0x05040100u);
    out[3] = __builtin_amdgcn_perm(u1, t1, 0x07060302u);
}

// a sequence's length: from the device where there is one, within what the host said
__device__ __forceinline__ int pc_length(const int* dev, int b, int bound) { return dev ? min(max(dev[b], 0), bound) : bound; }

// the cache itself: pointers, sizes, offsets of `batch` sequences
inline int pc_check(const ps_cache* c, int batch) {
    if (!c || !c->k_codes || !c->v_codes || !c->k_scale || !c->v_scale || !c->kv_offsets) return PS_ERR_NULL;
    if (batch < 1 || c->n_kv_heads < 1 || c->head_dim < 1) return PS_ERR_SHAPE;
    if (c->head_dim != 64 && c->head_dim != 128) return PS_ERR_UNSUPPORTED;
    if (batch > PC_SEQS || c->n_kv_heads > 1024) return PS_ERR_UNSUPPORTED;
    for (int b = 0; b <= batch; ++b) {
        const int64_t o = c->kv_offsets[b];
        if (o < 0 || o % PC_BLOCK != 0 || (b > 0 && o < c->kv_offsets[b - 1])) return PS_ERR_OFFSETS;
        if (o >= 1LL << 36) return PS_ERR_UNSUPPORTED;
    }
    if ((((uintptr_t)c->k_codes | (uintptr_t)c->v_codes) & 15) || (((uintptr_t)c->k_scale | (uintptr_t)c->v_scale) & 3)) return PS_ERR_UNSUPPORTED;
    return PS_OK;
}
inline bool aligned4(const void* p) { return ((uintptr_t)p & 3) == 0; }
// bytes between rows of `row` elements: stride, or no gap; 0 if it cannot be taken
inline int pc_stride(int64_t stride, int64_t row, int dtype, int64_t* bytes) {
    if (stride == 0) stride = row;
    if (stride < row) return PS_ERR_SHAPE;
    if (stride > 1LL << 32 || (dtype == PS_BF16 && (stride & 1))) return PS_ERR_UNSUPPORTED;
    *bytes = stride * (dtype == PS_BF16 ? 2 : 4);
    return PS_OK;
}

}   // namespace

// What the kernels of group-wise parallel training share (ps_train.hip: attention; ps_train_grad.hip: its backward pass; ps_embed.hip;
// ps_loss.hip): accesses to rows that are aligned to 4 bytes only, rotary angles, bf16 high and low parts.
#pragma once
#include <algorithm>

#include "ps_device.h"
#include "ps_train.h"

namespace {

// Wide accesses to the caller's q, k, v and out, which are only promised to be aligned to 4 bytes: the types say so, and the
// compiler emits the same 16-byte instructions (global memory takes them at any multiple of 4).
typedef unsigned u32x4_q __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned u32x2_q __attribute__((ext_vector_type(2), aligned(4)));
typedef float f32x4_q __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ uint4 ld16_q(const void* p) { return __builtin_bit_cast(uint4, (u32x4)*reinterpret_cast<const u32x4_q*>(p)); }
__device__ __forceinline__ uint4 ldg_stream16_q(const void* p) {
    return __builtin_bit_cast(uint4, (u32x4)__builtin_nontemporal_load(reinterpret_cast<const u32x4_q*>(p)));
}
template <typename WT> __device__ __forceinline__ f32x4 load4_q(const void* p) {
    if constexpr (Traits<WT>::BF) {
        const u32x2 v = *reinterpret_cast<const u32x2_q*>(p);
        return f32x4{bf16_to_f32(v[0] & 0xFFFFu), bf16_to_f32(v[0] >> 16), bf16_to_f32(v[1] & 0xFFFFu), bf16_to_f32(v[1] >> 16)};
    } else {
        return *reinterpret_cast<const f32x4_q*>(p);
    }
}
__device__ __forceinline__ void stg_stream16_q(float* p, f32x4 v) { __builtin_nontemporal_store((f32x4_q)v, reinterpret_cast<f32x4_q*>(p)); }

// Division of numbers below 2^31 by one that the host knows: n / d = (n * mul) >> shift
struct GaDiv {
    unsigned mul, shift;
    __device__ __forceinline__ unsigned operator()(unsigned n) const { return (unsigned)((u64)n * mul >> shift); }
};
inline GaDiv ga_div(unsigned d) {
    unsigned s = 0;
    while ((1ull << s) < d) ++s;
    return GaDiv{(unsigned)(((1ull << (31 + s)) + d - 1) / d), 31 + s};   // (mul * d exceeds 2^(31 + s) by less than d <= 2^s)
}

// 2^x: Taylor's series of e^(f ln 2), |f| <= 1/2, to the 13th power (the next is 4e-18)
__device__ __forceinline__ double ga_exp2(double x) {
    const double n = rint(x), y = (x - n) * 0.69314718055994530942;
    double p = 1.0 / 6227020800.0;
    constexpr double c[13] = {1.0, 1.0, 1.0 / 2, 1.0 / 6, 1.0 / 24, 1.0 / 120, 1.0 / 720, 1.0 / 5040, 1.0 / 40320, 1.0 / 362880,
                              1.0 / 3628800, 1.0 / 39916800, 1.0 / 479001600};
#pragma unroll
    for (int i = 12; i >= 0; --i) p = fma(p, y, c[i]);
    return ldexp(p, (int)n);
}
// cosine and sine of a >= 0: the multiple of pi / 2 taken off in two parts (Cody and Waite's reduction; the first product is exact inside its fma, the second
// part is below 1e-9), Taylor's series on [-pi / 4, pi / 4] to r^16 and r^17 (what follows is below 2e-18).  Angles beyond
// 2^22 (a base below 1) are the library's business
__device__ __forceinline__ float2 ga_cos_sin(double a) {
    if (!(a <= 4194304.0)) return make_float2((float)cos(a), (float)sin(a));
    const double n = rint(a * 0.63661977236758134308);
    const double r = fma(-n, 6.123233995736766036e-17, fma(-n, 1.5707963267948965580, a)), z = r * r;
    constexpr double cc[9] = {1.0, -1.0 / 2, 1.0 / 24, -1.0 / 720, 1.0 / 40320, -1.0 / 3628800, 1.0 / 479001600, -1.0 / 87178291200.0, 1.0 / 20922789888000.0};
    constexpr double sc[9] = {1.0, -1.0 / 6, 1.0 / 120, -1.0 / 5040, 1.0 / 362880, -1.0 / 39916800, 1.0 / 6227020800.0, -1.0 / 1307674368000.0, 1.0 / 355687428096000.0};
    double c = cc[8], s = sc[8];
#pragma unroll
    for (int i = 7; i >= 0; --i) {
        c = fma(c, z, cc[i]);
        s = fma(s, z, sc[i]);
    }
    const float fc = (float)c, fs = (float)(s * r);
    const int q = (int)n;                                   // quarter turns
    const float x = q & 1 ? fs : fc, y = q & 1 ? fc : fs;
    return make_float2((q + 1) & 2 ? -x : x, q & 2 ? -y : y);
}

// the largest of z, |a|, |b|, or NaN if there is one
__device__ __forceinline__ float abs_max3(float z, float a, float b) {
    return __builtin_elementwise_maximum(__builtin_elementwise_maximum(z, __builtin_fabsf(a)), __builtin_fabsf(b));
}

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

__device__ __forceinline__ bf16x8 split_hi(const float (&v)[8], unsigned (&hi)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) hi[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
    return __builtin_bit_cast(bf16x8, make_uint4(hi[0], hi[1], hi[2], hi[3]));
}
__device__ __forceinline__ bf16x8 split_lo(const float (&v)[8], const unsigned (&hi)[4]) {
    unsigned lo[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        lo[i] = pack_bf16x2(v[2 * i] - __uint_as_float(hi[i] << 16), v[2 * i + 1] - __uint_as_float(hi[i] & 0xFFFF0000u));
    return __builtin_bit_cast(bf16x8, make_uint4(lo[0], lo[1], lo[2], lo[3]));
}

constexpr long long GA_MAX_WG = 0x7FFFFFFF;                // the attention's kernels number their workgroups in 31 bits (the float32 ones in 32)
constexpr int GF_ROWS = 64;

// the arguments of the attention and of its backward pass, but for the pointers
inline int ga_check(const ps_group_attn_args* a) {
    if (!a) return PS_ERR_NULL;
    if (a->seqs < 1 || a->tokens < 1 || a->k < 0 || a->n_heads < 1 || a->n_kv_heads < 1 || a->head_dim < 1) return PS_ERR_SHAPE;
    if (a->dtype != PS_F32 && a->dtype != PS_BF16) return PS_ERR_SHAPE;
    if (a->n_heads % a->n_kv_heads != 0 || !(a->rope_base > 0.f)) return PS_ERR_SHAPE;
    if (a->head_dim != 64 && a->head_dim != 128) return PS_ERR_UNSUPPORTED;
    if (a->k > 15 || (long long)a->tokens + a->k > (1 << 20)) return PS_ERR_UNSUPPORTED;
    if (a->n_heads > 65535 || a->seqs > 65535) return PS_ERR_UNSUPPORTED;
    if ((long long)(a->k + 1) * a->n_kv_heads * a->head_dim * 4 > (1LL << 27)) return PS_ERR_UNSUPPORTED;   // 32-bit offsets inside a key tile
    if (a->dtype == PS_F32 && ((long long)a->tokens * (a->k + 1) + GF_ROWS - 1) / GF_ROWS * a->n_heads > GA_MAX_WG) return PS_ERR_UNSUPPORTED;   // (its rows would be terabytes)
    return PS_OK;
}

inline size_t a256(size_t v) { return (v + 255) & ~(size_t)255; }

}   // namespace

// The target's distributions from its logits, and draws from them (see include/ps_verify.h).
//
//   e_i = 2^y_i,  y_i = (logits_i - max) log2(e) / temperature;  kept = {i : c_i <= bound, e_i >= min_p},  probs_i = e_i / sum of kept e
//
// c_i = (logit, descending; id, ascending) as one whole number puts the tokens in the order in which top-k and top-p take them, so what
// either keeps is everything up to one bound.  The bound is found without sorting the vocabulary: a histogram of y in steps of 1/32 (counts for
// top-k, sums of e for top-p) says which step the bound lies in, and the few tokens of that step are ordered in LDS; where
// there are many of them (equal logits), c is found eight bits at a time.  e is a whole number of 2^-F (F = 62 - log2 V, at most 52), from a double: sums
// are exact in any order, whoever adds them, and their error is far below what decides a draw.
//
// One workgroup of 1024 threads per row; the row stays in registers between the passes as far as it fits.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ps_cache_device.h"

namespace {

constexpr int TP_THREADS = 1024, TP_WAVES = TP_THREADS / 64;
constexpr int TP_BINS = 2048, TP_PER_POWER = 32;   // steps of y: 64 powers of two, what is below has no mass in F <= 52 bits
constexpr int TP_SHORT = 64;                       // a step with more tokens is cut into as many parts again
constexpr int TP_LIST = 2048;                      // tokens of one step that are ordered in LDS
constexpr int TP_MAX_LOG = 20;                     // vocab <= 2^20: an id takes 20 bits of c
constexpr int TP_MAX_CELLS = 4096;                 // wavefronts' shares of a row: 2^20 / (64 * 4)

struct TpParams {
    const char* logits;
    const float* temperature;
    const int* top_k;
    const float *top_p, *min_p, *r;
    float* probs;
    int* ids;
    float* id_probs;
    int rows, vocab, frac;                         // F
};

typedef unsigned u32x4_h __attribute__((ext_vector_type(4), aligned(2)));

template <typename LT> struct Vec;                 // 16 bytes of logits
template <> struct Vec<float> {
    static constexpr int N = 4;
    static __device__ __forceinline__ float get(const u32x4& v, int e) { return __uint_as_float(v[e]); }
};
template <> struct Vec<bf16_t> {
    static constexpr int N = 8;
    static __device__ __forceinline__ float get(const u32x4& v, int e) { return __uint_as_float(e & 1 ? v[e >> 1] & 0xFFFF0000u : v[e >> 1] << 16); }
};

// logits 16 bytes at a time; what is behind the row's end is -Inf
template <typename LT> __device__ __forceinline__ u32x4 load_vec(const char* row, int i, int vocab) {
    constexpr int N = Vec<LT>::N;
    const char* p = row + (size_t)i * 16;
    if ((i + 1) * N <= vocab) return *reinterpret_cast<const u32x4_h*>(p);
    u32x4 v = Traits<LT>::BF ? u32x4{0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u} : u32x4{0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u};
#pragma unroll
    for (int e = 0; e < N; ++e)
        if (i * N + e < vocab) {
            if constexpr (Traits<LT>::BF) {
                const unsigned x = reinterpret_cast<const uint16_t*>(p)[e];
                v[e >> 1] = e & 1 ? (v[e >> 1] & 0xFFFFu) | x << 16 : (v[e >> 1] & 0xFFFF0000u) | x;
            } else v[e] = reinterpret_cast<const unsigned*>(p)[e];
        }
    return v;
}

// 2^f, |f| <= 1/2: Taylor's series of e^(f ln 2) to the 10th power (the next is 2e-13)
__device__ __forceinline__ double exp2_part(double f) {
    const double y = f * 0.69314718055994530942;
    constexpr double c[11] = {1.0, 1.0, 1.0 / 2, 1.0 / 6, 1.0 / 24, 1.0 / 120, 1.0 / 720, 1.0 / 5040, 1.0 / 40320, 1.0 / 362880, 1.0 / 3628800};
    double p = c[10];
#pragma unroll
    for (int i = 9; i >= 0; --i) p = fma(p, y, c[i]);
    return p;
}

struct Row {
    double max, c;                                 // the largest logit, log2(e) / temperature
    double min_p;
    int frac;
    __device__ __forceinline__ double y(float l) const { return ((double)l - max) * c; }   // (NaN for -Inf at an infinite temperature)
    __device__ __forceinline__ double e(float l) const {
        const double v = y(l), n = rint(v);
        return v > -1000.0 && l > -__builtin_inff() ? ldexp(exp2_part(v - n), (int)n) : 0.0;
    }
    // e as a whole number of 2^-frac; 0 below that, and for what min_p cuts
    __device__ __forceinline__ u64 mass(float l) const {
        const double v = y(l);
        if (!(v > -64.0) || l == -__builtin_inff()) return 0;
        const double n = rint(v), p = exp2_part(v - n);
        if (min_p > 0.0 && ldexp(p, (int)n) < min_p) return 0;
        return (u64)(ldexp(p, (int)n + frac) + 0.5);
    }
    // how many steps of y below the largest, at most the last one
    __device__ __forceinline__ double steps(float l) const {
        const double v = y(l) * -TP_PER_POWER;
        return v < TP_BINS - 1 && l > -__builtin_inff() ? v : TP_BINS - 1;
    }
};
// the token's place: descending logit (0 and -0 are equal), ascending id
__device__ __forceinline__ u64 place(float l, int id) {
    const unsigned u = __float_as_uint(l + 0.f);
    const unsigned key = u >> 31 ? u : ~u & 0x7FFFFFFFu;
    return (u64)key << TP_MAX_LOG | (unsigned)id;
}

struct Shared {
    union {
        struct { u64 mass[TP_BINS]; unsigned count[TP_BINS]; } h;
        u64 cell[TP_MAX_CELLS];
    };
    u64 list[TP_LIST], list_mass[TP_LIST];
    u64 red[TP_WAVES + 1];
    u64 found_before, found_total;
    u64 bound;
    unsigned red32[TP_WAVES];
    int found, n_list, bad;
};

__device__ __forceinline__ u64 shfl_up64(u64 v, int d) {
    return (u64)__shfl_up((unsigned)(v >> 32), d) << 32 | __shfl_up((unsigned)v, d);
}
__device__ __forceinline__ u64 wave_scan_u64(u64 v) {       // inclusive
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const u64 o = shfl_up64(v, d);
        if ((int)(threadIdx.x & 63) >= d) v += o;
    }
    return v;
}
__device__ __forceinline__ u64 lane63_u64(u64 v) {
    return (u64)(unsigned)__builtin_amdgcn_readlane((unsigned)(v >> 32), 63) << 32 | (unsigned)__builtin_amdgcn_readlane((unsigned)v, 63);
}
// inclusive scan over the threads; total to every thread.  Synchronises before and after
__device__ __forceinline__ u64 block_scan_u64(u64 v, Shared& S, u64& total) {
    const int wave = threadIdx.x >> 6;
    v = wave_scan_u64(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) S.red[wave] = v;
    __syncthreads();
    u64 base = 0;
    total = 0;
    for (int w = 0; w < TP_WAVES; ++w) {
        if (w < wave) base += S.red[w];
        total += S.red[w];
    }
    __syncthreads();
    return base + v;
}

template <typename LT, int RES> struct Logits {
    u32x4 v[RES];
    const char* row;
    int vocab, nvec;
    __device__ __forceinline__ void load() {
#pragma unroll
        for (int i = 0; i < RES; ++i) v[i] = load_vec<LT>(row, i * TP_THREADS + (int)threadIdx.x, vocab);
    }
    // f(vector, its number), by whole wavefronts: what is behind the row's end is -Inf
    template <typename F> __device__ __forceinline__ void each(F f) const {
#pragma unroll
        for (int i = 0; i < RES; ++i)
            if (i * TP_THREADS < nvec) f(v[i], i * TP_THREADS + (int)threadIdx.x);
        for (int i = RES * TP_THREADS; i < nvec; i += TP_THREADS) f(load_vec<LT>(row, i + (int)threadIdx.x, vocab), i + (int)threadIdx.x);
    }
    // f(logit, id) of the row's tokens
    template <typename F> __device__ __forceinline__ void tokens(F f) const {
        each([&](const u32x4& x, int at) {
#pragma unroll
            for (int e = 0; e < Vec<LT>::N; ++e)
                if (at * Vec<LT>::N + e < vocab) f(Vec<LT>::get(x, e), at * Vec<LT>::N + e);
        });
    }
};

// The place up to which tokens are kept, of those with places <= `within`: BY_MASS: the first with which the sum of e reaches top_p of their sum;
// else the top_k-th.  Every thread returns it.
template <bool BY_MASS, typename LT, int RES>
__device__ u64 find_bound(const Logits<LT, RES>& L, const Row& R, Shared& S, u64 within, u64 k, double top_p) {
    const int tid = threadIdx.x;
    auto weight = [&](float l) { return BY_MASS ? R.mass(l) : (u64)1; };
    u64 before = 0, want = k;                               // the sum over the steps in front; the sum to be reached
    int step[2] = {0, 0}, levels = 0;                       // the step, and the part of it (2048 of them), that the bound lies in
    auto inside = [&](float l, int id) {
        if (within != ~0ull && place(l, id) > within) return false;
        if (levels == 0) return true;
        const double v = R.steps(l);
        if ((int)v != step[0]) return false;
        return levels == 1 || (int)((v - step[0]) * TP_BINS) == step[1];
    };
    unsigned in_step;
    do {
        for (int i = tid; i < TP_BINS; i += TP_THREADS) { S.h.mass[i] = 0; S.h.count[i] = 0; }
        __syncthreads();
        L.tokens([&](float l, int id) {
            if (!inside(l, id)) return;
            const double v = R.steps(l);
            const int bin = levels == 0 ? (int)v : (int)((v - step[0]) * TP_BINS);
            __hip_atomic_fetch_add(&S.h.count[bin], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
            if constexpr (BY_MASS) {
                const u64 m = R.mass(l);
                if (m) __hip_atomic_fetch_add(&S.h.mass[bin], m, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
            }
        });
        __syncthreads();
        constexpr int PER = TP_BINS / TP_THREADS;
        u64 own[PER], sum = 0, total;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            own[i] = BY_MASS ? S.h.mass[tid * PER + i] : S.h.count[tid * PER + i];
            sum += own[i];
        }
        u64 upto = block_scan_u64(sum, S, total) - sum + before;
        if (BY_MASS && levels == 0) {
            const double t = ceil(top_p * (double)total);
            want = t >= 1.0 ? min((u64)t, total) : 1;
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (upto < want && upto + own[i] >= want) { S.found = tid * PER + i; S.found_before = upto; S.n_list = 0; }
            upto += own[i];
        }
        __syncthreads();
        step[levels++] = S.found;
        before = S.found_before;
        in_step = S.h.count[S.found];
        __syncthreads();
    } while (levels < 2 && in_step > TP_SHORT && step[0] < TP_BINS - 1);   // (the last step has no end)
    if (in_step <= TP_LIST) {
        L.tokens([&](float l, int id) {
            if (!inside(l, id)) return;
            const int at = __hip_atomic_fetch_add(&S.n_list, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
            S.list[at] = place(l, id);
            S.list_mass[at] = weight(l);
        });
        __syncthreads();
        // the bound: the token with which the sum reaches `want` (in any order of the list: whole numbers)
        const int n = S.n_list;
        for (int i = tid; i < n; i += TP_THREADS) {
            const u64 c = S.list[i];
            u64 less = before;
            for (int j = 0; j < n; ++j) less += S.list[j] < c ? S.list_mass[j] : 0;
            if (less < want && less + S.list_mass[i] >= want) S.bound = c;
        }
        __syncthreads();
        const u64 bound = S.bound;
        __syncthreads();
        return bound;
    }
    // many equal or nearly equal logits: the place's 52 bits, four of them and then eight at a time
    u64 prefix = 0;
    for (int shift = 48; shift >= 0; shift -= 8) {
        const int bits = shift == 48 ? 4 : 8;
        if (tid < 256) S.h.mass[tid] = 0;
        __syncthreads();
        L.tokens([&](float l, int id) {
            if (!inside(l, id)) return;
            const u64 c = place(l, id);
            if (c >> (shift + bits) != prefix) return;
            const u64 m = weight(l);
            if (m) __hip_atomic_fetch_add(&S.h.mass[(unsigned)(c >> shift) & ((1u << bits) - 1)], m, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        });
        __syncthreads();
        u64 total;
        const u64 w = tid < 1 << bits ? S.h.mass[tid] : 0;
        const u64 to = before + block_scan_u64(w, S, total);
        if (to - w < want && to >= want) { S.found = tid; S.found_before = to - w; }
        __syncthreads();
        prefix = prefix << bits | (unsigned)S.found;
        before = S.found_before;
        __syncthreads();
    }
    return prefix;
}

template <typename LT, int RES>
__global__ __launch_bounds__(TP_THREADS) void target_probs_kernel(const TpParams P) {
    constexpr int N = Vec<LT>::N;
    __shared__ Shared S;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = P.vocab;
    const size_t row = blockIdx.x;
    const int b = (int)(row / (unsigned)P.rows);
    Logits<LT, RES> L;
    L.row = P.logits + row * V * Traits<LT>::ESZ; L.vocab = V; L.nvec = (V + N - 1) / N;
    L.load();
    const float t_in = P.temperature ? P.temperature[b] : 1.f;
    const bool greedy = !(t_in > 0.f);
    const int k_in = P.top_k ? P.top_k[b] : 0;
    const int k = greedy ? 1 : k_in < 1 || k_in > V ? V : k_in;
    const float p_in = P.top_p ? P.top_p[b] : 1.f, min_p = P.min_p ? P.min_p[b] : 0.f;

    // the largest logit, and whether any is NaN or +Inf
    float mx = -__builtin_inff();
    bool bad = false;
    L.each([&](const u32x4& x, int) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float l = Vec<LT>::get(x, e);
            bad |= !(l < __builtin_inff());
            mx = fmaxf(mx, l);
        }
    });
    mx = __ballot(bad) ? __builtin_nanf("") : wave_max(mx);
    if (lane == 0) S.red32[wave] = __float_as_uint(mx);
    __syncthreads();
    mx = -__builtin_inff();
    bad = false;
    for (int w = 0; w < TP_WAVES; ++w) {
        const float m = __uint_as_float(S.red32[w]);
        bad |= m != m;
        mx = fmaxf(mx, m);
    }
    float* out = P.probs ? P.probs + row * V : nullptr;
    if (bad || mx == -__builtin_inff()) {
        const float fill = bad ? __builtin_nanf("") : 0.f;
        if (out) for (int i = tid; i < V; i += TP_THREADS) out[i] = fill;
        if (P.ids && tid == 0) {
            P.ids[row] = -1;
            if (P.id_probs) P.id_probs[row] = fill;
        }
        return;
    }
    Row R;
    R.max = mx; R.c = 1.4426950408889634074 / (greedy ? 1.0 : (double)t_in); R.frac = P.frac; R.min_p = 0.0;
    u64 bound = ~0ull;
    if (k == 1) {                                           // the first of the largest
        unsigned id = ~0u;
        L.tokens([&](float l, int i) { if (l == mx) id = min(id, (unsigned)i); });
        id = ~wave_max_u32(~id);
        __syncthreads();
        if (lane == 0) S.red32[wave] = id;
        __syncthreads();
        for (int w = 0; w < TP_WAVES; ++w) id = min(id, S.red32[w]);
        bound = place(mx, (int)id);
    } else {
        if (k < V) bound = find_bound<false>(L, R, S, bound, (u64)k, 0.0);
        if (p_in < 1.f) bound = find_bound<true>(L, R, S, bound, 0, (double)p_in);
    }
    R.min_p = min_p > 0.f ? (double)fminf(min_p, 1.f) : 0.0;

    // the sum of the kept e, by the wavefronts' shares in id order
    __syncthreads();
    L.each([&](const u32x4& x, int at) {
        u64 m = 0;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float l = Vec<LT>::get(x, e);
            if (at * N + e < V && place(l, at * N + e) <= bound) m += R.mass(l);
        }
        m = lane63_u64(wave_scan_u64(m));
        if (lane == 0) S.cell[at / 64] = m;
    });
    __syncthreads();
    constexpr int PER = TP_MAX_CELLS / TP_THREADS;
    const int cells = (L.nvec + TP_THREADS - 1) / TP_THREADS * TP_WAVES;
    u64 own[PER], sum = 0, total;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        own[i] = tid * PER + i < cells ? S.cell[tid * PER + i] : 0;
        sum += own[i];
    }
    u64 upto = block_scan_u64(sum, S, total) - sum;
    const double whole = ldexp((double)total, -P.frac);     // the sum of the kept e
    if (P.ids) {
        const double t = (double)P.r[row] * (double)total;
        const u64 want = t >= 1.0 ? min((u64)t, total - 1) : 0;   // the drawn token is the first with which the sum passes it
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (upto <= want && upto + own[i] > want) { S.found = tid * PER + i; S.found_before = upto; }
            upto += own[i];
        }
        __syncthreads();
        if (wave == 0) {
            const int at = S.found * 64 + lane;
            const u32x4 x = load_vec<LT>(L.row, at, V);
            u64 m[N], all = 0;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float l = Vec<LT>::get(x, e);
                m[e] = at * N + e < V && place(l, at * N + e) <= bound ? R.mass(l) : 0;
                all += m[e];
            }
            u64 to = S.found_before + wave_scan_u64(all) - all;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                if (to <= want && to + m[e] > want) {
                    P.ids[row] = at * N + e;
                    if (P.id_probs) P.id_probs[row] = (float)(R.e(Vec<LT>::get(x, e)) / whole);
                }
                to += m[e];
            }
        }
    }
    if (!out) return;
    const float inv = (float)(1.0 / whole);
    L.each([&](const u32x4& x, int at) {
        float p[N];
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float l = Vec<LT>::get(x, e);
            p[e] = 0.f;
            if (l > -__builtin_inff() && place(l, at * N + e) <= bound && (R.min_p == 0.0 || R.mass(l))) {
                const double y = R.y(l), n = rint(y);
                p[e] = ldexpf(__builtin_amdgcn_exp2f((float)(y - n)) * inv, (int)n);
            }
        }
#pragma unroll
        for (int q = 0; q < N; q += 4) {
            if (at * N + q + 4 <= V) *reinterpret_cast<f32x4_q*>(out + (size_t)at * N + q) = f32x4{p[q], p[q + 1], p[q + 2], p[q + 3]};
            else
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (at * N + q + e < V) out[(size_t)at * N + q + e] = p[q + e];
        }
    });
}

template <typename LT> void go(const TpParams& P, int total, hipStream_t s) {
    constexpr int N = Vec<LT>::N;
    if (P.vocab <= 4 * TP_THREADS * N) hipLaunchKernelGGL((target_probs_kernel<LT, 4>), dim3(total), dim3(TP_THREADS), 0, s, P);
    else hipLaunchKernelGGL((target_probs_kernel<LT, 16>), dim3(total), dim3(TP_THREADS), 0, s, P);
}

int check(const ps_target_probs_args* a) {
    if (!a) return PS_ERR_NULL;
    if (a->batch < 1 || a->rows < 1 || a->vocab < 1) return PS_ERR_SHAPE;
    if (a->dtype != PS_F32 && a->dtype != PS_BF16) return PS_ERR_SHAPE;
    if (a->vocab > 1 << TP_MAX_LOG || (long long)a->batch * a->rows > 1 << 20) return PS_ERR_UNSUPPORTED;
    return PS_OK;
}

}   // namespace

extern "C" size_t ps_target_probs_workspace_bytes(const ps_target_probs_args* a) {
    return check(a) == PS_OK ? 0 : 0;
}

extern "C" int ps_target_probs(const ps_target_probs_args* a, void* stream) {
    const int st = check(a);
    if (st != PS_OK) return st;
    if (!a->logits || (!a->probs && !a->ids) || (a->ids && !a->r) || (a->id_probs && !a->ids)) return PS_ERR_NULL;
    if ((uintptr_t)a->logits & (a->dtype == PS_BF16 ? 1 : 3)) return PS_ERR_UNSUPPORTED;
    if (!aligned4(a->temperature) || !aligned4(a->top_k) || !aligned4(a->top_p) || !aligned4(a->min_p) || !aligned4(a->r) || !aligned4(a->probs) ||
        !aligned4(a->ids) || !aligned4(a->id_probs)) return PS_ERR_UNSUPPORTED;
    TpParams P = {};
    P.logits = (const char*)a->logits; P.temperature = a->temperature; P.top_k = a->top_k; P.top_p = a->top_p; P.min_p = a->min_p; P.r = a->r;
    P.probs = a->probs; P.ids = a->ids; P.id_probs = a->id_probs; P.rows = a->rows; P.vocab = a->vocab;
    int log = 0;
    while (1 << log < a->vocab) ++log;
    P.frac = std::min(52, 62 - log);
    const int total = a->batch * a->rows;
    if (a->dtype == PS_BF16) go<bf16_t>(P, total, (hipStream_t)stream);
    else go<float>(P, total, (hipStream_t)stream);
    return hipGetLastError() == hipSuccess ? PS_OK : PS_ERR_DEVICE;
}

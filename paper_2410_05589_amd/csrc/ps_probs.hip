// The target's distributions from its logits, and draws from them (see include/ps_verify.h).
//
//   e_i = 2^y_i,  y_i = (logits_i - max) log2(e) / temperature;  kept = {i : c_i <= bound, e_i >= min_p},  probs_i = e_i / sum of kept e
//
// c_i = (logit, descending; id, ascending) as one whole number puts the tokens in the order in which top-k and top-p take them, so what
// either keeps is everything up to one token, the bound, and min_p is a bound too.  Nothing is sorted:
//   top-k, small k   the k-th largest of the threads' own maxima is a lower limit; the few tokens above it are listed in LDS
//   top-p, large k   a histogram of y in steps of 1/32 (sums of e, or counts) says which step the bound lies in; that step's tokens are listed
//   the list         ordered by c eleven bits at a time, from the highest bit in which its tokens differ
// e is a whole number of 2^-F (F = 62 - log2 V, at most 51), from a double: sums are exact in any order, whoever adds them, and
// their error is far below what decides a draw.
//
// One workgroup of 1024 threads per row, two of them on a compute unit; the row is read again by each pass, from the caches.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ps_cache_device.h"

namespace {

constexpr int TP_THREADS = 1024, TP_WAVES = TP_THREADS / 64;
constexpr int TP_BINS = 2048;                      // steps of 1/32 in y: 64 powers of two, what is below has no mass in F <= 51 bits
constexpr int TP_LIST = 2 * TP_THREADS;            // tokens that are ordered in LDS
constexpr int TP_SMALL_K = 512;                    // top-k by the threads' maxima
constexpr int TP_MAX_LOG = 20;                     // vocab <= 2^20: an id takes 20 bits of c
constexpr int TP_MAX_CELLS = 4096;                 // wavefronts' shares of a row: 2^20 / (64 * 4)
constexpr int TP_TABLE = 64;                       // 2^(j/64)

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

// The place up to which tokens are kept
struct Bound {
    float l;
    unsigned id;
    __device__ __forceinline__ bool keeps(float x, unsigned i) const { return x > l || (x == l && i <= id); }
};

// the token's place: descending logit (0 and -0 are equal), ascending id
__device__ __forceinline__ u64 place(float l, int id) {
    const unsigned u = __float_as_uint(l + 0.f);
    const unsigned key = u >> 31 ? u : ~u & 0x7FFFFFFFu;
    return (u64)key << TP_MAX_LOG | (unsigned)id;
}
__device__ __forceinline__ Bound bound_of(u64 c) {
    const unsigned key = (unsigned)(c >> TP_MAX_LOG);
    return {__uint_as_float(key >> 31 ? key : ~key & 0x7FFFFFFFu), (unsigned)c & ((1u << TP_MAX_LOG) - 1)};
}

__device__ __forceinline__ float uniform(float v) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v))); }
__device__ __forceinline__ double uniform(double v) {
    return __hiloint2double(__builtin_amdgcn_readfirstlane(__double2hiint(v)), __builtin_amdgcn_readfirstlane(__double2loint(v)));
}

struct Shared {
    double table[TP_TABLE];
    union {
        struct { u64 mass[TP_BINS]; unsigned count[TP_BINS]; } h;
        u64 cell[TP_MAX_CELLS];
    };
    u64 list[TP_LIST];
    u64 red[TP_WAVES], red2[TP_WAVES];
    u64 found_before;
    unsigned red32[TP_WAVES];
    int found, n_list;
};

struct Row {
    double max, c;                                 // the largest logit, 64 log2(e) / temperature
    int frac;
    const double* table;
    // e = 2^(k / 64) * (1 + ...): k = rint(64 y), the rest by Taylor's series to the 4th power (the next is 4e-14).  Below 2^-80, and for -Inf: 2^-80
    __device__ __forceinline__ double part(float l, int& k) const {
        constexpr double big = 6755399441055744.0, q = 0.69314718055994530942 / TP_TABLE;   // 1.5 * 2^52: the sum's low word is the rounded number
        const double u = __builtin_fmax(((double)l - max) * c, -80.0 * TP_TABLE), t = u + big, r = u - (t - big);
        k = __double2loint(t);
        double p = fma(r, q * q * q * q / 24, q * q * q / 6);
        p = fma(p, r, q * q / 2);
        p = fma(p, r, q);
        p = fma(p, r, 1.0);
        return p * table[k & (TP_TABLE - 1)];
    }
    __device__ __forceinline__ double e(float l) const {
        int k;
        const double p = part(l, k);
        return ldexp(p, k >> 6);
    }
    // e as a whole number of 2^-frac, below 2^52
    __device__ __forceinline__ u64 mass(float l, int& k) const {
        const double p = part(l, k), x = ldexp(p, (k >> 6) + frac) + 4503599627370496.0;
        return (u64)(unsigned)(__double2hiint(x) - 0x43300000) << 32 | (unsigned)__double2loint(x);
    }
    __device__ __forceinline__ u64 mass(float l) const { int k; return mass(l, k); }
    __device__ __forceinline__ int step(float l) const {
        constexpr double big = 6755399441055744.0;
        const double u = __builtin_fmax(((double)l - max) * c, -80.0 * TP_TABLE);
        return step_of(__double2loint(u + big));
    }
    static __device__ __forceinline__ int step_of(int k) { return min(-k >> 1, TP_BINS - 1); }
};

__device__ __forceinline__ u64 shfl_up64(u64 v, int d) {
    return (u64)__shfl_up((unsigned)(v >> 32), d) << 32 | __shfl_up((unsigned)v, d);
}
__device__ __forceinline__ u64 shfl_xor64(u64 v, int d) {
    return (u64)__shfl_xor((unsigned)(v >> 32), d) << 32 | __shfl_xor((unsigned)v, d);
}
__device__ __forceinline__ u64 wave_scan_u64(u64 v) {       // inclusive
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const u64 o = shfl_up64(v, d);
        if ((int)(threadIdx.x & 63) >= d) v += o;
    }
    return v;
}
// lane 0 has the sum
__device__ __forceinline__ u64 wave_sum_u64(u64 v) {
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) v += shfl_xor64(v, d);
    return v;
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

template <typename LT> struct Logits {
    const char* row;
    int vocab, nvec;
    // f(vector, its number), by whole wavefronts: what is behind the row's end is -Inf
    template <typename F> __device__ __forceinline__ void each(F f) const {
        u32x4 x = load_vec<LT>(row, (int)threadIdx.x, vocab), next = load_vec<LT>(row, TP_THREADS + (int)threadIdx.x, vocab);
        for (int i = 0; i < nvec; i += TP_THREADS) {        // two vectors ahead
            const u32x4 after = load_vec<LT>(row, i + 2 * TP_THREADS + (int)threadIdx.x, vocab);
            f(x, i + (int)threadIdx.x);
            x = next;
            next = after;
        }
    }
    // f(logit, id) of the row's tokens
    template <typename F> __device__ __forceinline__ void tokens(F f) const {
        each([&](const u32x4& x, int at) {
#pragma unroll
            for (int e = 0; e < Vec<LT>::N; ++e) {
                if (at * Vec<LT>::N + e < vocab) f(Vec<LT>::get(x, e), at * Vec<LT>::N + e);
                if (e & 1) __builtin_amdgcn_sched_barrier(0);   // (two at a time: registers)
            }
        });
    }
};

__device__ __forceinline__ void list_add(Shared& S, u64 c) {
    const int at = __hip_atomic_fetch_add(&S.n_list, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    if (at < TP_LIST) S.list[at] = c;
}

// The histogram's first entry with which the sum, `before` in front of it, reaches `want`; S.found, S.found_before to every thread
__device__ __forceinline__ u64 find_in_bins(Shared& S, u64 before, u64 want, double of_all) {
    constexpr int PER = TP_BINS / TP_THREADS;
    u64 own[PER], sum = 0, total;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        own[i] = S.h.mass[threadIdx.x * PER + i];
        sum += own[i];
    }
    u64 upto = block_scan_u64(sum, S, total) - sum + before;
    if (of_all >= 0.0) {                                    // (a share of the whole)
        const double t = ceil(of_all * (double)total);
        want = t >= 1.0 ? min((u64)t, total) : 1;
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (upto < want && upto + own[i] >= want) { S.found = threadIdx.x * PER + i; S.found_before = upto; }
        upto += own[i];
    }
    __syncthreads();
    return want;
}

// Of the list's n tokens, with weights w(logit): the first, in the order of places, with which the sum (`before` in front of them) reaches `want`.
// of_all: as above.  Takes and leaves synchronised; S.found_before: the sum up to and with that token
template <typename W> __device__ __forceinline__ u64 find_in_list(Shared& S, int n, u64 before, u64 want, double of_all, W w) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    u64 c[2], m[2];
    bool live[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        live[i] = tid + i * TP_THREADS < n;
        c[i] = live[i] ? S.list[tid + i * TP_THREADS] : 0;
        m[i] = live[i] ? w(bound_of(c[i]).l) : 0;
    }
    for (int round = 0; round < 6; ++round) {               // (52 bits, eleven and more at a time)
        u64 all = ~0ull, any = 0;                           // bits that every one has, that one has at least
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (live[i]) { all &= c[i]; any |= c[i]; }
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) { all &= shfl_xor64(all, d); any |= shfl_xor64(any, d); }
        if (lane == 0) { S.red[wave] = all; S.red2[wave] = any; }
        for (int i = tid; i < TP_BINS; i += TP_THREADS) S.h.mass[i] = 0;
        __syncthreads();
        for (int i = 0; i < TP_WAVES; ++i) { all &= S.red[i]; any |= S.red2[i]; }
        const u64 differ = all ^ any;
        const int shift = differ ? max(0, 63 - __builtin_clzll(differ) - 10) : 0;
#pragma unroll
        for (int i = 0; i < 2; ++i)
            if (live[i] && m[i]) __hip_atomic_fetch_add(&S.h.mass[(c[i] >> shift) & (TP_BINS - 1)], m[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        __syncthreads();
        want = find_in_bins(S, before, want, of_all);
        of_all = -1.0;
        const int digit = S.found;
        before = S.found_before;
#pragma unroll
        for (int i = 0; i < 2; ++i) live[i] = live[i] && (int)((c[i] >> shift) & (TP_BINS - 1)) == digit;
        if (differ >> 11 == 0) {                            // these eleven bits were the last ones
            const u64 at = (any & ~(u64)(TP_BINS - 1)) | digit;
            if (tid == 0) S.found_before = before + S.h.mass[digit];
            __syncthreads();
            return at;
        }
        __syncthreads();
    }
    return 0;
}

// The bound of the row's tokens that `within` keeps: the first token with which the sum of e (BY_MASS) reaches top_p of their sum, or the
// top_k-th.  S.found_before: the sum up to and with it
template <bool BY_MASS, typename LT>
__device__ __forceinline__ u64 find_in_row(const Logits<LT>& L, const Row& R, Shared& S, Bound within, u64 want, double of_all) {
    const int tid = threadIdx.x;
    auto weight = [&](float l) { return BY_MASS ? R.mass(l) : (u64)1; };
    for (int i = tid; i < TP_BINS; i += TP_THREADS) S.h.mass[i] = 0;
    if (tid == 0) S.n_list = 0;
    __syncthreads();
    L.tokens([&](float l, int id) {
        if (!within.keeps(l, id)) return;
        if constexpr (BY_MASS) {
            int k;
            const u64 m = R.mass(l, k);
            __hip_atomic_fetch_add(&S.h.mass[R.step_of(k)], m, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        } else __hip_atomic_fetch_add((unsigned*)&S.h.mass[R.step(l)], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    });
    __syncthreads();
    want = find_in_bins(S, 0, want, of_all);
    const int step = S.found;
    u64 before = S.found_before;
    L.tokens([&](float l, int id) {
        if (R.step(l) == step && within.keeps(l, id)) list_add(S, place(l, id));
    });
    __syncthreads();
    if (S.n_list <= TP_LIST) return find_in_list(S, S.n_list, before, want, -1.0, weight);
    // more tokens than the list holds (equal or nearly equal logits): eleven bits of the place at a time, until few enough are left
    u64 prefix = 0;
    for (int shift = 44;; shift -= 11) {
        __syncthreads();
        for (int i = tid; i < TP_BINS; i += TP_THREADS) { S.h.mass[i] = 0; S.h.count[i] = 0; }
        if (tid == 0) S.n_list = 0;
        __syncthreads();
        L.tokens([&](float l, int id) {
            const u64 c = place(l, id);
            if (R.step(l) != step || !within.keeps(l, id) || c >> (shift + 11) != prefix) return;
            const int digit = (int)(c >> shift) & (TP_BINS - 1);
            __hip_atomic_fetch_add(&S.h.count[digit], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
            __hip_atomic_fetch_add(&S.h.mass[digit], weight(l), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
        });
        __syncthreads();
        find_in_bins(S, before, want, -1.0);
        prefix = prefix << 11 | (unsigned)S.found;
        before = S.found_before;
        if (S.h.count[S.found] > TP_LIST && shift > 0) continue;   // (at the last digit it is one token)
        L.tokens([&](float l, int id) {
            const u64 c = place(l, id);
            if (c >> shift == prefix && R.step(l) == step && within.keeps(l, id)) list_add(S, c);
        });
        __syncthreads();
        return find_in_list(S, S.n_list, before, want, -1.0, weight);
    }
}

template <typename LT>
__global__ __launch_bounds__(TP_THREADS, 4) void target_probs_kernel(const TpParams P) {
    constexpr int N = Vec<LT>::N;
    __shared__ Shared S;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = P.vocab;
    const size_t row = blockIdx.x;
    const int b = (int)(row / (unsigned)P.rows);
    Logits<LT> L;
    L.row = P.logits + row * V * Traits<LT>::ESZ; L.vocab = V; L.nvec = (V + N - 1) / N;
    const float t_in = P.temperature ? P.temperature[b] : 1.f;
    const bool greedy = !(t_in > 0.f);
    const int k_in = P.top_k ? P.top_k[b] : 0;
    const int k = greedy ? 1 : k_in < 1 || k_in > V ? V : k_in;
    const float p_in = P.top_p ? P.top_p[b] : 1.f, m_in = P.min_p ? P.min_p[b] : 0.f, min_p = m_in > 0.f ? fminf(m_in, 1.f) : 0.f;
    if (tid < TP_TABLE) S.table[tid] = ga_exp2(tid * (1.0 / TP_TABLE));

    // the largest logit, and whether any is NaN or +Inf; each thread's first of its largest
    float mx = -__builtin_inff();
    unsigned first = 0;
    bool bad = false;
    L.each([&](const u32x4& x, int at) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float l = Vec<LT>::get(x, e);
            bad |= !(l < __builtin_inff());
            if (l > mx) { mx = l; first = at * N + e; }
        }
    });
    const float mine = mx;
    mx = __ballot(bad) ? __builtin_nanf("") : wave_max(mx);
    if (lane == 0) S.red32[wave] = __float_as_uint(mx);
    if (tid == 0) S.n_list = 0;
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
    R.max = uniform(mx); R.c = uniform(1.4426950408889634074 * TP_TABLE / (greedy ? 1.0 : (double)t_in)); R.frac = P.frac; R.table = S.table;
    Bound bound = {-__builtin_inff(), ~0u};
    u64 total = 0;                                          // the sum of the kept e, where it is known
    auto mass = [&](float l) { return R.mass(l); };
    auto one = [](float) { return (u64)1; };
    if (k == 1) {                                           // the first of the largest
        unsigned id = mine == mx ? first : ~0u;
        id = ~wave_max_u32(~id);
        __syncthreads();
        if (lane == 0) S.red32[wave] = id;
        __syncthreads();
        for (int w = 0; w < TP_WAVES; ++w) id = min(id, S.red32[w]);
        bound = {mx, id};
        total = R.mass(mx);
    } else {
        bool listed = false, all = k == V;                  // all: no top-k, or one that only drops tokens at -Inf
        if (k <= TP_SMALL_K && k < L.nvec) {
            // every one of the k threads with the largest maxima has a token at or above the k-th of them: so have the k largest tokens
            S.list[tid] = place(mine, first);
            __syncthreads();
            const Bound least = bound_of(find_in_list(S, TP_THREADS, 0, (u64)k, -1.0, one));
            if (least.l == -__builtin_inff()) all = true;
            else {
                L.tokens([&](float l, int id) { if (least.keeps(l, id)) list_add(S, place(l, id)); });
                __syncthreads();
                listed = S.n_list <= TP_LIST;
            }
        }
        if (listed) {
            const int n = S.n_list;
            bound = bound_of(find_in_list(S, n, 0, (u64)k, -1.0, one));
            u64 m = 0;
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (tid + i * TP_THREADS < n) {             // tokens behind the bound leave the list: the last place, without mass
                    const Bound at = bound_of(S.list[tid + i * TP_THREADS]);
                    if (bound.keeps(at.l, at.id)) m += R.mass(at.l);
                    else S.list[tid + i * TP_THREADS] = place(-__builtin_inff(), at.id);
                }
            block_scan_u64(m, S, total);
            if (p_in < 1.f) {
                bound = bound_of(find_in_list(S, n, 0, 0, fmax((double)p_in, 0.0), mass));
                total = S.found_before;
            }
        } else {
            if (!all) bound = bound_of(find_in_row<false>(L, R, S, bound, (u64)k, -1.0));
            if (p_in < 1.f) {
                __syncthreads();
                bound = bound_of(find_in_row<true>(L, R, S, bound, 0, fmax((double)p_in, 0.0)));
                total = S.found_before;
            }
        }
    }
    if (min_p > 0.f && R.c > 0.0) {                         // the least logit with e >= min_p: near max + log2(min_p) / c, tried out
        const float near = (float)(R.max + log2((double)min_p) * TP_TABLE / R.c);
        const unsigned key = (unsigned)(place(near, 0) >> TP_MAX_LOG) + 31 - lane;   // ascending logits along the lanes
        const float l = bound_of((u64)key << TP_MAX_LOG).l;
        const u64 fine = __ballot(R.e(l) >= (double)min_p && l <= mx);
        const float least = fminf(mx, __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(l), fine ? __builtin_ctzll(fine) : 63)));
        if (least > bound.l) { bound = {least, ~0u}; total = 0; }
    }

    // the sum of the kept e, by the wavefronts' shares in id order, where it is not known or a token is drawn
    if (P.ids || total == 0) {
        __syncthreads();
        L.each([&](const u32x4& x, int at) {
            u64 m = 0;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float l = Vec<LT>::get(x, e);
                if (at * N + e < V && bound.keeps(l, at * N + e)) m += R.mass(l);
            }
            if (__ballot(m != 0)) m = wave_sum_u64(m);
            if (lane == 0) S.cell[at / 64] = m;
        });
        __syncthreads();
        constexpr int PER = TP_MAX_CELLS / TP_THREADS;
        const int cells = (L.nvec + TP_THREADS - 1) / TP_THREADS * TP_WAVES;
        u64 own[PER], sum = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            own[i] = tid * PER + i < cells ? S.cell[tid * PER + i] : 0;
            sum += own[i];
        }
        u64 upto = block_scan_u64(sum, S, total) - sum;
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
                    m[e] = at * N + e < V && bound.keeps(l, at * N + e) ? R.mass(l) : 0;
                    all += m[e];
                }
                u64 to = S.found_before + wave_scan_u64(all) - all;
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    if (to <= want && to + m[e] > want) {
                        P.ids[row] = at * N + e;
                        if (P.id_probs) P.id_probs[row] = (float)(R.e(Vec<LT>::get(x, e)) / ldexp((double)total, -P.frac));
                    }
                    to += m[e];
                }
            }
        }
    }
    if (!out) return;
    const double cy = R.c / TP_TABLE;
    const float inv = (float)(1.0 / ldexp((double)total, -P.frac));
    L.each([&](const u32x4& x, int at) {
        float p[N];
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float l = Vec<LT>::get(x, e);
            p[e] = 0.f;
            if (bound.keeps(l, at * N + e) && l > -__builtin_inff()) {
                const double y = __builtin_fmax(((double)l - R.max) * cy, -1000.0), n = rint(y);
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
    hipLaunchKernelGGL((target_probs_kernel<LT>), dim3(total), dim3(TP_THREADS), 0, s, P);
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
    P.frac = std::min(51, 62 - log);
    const int total = a->batch * a->rows;
    if (a->dtype == PS_BF16) go<bf16_t>(P, total, (hipStream_t)stream);
    else go<float>(P, total, (hipStream_t)stream);
    return hipGetLastError() == hipSuccess ? PS_OK : PS_ERR_DEVICE;
}

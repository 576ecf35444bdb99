// The target's distributions from its logits, and draws from them (see include/ps_verify.h).
//
//   e_i = 2^y_i,  y_i = (logits_i - max) log2(e) / temperature;  kept = {i : c_i <= bound, e_i >= min_p},  probs_i = e_i / sum of kept e
//
// c_i = (logit, descending; id, ascending) as one whole number puts the tokens in the order in which top-k and top-p take them, so what
// either keeps is everything up to one token, the bound, and min_p is a bound too.  Nothing is sorted:
//   top-k, small k   a histogram of the threads' own maxima gives a lower limit that k tokens reach; the few tokens above it are listed in LDS
//   top-p, large k   a histogram of y in steps of 1/32 (sums of e, or counts) says which step the bound lies in; that step's tokens are listed
//   a listed top-k   has all that may be kept: probabilities, further bounds and draws need the list alone
//   the list         up to 64 tokens by comparing all with all in a wavefront, more by eleven bits of c at a time, from the highest that differs
// e is a whole number of 2^-F (F = 62 - log2 V, at most 51), from a double: sums are exact in any order, whoever adds them, and
// their error is far below what decides a draw.  (Doubles cost no more instructions here than floats, a histogram no more than its additions.)
//
// One workgroup per row (few rows of a large vocabulary: several, see below); the row is read again by each pass, from the caches.  What bounds it: a pass over a row
// that makes masses is 25 instructions per token (V 128256: 12 us on one compute unit), one that only compares is a read.  Measured (us; V 32000 float32, 61 rows,
// top-k 50 and top-p 0.95, probabilities: 18, 3 of them the bytes at a copy's rate; V 128256 bf16, 488 rows: greedy 88, k 50 96, no filter but min-p 132, top-p 175,
// settings of each sequence 139 to 171, bytes 73).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ps_cache_device.h"

namespace {

constexpr int TP_BINS = 2048;                      // steps of 1/32 in y: 64 powers of two, what is below has no mass in F <= 51 bits
constexpr int TP_LIST = 2048;                      // tokens that are ordered in LDS
// top-k by the threads' maxima.  (V 32000, 64 rows, us, by maxima / by the histogram of all: k 50 17.2 / 24.6, k 300 23.0 / 28.0; 512 threads have no more maxima)
constexpr int TP_SMALL_K = 512;
constexpr int TP_MAX_LOG = 20;                     // vocab <= 2^20: an id takes 20 bits of c
constexpr int TP_MAX_CELLS = 4096;                 // wavefronts' shares of a row: 2^20 / (64 * 4)
constexpr int TP_TABLE_LOG = 8, TP_TABLE = 1 << TP_TABLE_LOG;   // 2^(j/256)
constexpr int TP_K_PER_STEP_LOG = TP_TABLE_LOG - 5;

struct TpParams {
    const char* logits;
    const float* temperature;
    const int* top_k;
    const float *top_p, *min_p, *r;
    float* probs;
    int* ids;
    float* id_probs;
    int rows, vocab, frac;                         // F
    int parts, part_vecs;                          // workgroups per row, vectors of each
    char* work;                                    // of each row: see Work
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

__device__ __forceinline__ float uniform(float v) { return __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(v))); }
__device__ __forceinline__ double uniform(double v) {
    return __hiloint2double(__builtin_amdgcn_readfirstlane(__double2hiint(v)), __builtin_amdgcn_readfirstlane(__double2loint(v)));
}
__device__ __forceinline__ u64 lane_u64(u64 v, int lane) {
    return (u64)(unsigned)__builtin_amdgcn_readlane((unsigned)(v >> 32), lane) << 32 | (unsigned)__builtin_amdgcn_readlane((unsigned)v, lane);
}
template <int CTRL, int ROW_MASK> __device__ __forceinline__ u64 dpp_u64(u64 self, u64 v) {
    const unsigned lo = __builtin_amdgcn_update_dpp((int)self, (int)v, CTRL, ROW_MASK, 0xF, false);
    const unsigned hi = __builtin_amdgcn_update_dpp((int)(self >> 32), (int)(v >> 32), CTRL, ROW_MASK, 0xF, false);
    return (u64)hi << 32 | lo;
}
// inclusive prefix sums over a row of 16 lanes, over the wavefront
__device__ __forceinline__ u64 row_scan(u64 v) {
    v += dpp_u64<0x111, 0xF>(0, v);    // row_shr:1, 2, 4, 8
    v += dpp_u64<0x112, 0xF>(0, v);
    v += dpp_u64<0x114, 0xF>(0, v);
    v += dpp_u64<0x118, 0xF>(0, v);
    return v;
}
__device__ __forceinline__ u64 wave_scan(u64 v) {
    v = row_scan(v);
    v += dpp_u64<0x142, 0xA>(0, v);    // row_bcast:15 into rows 1 and 3
    v += dpp_u64<0x143, 0xC>(0, v);    // row_bcast:31 into rows 2 and 3
    return v;
}

struct Shared {
    double table[TP_TABLE];
    union {
        struct { u64 mass[TP_BINS]; unsigned count[TP_BINS]; } h;
        u64 cell[TP_MAX_CELLS];
    };
    u64 list[TP_LIST];
    u64 red[16], red2[16];
    u64 found_before, found_at;
    unsigned red32[16];
    int found, n_list;
};

struct Row {
    double max, c;                                 // the largest logit, 256 log2(e) / temperature
    const double* table;                           // 2^(j/256 + frac)
    // k = rint(256 y); below -80 * 256, and for -Inf: that
    __device__ __forceinline__ double split(float l, int& k) const {
        constexpr double big = 6755399441055744.0;  // 1.5 * 2^52: the sum's low word is the rounded number
        const double u = __builtin_fmax(((double)l - max) * c, -80.0 * TP_TABLE), t = u + big;
        k = __double2loint(t);
        return u - (t - big);
    }
    // e 2^frac = 2^(k / 256 + frac) * (1 + ...): the rest by Taylor's series to the third power (the next is 1.4e-13)
    __device__ __forceinline__ double scaled(float l, int& k) const {
        constexpr double q = 0.69314718055994530942 / TP_TABLE;
        const double r = split(l, k);
        double p = fma(r, q * q * q / 6, q * q / 2);
        p = fma(p, r, q);
        p = fma(p, r, 1.0) * table[k & (TP_TABLE - 1)];
        return __hiloint2double(__double2hiint(p) + ((k >> TP_TABLE_LOG) << 20), __double2loint(p));
    }
    // as a whole number, below 2^52
    __device__ __forceinline__ u64 mass(float l, int& k) const {
        const double x = scaled(l, k) + 4503599627370496.0;
        return (u64)(unsigned)(__double2hiint(x) - 0x43300000) << 32 | (unsigned)__double2loint(x);
    }
    __device__ __forceinline__ u64 mass(float l) const { int k; return mass(l, k); }
    __device__ __forceinline__ int step(float l) const {
        int k;
        split(l, k);
        return step_of(k);
    }
    static __device__ __forceinline__ int step_of(int k) { return min(-k >> TP_K_PER_STEP_LOG, TP_BINS - 1); }
    // about the least logit of a step
    __device__ __forceinline__ float end_of(int step) const { return (float)(max - (((step + 1) << TP_K_PER_STEP_LOG) - 0.5) / c); }
    __device__ __forceinline__ float near_e(float e) const { return (float)(max + log2((double)e) * TP_TABLE / c); }
};

// The token's place: descending logit (0 and -0 are equal), ascending id; and the place up to which tokens are kept
__device__ __forceinline__ unsigned key_of(float l) {
    const unsigned u = __float_as_uint(l + 0.f);
    return u >> 31 ? u : ~u & 0x7FFFFFFFu;
}
__device__ __forceinline__ float logit_of(unsigned key) { return __uint_as_float(key >> 31 ? key : ~key & 0x7FFFFFFFu); }
__device__ __forceinline__ u64 place(float l, int id) { return (u64)key_of(l) << TP_MAX_LOG | (unsigned)id; }
__device__ __forceinline__ float logit_at(u64 c) { return logit_of((unsigned)(c >> TP_MAX_LOG)); }
__device__ __forceinline__ unsigned id_at(u64 c) { return (unsigned)c & ((1u << TP_MAX_LOG) - 1); }
struct Bound {
    float l;
    unsigned id;
    __device__ __forceinline__ bool keeps(float x, unsigned i) const { return x > l || (x == l && i <= id); }
    __device__ __forceinline__ bool all() const { return l == -__builtin_inff() && id == ~0u; }
    // of a vector's logits, ids from `first` on, the ones that are kept (most vectors have no logit like the bound's)
    template <int N> __device__ __forceinline__ unsigned kept(const float (&x)[N], unsigned first) const {
        unsigned yes = 0, same = 0;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            yes |= x[e] > l ? 1u << e : 0;
            same |= x[e] == l ? 1u << e : 0;
        }
        if (__ballot(same != 0)) {
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (first + e > id) same &= ~(1u << e);
            yes |= same;
        }
        return yes;
    }
};
__device__ __forceinline__ Bound bound_of(u64 c) {
    return {uniform(logit_of((unsigned)(c >> TP_MAX_LOG))), (unsigned)__builtin_amdgcn_readfirstlane((unsigned)c & ((1u << TP_MAX_LOG) - 1))};
}
// The least float, at most `max`, for which `pred` holds; it holds for max and for everything between.  near: about where.  Wavefronts do it alike
template <typename F> __device__ __forceinline__ float least_float(float max, float near, F pred) {
    unsigned a = key_of(max), b = 0xFF800000u;              // holds at a; b: one behind the last (-Inf: not asked)
    {
        const unsigned first = key_of(near) - 32, at = first + (threadIdx.x & 63);
        if (first >= a && first < b - 64) {                 // (the 64 floats around `near`: one look where it changes among them)
            const u64 yes = __ballot(pred(logit_of(at)));
            if ((yes & 1) && ~yes) return uniform(logit_of(first + (unsigned)__builtin_ctzll(~yes) - 1));
        }
    }
    while (b - a > 1) {
        const unsigned stride = (b - a + 63) >> 6, at = a + (threadIdx.x & 63) * stride;
        const u64 yes = __ballot(at < b && pred(logit_of(at)));
        const int n = ~yes ? __builtin_ctzll(~yes) : 64;    // (at least one: a itself)
        a += (unsigned)(n - 1) * stride;
        b = min(b, a + stride);
    }
    return uniform(logit_of(a));
}

template <typename LT, int T> struct Logits {               // T threads
    const char* row;
    int vocab, nvec;                                        // tokens of the row; vectors up to the end of
    int begin = 0;                                          // this workgroup's part, which begins here
    // f(vector, its number), by whole wavefronts: what is behind the row's end is -Inf
    template <typename F> __device__ __forceinline__ void each(F f) const {
        u32x4 x = load_vec<LT>(row, begin + (int)threadIdx.x, vocab), next = load_vec<LT>(row, begin + T + (int)threadIdx.x, vocab);
        for (int i = begin; i < nvec; i += T) {             // two vectors ahead
            const u32x4 after = load_vec<LT>(row, i + 2 * T + (int)threadIdx.x, vocab);
            f(x, i + (int)threadIdx.x);
            x = next;
            next = after;
        }
    }
    // f(logit, id) of the row's tokens, and of some behind its end at -Inf
    template <typename F> __device__ __forceinline__ void tokens(F f) const {
        each([&](const u32x4& x, int at) {
#pragma unroll
            for (int e = 0; e < Vec<LT>::N; ++e) {
                f(Vec<LT>::get(x, e), at * Vec<LT>::N + e);
                if (e & 1) __builtin_amdgcn_sched_barrier(0);   // (two at a time: registers)
            }
        });
    }
};

__device__ __forceinline__ void lds_add(u64* p, u64 v) { __hip_atomic_fetch_add(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP); }
__device__ __forceinline__ void lds_add(unsigned* p, unsigned v) { __hip_atomic_fetch_add(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP); }
__device__ __forceinline__ void list_add(Shared& S, u64 c, int vocab) {
    if (((unsigned)c & ((1u << TP_MAX_LOG) - 1)) >= (unsigned)vocab) return;
    const int at = __hip_atomic_fetch_add(&S.n_list, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    if (at < TP_LIST) S.list[at] = c;
}

// inclusive prefix sums over the threads; total to every thread.  Synchronises once, behind which S.red may be used again only after another barrier
template <int T> __device__ __forceinline__ u64 block_scan(u64 v, Shared& S, u64& total) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    v = wave_scan(v);
    if (lane == 63) S.red[wave] = v;
    __syncthreads();
    const u64 w = row_scan((lane & 15) < T / 64 ? S.red[lane & 15] : 0);
    total = lane_u64(w, 15);
    const u64 upto = lane_u64(w, __builtin_amdgcn_readfirstlane(max(wave - 1, 0)));
    return v + (wave > 0 ? upto : 0);
}

// The histogram's first entry with which the sum, `before` in front of it, reaches `want`; S.found, S.found_before to every thread.  of_all >= 0: want is that
// share of the whole.  Takes and leaves synchronised
template <int T> __device__ __forceinline__ u64 find_in_bins(Shared& S, u64 before, u64 want, double of_all) {
    constexpr int PER = TP_BINS / T;
    u64 own[PER], sum = 0, total;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        own[i] = S.h.mass[threadIdx.x * PER + i];
        sum += own[i];
    }
    u64 upto = block_scan<T>(sum, S, total) - sum + before;
    if (of_all >= 0.0) {
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

// Of the list's n tokens, with weights w(entry): the first, in the order of entries, with which the sum (`before` in front of them) reaches `want`.
// with: the sum up to and with that token.  Takes and leaves synchronised
template <int T, typename W> __device__ __forceinline__ u64 find_in_list(Shared& S, int n, u64 before, u64 want, double of_all, u64& with, W w) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if (n <= 64) {                                          // one wavefront
        if (wave == 0) {
            const u64 c = lane < n ? S.list[lane] : ~0ull, m = lane < n ? w(c) : 0;
            if (of_all >= 0.0) {
                const u64 total = lane_u64(wave_scan(m), 63);
                const double t = ceil(of_all * (double)total);
                want = t >= 1.0 ? min((u64)t, total) : 1;
            }
            u64 upto = before;                              // with everything up to the lane's own token
            for (int j = 0; j < n; ++j) {
                const u64 cj = lane_u64(c, j), mj = lane_u64(m, j);
                upto += cj <= c ? mj : 0;
            }
            const u64 hit = __ballot(upto >= want && upto - m < want && m);
            const int at = hit ? __builtin_ctzll(hit) : 0;
            S.found_at = lane_u64(c, at);
            S.found_before = lane_u64(upto, at);
        }
        __syncthreads();
        with = S.found_before;
        const u64 at = S.found_at;
        __syncthreads();                                    // (both may be written again)
        return at;
    }
    constexpr int PER = TP_LIST / T;
    u64 c[PER], m[PER];
    unsigned live = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const bool is = tid + i * T < n;
        c[i] = is ? S.list[tid + i * T] : 0;
        m[i] = is ? w(c[i]) : 0;
        if (m[i]) live |= 1u << i;
    }
    for (int round = 0; round < 6; ++round) {               // (52 bits, eleven and more at a time)
        u64 none = 0, any = 0;                              // bits that one lacks, that one has
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (live >> i & 1) { none |= ~c[i]; any |= c[i]; }
#define TP_OR(CTRL, RM) { none |= dpp_u64<CTRL, RM>(0, none); any |= dpp_u64<CTRL, RM>(0, any); }
        PS_DPP_STEPS(TP_OR)
#undef TP_OR
        if (lane == 63) { S.red[wave] = none; S.red2[wave] = any; }
        for (int i = tid; i < TP_BINS; i += T) S.h.mass[i] = 0;
        __syncthreads();
        none = (lane & 15) < T / 64 ? S.red[lane & 15] : 0;
        any = (lane & 15) < T / 64 ? S.red2[lane & 15] : 0;
#define TP_OR(CTRL, RM) { none |= dpp_u64<CTRL, RM>(0, none); any |= dpp_u64<CTRL, RM>(0, any); }
        PS_DPP_ROW_STEPS(TP_OR)
#undef TP_OR
        any = lane_u64(any, 0);
        const u64 differ = any & lane_u64(none, 0);
        const int shift = differ ? max(0, 63 - __builtin_clzll(differ) - 10) : 0;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (live >> i & 1) lds_add(&S.h.mass[(c[i] >> shift) & (TP_BINS - 1)], m[i]);
        __syncthreads();
        want = find_in_bins<T>(S, before, want, of_all);
        of_all = -1.0;
        const int digit = S.found;
        before = S.found_before;
        if (differ >> 11 == 0) {                            // these eleven bits were the last ones
            with = before + S.h.mass[digit];
            __syncthreads();
            return (any & ~(u64)(TP_BINS - 1)) | (unsigned)digit;
        }
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if ((int)((c[i] >> shift) & (TP_BINS - 1)) != digit) live &= ~(1u << i);
        __syncthreads();
    }
    return ~0ull;
}

// The bound of the row's tokens that `within` keeps: the first token with which the sum of e (BY_MASS) reaches top_p of their sum, or the
// top_k-th.  with: the sum up to and with it.  Synchronises before it writes anything shared: wavefronts may still read what it resets
template <bool BY_MASS, typename LT, int T>
__device__ __forceinline__ u64 find_in_row(const Logits<LT, T>& L, const Row& R, float mx, Shared& S, Bound within, u64 want, double of_all, u64& with) {
    const int tid = threadIdx.x;
    __syncthreads();
    auto weight = [&](u64 c) { return BY_MASS ? R.mass(logit_at(c)) : (u64)1; };
    for (int i = tid; i < TP_BINS; i += T) S.h.mass[i] = 0;
    if (tid == 0) S.n_list = 0;
    __syncthreads();
    auto count = [&](float l) {
        if constexpr (BY_MASS) {
            int k;
            const u64 m = R.mass(l, k);
            lds_add(&S.h.mass[R.step_of(k)], m);
        } else lds_add((unsigned*)&S.h.mass[R.step(l)], 1u);
    };
    // (what is behind the row's end has no mass, and counts in the last step, behind all that is wanted)
    if (within.all()) L.tokens([&](float l, int) { count(l); });
    else L.tokens([&](float l, int id) { if (within.keeps(l, id)) count(l); });
    __syncthreads();
    want = find_in_bins<T>(S, 0, want, of_all);
    const int step = S.found;
    u64 before = S.found_before;
    // the step's logits: least <= l < above
    const float least = step < TP_BINS - 1 ? least_float(mx, R.end_of(step), [&](float l) { return R.step(l) <= step; }) : -__builtin_inff();
    const float above = step > 0 ? least_float(mx, R.end_of(step - 1), [&](float l) { return R.step(l) < step; }) : __builtin_inff();
    L.tokens([&](float l, int id) {
        if (l >= least && l < above && within.keeps(l, id)) list_add(S, place(l, id), L.vocab);
    });
    __syncthreads();
    if (S.n_list <= TP_LIST) return find_in_list<T>(S, S.n_list, before, want, -1.0, with, weight);
    // more tokens than the list holds (equal or nearly equal logits): eleven bits of the place at a time, until few enough are left
    u64 prefix = 0;
    for (int shift = 44;; shift -= 11) {
        __syncthreads();
        for (int i = tid; i < TP_BINS; i += T) { S.h.mass[i] = 0; S.h.count[i] = 0; }
        if (tid == 0) S.n_list = 0;
        __syncthreads();
        L.tokens([&](float l, int id) {
            const u64 c = place(l, id);
            if (!(l >= least && l < above && within.keeps(l, id)) || c >> (shift + 11) != prefix || id >= L.vocab) return;
            const int digit = (int)(c >> shift) & (TP_BINS - 1);
            lds_add(&S.h.count[digit], 1u);
            lds_add(&S.h.mass[digit], weight(c));
        });
        __syncthreads();
        find_in_bins<T>(S, before, want, -1.0);
        prefix = prefix << 11 | (unsigned)S.found;
        before = S.found_before;
        if (S.h.count[S.found] > TP_LIST && shift > 0) continue;   // (at the last digit it is one token)
        L.tokens([&](float l, int id) {
            const u64 c = place(l, id);
            if (c >> shift == prefix && l >= least && l < above && within.keeps(l, id)) list_add(S, c, L.vocab);   // (the step's: what is in front of it is in `before`)
        });
        __syncthreads();
        return find_in_list<T>(S, S.n_list, before, want, -1.0, with, weight);
    }
}

// the sums of the kept e of the wavefronts' vectors, in id order (S.cell), and of all
template <int T, typename LT> __device__ __forceinline__ u64 sum_cells(const Logits<LT, T>& L, const Row& R, Shared& S, Bound bound) {
    constexpr int N = Vec<LT>::N, PER = TP_MAX_CELLS / T;
    const int tid = threadIdx.x, lane = tid & 63;
    const bool all = bound.all();
    L.each([&](const u32x4& x, int at) {
        u64 m = 0;
        if (all) {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                m += R.mass(Vec<LT>::get(x, e));
                if (e & 1) __builtin_amdgcn_sched_barrier(0);
            }
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float l = Vec<LT>::get(x, e);
                if (bound.keeps(l, at * N + e)) m += R.mass(l);
                if (e & 1) __builtin_amdgcn_sched_barrier(0);
            }
        }
        if (__ballot(m != 0)) m = wave_scan(m);
        if (lane == 63) S.cell[(at - L.begin) >> 6] = m;
    });
    __syncthreads();
    const int cells = (L.nvec - L.begin + T - 1) / T * (T / 64);
    u64 sum = 0, total;
    for (int i = 0; i < PER; ++i) sum += tid * PER + i < cells ? S.cell[tid * PER + i] : 0;
    block_scan<T>(sum, S, total);
    return total;
}
// The mass up to which the draw goes: the drawn token is the first with which the sum passes it
__device__ __forceinline__ u64 drawn_mass(float r, u64 total) {
    const double t = (double)r * (double)total;
    return t >= 1.0 ? min((u64)t, total - 1) : 0;
}
// The token with which the sum, `before` in front of the part, passes `want`; takes S.cell
template <int T, typename LT>
__device__ __forceinline__ void draw_from_cells(const TpParams& P, const Logits<LT, T>& L, const Row& R, Shared& S, Bound bound, size_t row, u64 before, u64 want, u64 total) {
    constexpr int N = Vec<LT>::N, PER = TP_MAX_CELLS / T;
    const int tid = threadIdx.x, lane = tid & 63;
    const int cells = (L.nvec - L.begin + T - 1) / T * (T / 64);
    u64 sum = 0, all;
    for (int i = 0; i < PER; ++i) sum += tid * PER + i < cells ? S.cell[tid * PER + i] : 0;
    __syncthreads();
    u64 upto = before + block_scan<T>(sum, S, all) - sum;
    if (upto <= want && upto + sum > want)
        for (int i = 0; i < PER; ++i) {
            const u64 own = tid * PER + i < cells ? S.cell[tid * PER + i] : 0;
            if (upto <= want && upto + own > want) { S.found = tid * PER + i; S.found_before = upto; }
            upto += own;
        }
    __syncthreads();
    if (tid >= 64) return;
    const int at = L.begin + S.found * 64 + lane;
    const u32x4 x = load_vec<LT>(L.row, at, L.vocab);
    u64 mine = 0;
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const float l = Vec<LT>::get(x, e);
        if (bound.keeps(l, at * N + e)) mine += R.mass(l);
    }
    u64 to = S.found_before + wave_scan(mine) - mine;
    if (to <= want && to + mine > want)
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float l = Vec<LT>::get(x, e);
            const u64 m = bound.keeps(l, at * N + e) ? R.mass(l) : 0;
            if (to <= want && to + m > want) {
                P.ids[row] = at * N + e;
                int kk;
                if (P.id_probs) P.id_probs[row] = (float)(R.scaled(l, kk) / (double)total);
            }
            to += m;
        }
}
template <int T, typename LT>
__device__ __forceinline__ void draw(const TpParams& P, const Logits<LT, T>& L, const Row& R, Shared& S, Bound bound, size_t row, u64 before, u64 want, u64 total) {
    sum_cells<T>(L, R, S, bound);
    draw_from_cells<T>(P, L, R, S, bound, row, before, want, total);
}
// a kept token's probability
struct Prob {
    double max, c;
    float inv;
    __device__ __forceinline__ Prob(const Row& R, int frac, u64 total) : max(R.max), c(R.c / TP_TABLE), inv((float)(1.0 / ldexp((double)total, -frac))) {}
    __device__ __forceinline__ float operator()(float l) const {
        const double y = __builtin_fmax(((double)l - max) * c, -1000.0), t = y + 6755399441055744.0;   // (1.5 * 2^52: the low word is rint(y))
        return ldexpf(__builtin_amdgcn_exp2f((float)(y - (t - 6755399441055744.0))) * inv, __double2loint(t));
    }
};
// The probabilities of a row whose kept tokens are all in the list: zeros, which need no look at the logits, and theirs (488 rows of V 128256 bf16, greedy 110 -> 89 us, k 50
// 114 -> 97)
template <int T> __device__ __forceinline__ void write_listed(const TpParams& P, const Row& R, Shared& S, int n, Bound bound, size_t row, u64 total) {
    float* out = P.probs + row * P.vocab;
    const Prob prob(R, P.frac, total);
    for (int i = threadIdx.x * 4; i < P.vocab; i += T * 4) {
        if (i + 4 <= P.vocab) *reinterpret_cast<f32x4_q*>(out + i) = f32x4{0, 0, 0, 0};
        else for (int e = i; e < P.vocab; ++e) out[e] = 0.f;
    }
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += T) {
        const u64 c = S.list[i];
        const float l = logit_at(c);
        if (bound.keeps(l, id_at(c))) out[id_at(c)] = prob(l);
    }
}
// The draw among them, in the order of ids; the list is turned into that of (id, logit)
template <int T> __device__ __forceinline__ void draw_listed(const TpParams& P, const Row& R, Shared& S, int n, Bound bound, size_t row, u64 total) {
    __syncthreads();
    for (int i = threadIdx.x; i < n; i += T) S.list[i] = (u64)id_at(S.list[i]) << 32 | (unsigned)(S.list[i] >> TP_MAX_LOG);
    __syncthreads();
    u64 with;
    auto kept = [&](u64 c) { const float l = logit_of((unsigned)c); return bound.keeps(l, (unsigned)(c >> 32)) ? R.mass(l) : 0; };
    const u64 at = find_in_list<T>(S, n, 0, drawn_mass(P.r[row], total) + 1, -1.0, with, kept);
    if (threadIdx.x == 0) {
        P.ids[row] = (int)(at >> 32);
        int k;
        if (P.id_probs) P.id_probs[row] = (float)(R.scaled(logit_of((unsigned)at), k) / (double)total);
    }
}
template <int T, typename LT>
__device__ __forceinline__ void write_probs(const TpParams& P, const Logits<LT, T>& L, const Row& R, Bound bound, size_t row, u64 total) {
    constexpr int N = Vec<LT>::N;
    const int V = L.vocab;
    float* out = P.probs + row * V;
    const bool all = bound.all();
    const Prob prob(R, P.frac, total);
    L.each([&](const u32x4& x, int at) {
        if (at >= L.nvec) return;                           // (the next part's)
        float p[N], l[N];
#pragma unroll
        for (int e = 0; e < N; ++e) l[e] = Vec<LT>::get(x, e);
        if (all) {
#pragma unroll
            for (int e = 0; e < N; ++e) {
                p[e] = prob(l[e]);                          // (-Inf: 2^-1000 is 0)
                if (e & 1) __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            const unsigned kept = bound.kept(l, at * N);
#pragma unroll
            for (int e = 0; e < N; ++e) p[e] = 0.f;
            if (__ballot(kept != 0)) {
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    if (kept >> e & 1) p[e] = prob(l[e]);
                    if (e & 1) __builtin_amdgcn_sched_barrier(0);
                }
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

// a row without mass (bad: with a NaN or +Inf)
__device__ __forceinline__ void no_token(const TpParams& P, size_t row, bool bad) {
    P.ids[row] = -1;
    if (P.id_probs) P.id_probs[row] = bad ? __builtin_nanf("") : 0.f;
}
// min_p's bound, where it is above `bound`
__device__ __forceinline__ void apply_min_p(const TpParams& P, const Row& R, float min_p, Bound& bound, u64& total) {
    if (!(min_p > 0.f)) return;
    // (exponentials stop at 2^-80: a min_p down there is compared in the exponent)
    const bool tiny = min_p < 0x1p-79f;
    const double least_e = tiny ? log2((double)min_p) * TP_TABLE : ldexp((double)min_p, P.frac);
    int kk;
    const float least = least_float((float)R.max, R.near_e(min_p), [&](float l) { return tiny ? ((double)l - R.max) * R.c >= least_e : R.scaled(l, kk) >= least_e; });
    if (least > bound.l) { bound = {least, ~0u}; total = 0; }
}

template <typename LT, int T>
__global__ __launch_bounds__(T, 4) void target_probs_kernel(const TpParams P) {
    constexpr int N = Vec<LT>::N, WAVES = T / 64;
    __shared__ Shared S;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = P.vocab;
    const size_t row = blockIdx.x;
    const int b = (int)(row / (unsigned)P.rows);
    Logits<LT, T> L;
    L.row = P.logits + row * V * Traits<LT>::ESZ; L.vocab = V; L.nvec = (V + N - 1) / N;
    const float t_in = P.temperature ? P.temperature[b] : 1.f;
    const bool greedy = !(t_in > 0.f);
    const int k_in = P.top_k ? P.top_k[b] : 0;
    const int k = greedy ? 1 : k_in < 1 || k_in > V ? V : k_in;
    const float p_in = P.top_p ? P.top_p[b] : 1.f, m_in = P.min_p ? P.min_p[b] : 0.f, min_p = m_in > 0.f ? fminf(m_in, 1.f) : 0.f;
    if (tid < TP_TABLE) S.table[tid] = ga_exp2(tid * (1.0 / TP_TABLE) + P.frac);

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
    const float mine = mx;
    mx = __ballot(bad) ? __builtin_nanf("") : wave_max(mx);
    if (lane == 0) S.red32[wave] = __float_as_uint(mx);
    if (tid == 0) { S.n_list = 0; S.found = V; }
    for (int i = tid; i < TP_BINS; i += T) S.h.mass[i] = 0;
    __syncthreads();
    mx = __uint_as_float(S.red32[lane % WAVES]);
    bad = __ballot(mx != mx);
    mx = uniform(row_max(mx));
    float* out = P.probs ? P.probs + row * V : nullptr;
    if (bad || mx == -__builtin_inff()) {
        if (out) for (int i = tid; i < V; i += T) out[i] = bad ? __builtin_nanf("") : 0.f;
        if (P.ids && tid == 0) no_token(P, row, bad);
        return;
    }
    Row R;
    R.max = mx; R.c = uniform(1.4426950408889634074 * TP_TABLE / (greedy ? 1.0 : (double)t_in)); R.table = S.table;
    Bound bound = {-__builtin_inff(), ~0u};
    u64 total = 0;                                          // the sum of the kept e, where it is known
    auto mass = [&](u64 c) { return R.mass(logit_at(c)); };
    auto one = [](u64) { return (u64)1; };
    int listed = -1;                                        // tokens in S.list, where these are all that may be kept
    if (k == 1) {                                           // the first of the largest
        L.tokens([&](float l, int id) { if (l == mx) __hip_atomic_fetch_min(&S.found, id, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP); });
        __syncthreads();
        bound = {mx, (unsigned)S.found};
        total = R.mass(mx);
        if (tid == 0) S.list[0] = place(mx, S.found);
        listed = 1;
        __syncthreads();
    } else {
        const bool all = k == V;                            // no top-k, or one that only drops tokens at -Inf
        u64 with = 0;
        if (k <= TP_SMALL_K && k <= min(T, L.nvec)) {
            // k threads' maxima are at or above some step: so are the k largest tokens, which are listed
            if (tid < L.nvec) lds_add((unsigned*)&S.h.mass[R.step(mine)], 1u);
            __syncthreads();
            find_in_bins<T>(S, 0, (u64)k, -1.0);
            const int step = S.found;
            if (step < TP_BINS - 1) {
                const float least = least_float(mx, R.end_of(step), [&](float l) { return R.step(l) <= step; });
                L.tokens([&](float l, int id) { if (l >= least) list_add(S, place(l, id), L.vocab); });
                __syncthreads();
                if (S.n_list <= TP_LIST) listed = S.n_list;
            }
        }
        if (listed >= 0) {
            const int n = listed;
            bound = bound_of(find_in_list<T>(S, n, 0, (u64)k, -1.0, with, one));
            u64 m = 0;
            for (int i = tid; i < n; i += T) {              // tokens behind the bound leave the list: the last place, without mass
                const u64 c = S.list[i];
                const float l = logit_at(c);
                const unsigned id = id_at(c);
                if (bound.keeps(l, id)) m += R.mass(l);
                else S.list[i] = place(-__builtin_inff(), id);
            }
            block_scan<T>(m, S, total);
            if (p_in < 1.f) {
                __syncthreads();
                bound = bound_of(find_in_list<T>(S, n, 0, 0, fmax((double)p_in, 0.0), with, mass));
                total = with;
            }
        } else {
            if (!all) bound = bound_of(find_in_row<false>(L, R, mx, S, bound, (u64)k, -1.0, with));
            if (p_in < 1.f) {
                bound = bound_of(find_in_row<true>(L, R, mx, S, bound, 0, fmax((double)p_in, 0.0), with));
                total = with;
            }
        }
    }
    apply_min_p(P, R, min_p, bound, total);

    // the sum of the kept e, where it is not known
    if (total == 0 && listed >= 0) {
        u64 m = 0;
        for (int i = tid; i < listed; i += T)
            if (bound.keeps(logit_at(S.list[i]), id_at(S.list[i]))) m += R.mass(logit_at(S.list[i]));
        __syncthreads();
        block_scan<T>(m, S, total);
    } else if (listed < 0 && (P.ids || total == 0)) {
        __syncthreads();
        total = sum_cells<T>(L, R, S, bound);
    }
    if (P.probs) {
        if (listed >= 0) write_listed<T>(P, R, S, listed, bound, row, total);
        else write_probs(P, L, R, bound, row, total);
    }
    if (P.ids) {
        if (listed < 0) draw_from_cells<T>(P, L, R, S, bound, row, 0, drawn_mass(P.r[row], total), total);
        else draw_listed<T>(P, R, S, listed, bound, row, total);
    }
}

// ------------------------------------------------------------------------------------------
// Few rows of a large vocabulary: several workgroups per row, a kernel for each pass.  What a row's workgroups tell each other is in the workspace.
// ------------------------------------------------------------------------------------------
// A workgroup's tokens are a multiple of TP_PART (a pass of 1024 threads over bf16).  Masses of a row take one workgroup long, but every kernel reads the row once more,
// and the chain is six kernels.  The host sees sizes and which settings are given, not what they say, so the rule goes by these; cut up / one workgroup per row,
// bf16, probabilities (d: draws), us:
//               no filter   top-p     top-p d    greedy   k 50, p   k 2000
//   V 128256,  8 rows  20 / 49   35 / 78    42 / 88    19 / 19   30 / 27    69 / 83
//   V 128256, 64 rows  32 / 53   54 / 81    66 / 90    23 / 22   44 / 30    90 / 86
//   V 128256, 96 rows  53 / 53   82 / 82   111 / 91    35 / 22   62 / 31   127 / 87
//   V 128256, 128      47 / 54   75 / 83    97 / 91    31 / 24   58 / 32   120 / 87
//   V 70000,   8 rows  20 / 30   34 / 51    41 / 58    20 / 12   31 / 21    60 / 58
//   V 64000,   8 rows  20 / 28   32 / 46    39 / 53    19 / 12   29 / 20    55 / 53
//   V 48000,   8 rows  20 / 23   32 / 39    39 / 44    20 / 10   29 / 18    51 / 45
//   V 32000,   8 rows  21 / 17   31 / 30    38 / 35    21 / 8    29 / 17    40 / 35
// Rows are cut up from TP_SPLIT_VOCAB on, up to TP_SPLIT_ROWS: there rows with masses gain up to 2.5, those with few (greedy, a small k) lose 1.2 to 1.8, and 2 to 2.5
// where they are only drawn (greedy, V 70000, 64 rows 26 / 11).  With more rows draws by top-p lose too; with a smaller vocabulary the gains go (48000: 1.2) and the losses stay.
// Calls with top-k and no top-p: one workgroup per row, which is right for a small k and not for a large one (V 128256, k 50, 8 rows 27 / 24, drawn 32 / 22, 64 rows 41 / 27; k 2000,
// 8 rows 69 / 83, drawn 72 / 64, 64 rows 90 / 86; V 260000, 8 rows, k 50 30 / 37, drawn 34 / 31, k 2000 91 / 134, drawn 94 / 100).
constexpr int TP_PART = 8192;
constexpr int TP_SPLIT_ROWS = 64;                  // rows up to which they are cut up,
constexpr int TP_SPLIT_VOCAB = 65536;              // from this vocabulary on
constexpr int TP_MAX_PARTS = 64;
struct Work {
    u64 hist[TP_BINS];
    u64 list[TP_LIST];
    u64 sum[TP_MAX_PARTS];                         // the parts' sums of the kept e
    float max[TP_MAX_PARTS];                       // their largest logits, NaN where one is NaN or +Inf
    int first[TP_MAX_PARTS];                       // the first token of theirs that has it
    u64 total;                                     // the sum over the row where it is known
    Bound bound;
    u64 before, want;                              // top-p: the sum in front of the listed step, the sum to be reached
    int n_list;
};

// A row's settings and its largest logit (every lane the same); false: nothing to be searched for (bad: NaN or +Inf; max -Inf: no mass)
struct Setting {
    float max, top_p, min_p;
    int k, first;                                  // first: the first token that has the largest logit
    bool bad;
    double c;
    bool search;                                   // top-k of more than one or top-p leave something out: the bound is in the workspace
    __device__ __forceinline__ bool plain() const { return bad || max == -__builtin_inff(); }
};
__device__ __forceinline__ Setting setting_of(const TpParams& P, const Work& W, int b) {
    Setting s;
    const float t = P.temperature ? P.temperature[b] : 1.f;
    const bool greedy = !(t > 0.f);
    const int k = P.top_k ? P.top_k[b] : 0;
    s.k = greedy ? 1 : k < 1 || k > P.vocab ? P.vocab : k;
    s.top_p = P.top_p ? P.top_p[b] : 1.f;
    const float m = P.min_p ? P.min_p[b] : 0.f;
    s.min_p = m > 0.f ? fminf(m, 1.f) : 0.f;
    s.search = s.k != 1 && (s.k < P.vocab || s.top_p < 1.f);
    const int lane = threadIdx.x & 63;
    const float x = lane < P.parts ? W.max[lane] : -__builtin_inff();
    s.bad = __ballot(x != x);
    s.max = wave_max(x);
    const u64 at = __ballot(x == s.max);                    // (parts in order: the first one has the first token)
    s.first = W.first[at ? __builtin_ctzll(at) : 0];
    s.c = uniform(1.4426950408889634074 * TP_TABLE / (greedy ? 1.0 : (double)t));
    return s;
}
static_assert(TP_MAX_PARTS <= 64, "a lane for each part");
static_assert(TP_PART % (1024 * Vec<bf16_t>::N) == 0, "parts end where passes of 1024 threads do");

template <typename LT> __device__ __forceinline__ Logits<LT, 1024> part_of(const TpParams& P, size_t row, int part) {
    Logits<LT, 1024> L;
    constexpr int N = Vec<LT>::N;
    L.row = P.logits + row * P.vocab * Traits<LT>::ESZ;
    L.vocab = P.vocab;
    L.begin = part * P.part_vecs;
    L.nvec = min((P.vocab + N - 1) / N, L.begin + P.part_vecs);
    return L;
}

template <typename LT> __global__ __launch_bounds__(1024) void part_max_kernel(const TpParams P) {
    __shared__ float s_max[16];
    __shared__ int s_first;
    const int tid = threadIdx.x, lane = tid & 63, part = blockIdx.x;
    const size_t row = blockIdx.y;
    Work& W = reinterpret_cast<Work*>(P.work)[row];
    for (int i = part * 1024 + tid; i < TP_BINS; i += P.parts * 1024) W.hist[i] = 0;
    if (part == 0 && tid == 0) W.n_list = 0;
    if (tid == 0) s_first = P.vocab;
    float mx = -__builtin_inff();
    int first = 0;
    bool bad = false;
    part_of<LT>(P, row, part).each([&](const u32x4& x, int at) {
#pragma unroll
        for (int e = 0; e < Vec<LT>::N; ++e) {
            const float l = Vec<LT>::get(x, e);
            bad |= !(l < __builtin_inff());
            first = l > mx ? at * Vec<LT>::N + e : first;
            mx = fmaxf(mx, l);
        }
    });
    const float mine = mx;
    mx = __ballot(bad) ? __builtin_nanf("") : wave_max(mx);
    if (lane == 0) s_max[tid >> 6] = mx;
    __syncthreads();
    mx = s_max[lane & 15];
    bad = __ballot(mx != mx);
    mx = row_max(mx);
    if (mine == mx) __hip_atomic_fetch_min(&s_first, first, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    __syncthreads();
    if (tid == 0) {
        W.max[part] = bad ? __builtin_nanf("") : mx;
        W.first[part] = s_first;
    }
}

// the row's bound and, where it is known, the sum of what it keeps
__device__ __forceinline__ void bound_of_row(const TpParams& P, const Work& W, const Setting& s, const Row& R, Bound& bound, u64& total) {
    if (s.search) { bound = W.bound; total = W.total; }
    else if (s.k == 1) { bound = {s.max, (unsigned)s.first}; total = R.mass(s.max); }
    else {
        bound = {-__builtin_inff(), ~0u};
        total = 0;
        apply_min_p(P, R, s.min_p, bound, total);
    }
}

// the histogram that the row's setting asks for: counts for top-k, else sums of e for top-p
template <typename LT> __global__ __launch_bounds__(1024, 4) void part_hist_kernel(const TpParams P) {
    __shared__ double s_table[TP_TABLE];
    __shared__ u64 s_hist[TP_BINS];
    const int tid = threadIdx.x;
    const size_t row = blockIdx.y;
    Work& W = reinterpret_cast<Work*>(P.work)[row];
    const Setting s = setting_of(P, W, (int)(row / (unsigned)P.rows));
    if (s.plain() || !s.search) return;
    if (tid < TP_TABLE) s_table[tid] = ga_exp2(tid * (1.0 / TP_TABLE) + P.frac);
    for (int i = tid; i < TP_BINS; i += 1024) s_hist[i] = 0;
    __syncthreads();
    const Row R = {s.max, s.c, s_table};
    const auto L = part_of<LT>(P, row, blockIdx.x);
    if (s.k < P.vocab) L.tokens([&](float l, int) { lds_add((unsigned*)&s_hist[R.step(l)], 1u); });
    else L.tokens([&](float l, int) {
        int k;
        const u64 m = R.mass(l, k);
        lds_add(&s_hist[R.step_of(k)], m);
    });
    __syncthreads();
    for (int i = tid; i < TP_BINS; i += 1024)
        if (s_hist[i]) __hip_atomic_fetch_add(&W.hist[i], s_hist[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The step that the bound lies in, from the row's histogram, and the range of logits whose tokens are listed: top-k everything down to that step, top-p the step
struct Range { float least, above; u64 before, want; };
__device__ __forceinline__ Range range_of(const TpParams& P, const Work& W, const Setting& s, const Row& R, Shared& S) {
    for (int i = threadIdx.x; i < TP_BINS; i += 1024) S.h.mass[i] = W.hist[i];
    __syncthreads();
    const bool count = s.k < P.vocab;
    Range r;
    r.want = find_in_bins<1024>(S, 0, (u64)s.k, count ? -1.0 : fmax((double)s.top_p, 0.0));
    const int step = S.found;
    r.before = count ? 0 : S.found_before;
    r.least = step < TP_BINS - 1 ? least_float(s.max, R.end_of(step), [&](float l) { return R.step(l) <= step; }) : -__builtin_inff();
    r.above = !count && step > 0 ? least_float(s.max, R.end_of(step - 1), [&](float l) { return R.step(l) < step; }) : __builtin_inff();
    return r;
}

template <typename LT> __global__ __launch_bounds__(1024, 4) void part_list_kernel(const TpParams P) {
    __shared__ Shared S;
    const int tid = threadIdx.x;
    const size_t row = blockIdx.y;
    Work& W = reinterpret_cast<Work*>(P.work)[row];
    const Setting s = setting_of(P, W, (int)(row / (unsigned)P.rows));
    if (s.plain() || !s.search) return;
    const Row R = {s.max, s.c, S.table};
    const Range r = range_of(P, W, s, R, S);
    if (blockIdx.x == 0 && tid == 0) { W.before = r.before; W.want = r.want; }
    part_of<LT>(P, row, blockIdx.x).tokens([&](float l, int id) {
        if (!(l >= r.least && l < r.above) || id >= P.vocab) return;
        const int at = __hip_atomic_fetch_add(&W.n_list, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (at < TP_LIST) W.list[at] = place(l, id);
    });
}

// the row's bound, by one workgroup
template <typename LT> __global__ __launch_bounds__(1024, 4) void row_bound_kernel(const TpParams P) {
    __shared__ Shared S;
    const int tid = threadIdx.x;
    const size_t row = blockIdx.x;
    Work& W = reinterpret_cast<Work*>(P.work)[row];
    const Setting s = setting_of(P, W, (int)(row / (unsigned)P.rows));
    if (s.plain() || !s.search) return;
    const Row R = {s.max, s.c, S.table};
    if (tid < TP_TABLE) S.table[tid] = ga_exp2(tid * (1.0 / TP_TABLE) + P.frac);
    Bound bound = {-__builtin_inff(), ~0u};
    u64 total = 0, with = 0;
    auto mass = [&](u64 c) { return R.mass(logit_at(c)); };
    const int n = W.n_list;
    if (n <= TP_LIST) {
        for (int i = tid; i < n; i += 1024) S.list[i] = W.list[i];
        __syncthreads();
        if (s.k < P.vocab) {
            bound = bound_of(find_in_list<1024>(S, n, 0, (u64)s.k, -1.0, with, [](u64) { return (u64)1; }));
            u64 m = 0;
            for (int i = tid; i < n; i += 1024) {           // tokens behind the bound leave the list: the last place, without mass
                const u64 c = S.list[i];
                const float l = logit_at(c);
                const unsigned id = id_at(c);
                if (bound.keeps(l, id)) m += R.mass(l);
                else S.list[i] = place(-__builtin_inff(), id);
            }
            block_scan<1024>(m, S, total);
            if (s.top_p < 1.f) {
                __syncthreads();
                bound = bound_of(find_in_list<1024>(S, n, 0, 0, fmax((double)s.top_p, 0.0), with, mass));
                total = with;
            }
        } else {
            bound = bound_of(find_in_list<1024>(S, n, W.before, W.want, -1.0, with, mass));
            total = with;
        }
    // More tokens than the list holds (a flat row, many equal logits, a top_k above 2000): the whole row, by this workgroup alone.  (8 rows of V 128256, top-p 0.9, us: temperature
    // 2 41, temperature 8, where the step has 7000 tokens, 189; one workgroup per row does that in 363 for 488 rows, 175 at temperature 1)
    } else {
        Logits<LT, 1024> L;
        L.row = P.logits + row * P.vocab * Traits<LT>::ESZ; L.vocab = P.vocab; L.nvec = (P.vocab + Vec<LT>::N - 1) / Vec<LT>::N;
        if (s.k < P.vocab) bound = bound_of(find_in_row<false>(L, R, s.max, S, bound, (u64)s.k, -1.0, with));
        if (s.top_p < 1.f) {
            bound = bound_of(find_in_row<true>(L, R, s.max, S, bound, 0, fmax((double)s.top_p, 0.0), with));
            total = with;
        }
    }
    apply_min_p(P, R, s.min_p, bound, total);
    if (tid == 0) { W.bound = bound; W.total = total; }
}

// the parts' sums of the kept e, where the row's is not known or a token is drawn
template <typename LT> __global__ __launch_bounds__(1024, 4) void part_sum_kernel(const TpParams P) {
    __shared__ double s_table[TP_TABLE];
    __shared__ u64 s_sum[16];
    const int tid = threadIdx.x;
    const size_t row = blockIdx.y;
    Work& W = reinterpret_cast<Work*>(P.work)[row];
    const Setting s = setting_of(P, W, (int)(row / (unsigned)P.rows));
    if (s.plain() || ((s.k == 1 || (s.search && W.total)) && !P.ids)) return;
    if (tid < TP_TABLE) s_table[tid] = ga_exp2(tid * (1.0 / TP_TABLE) + P.frac);
    __syncthreads();
    const Row R = {s.max, s.c, s_table};
    Bound bound;
    u64 total, m = 0;
    bound_of_row(P, W, s, R, bound, total);
    const auto L = part_of<LT>(P, row, blockIdx.x);
    if (bound.all()) L.tokens([&](float l, int) { m += R.mass(l); });
    else L.tokens([&](float l, int id) { if (bound.keeps(l, id)) m += R.mass(l); });
    m = wave_scan(m);
    if ((tid & 63) == 63) s_sum[tid >> 6] = m;
    __syncthreads();
    m = row_scan(s_sum[tid & 15]);
    if (tid == 15) W.sum[blockIdx.x] = m;
}

// the part's probabilities, and the drawn token where it is the part's
template <typename LT> __global__ __launch_bounds__(1024, 4) void part_out_kernel(const TpParams P) {
    __shared__ Shared S;
    const int tid = threadIdx.x, lane = tid & 63, part = blockIdx.x;
    const size_t row = blockIdx.y;
    Work& W = reinterpret_cast<Work*>(P.work)[row];
    const Setting s = setting_of(P, W, (int)(row / (unsigned)P.rows));
    const auto L = part_of<LT>(P, row, part);
    if (s.plain()) {
        if (P.probs) for (int i = L.begin * Vec<LT>::N + tid; i < min(P.vocab, L.nvec * Vec<LT>::N); i += 1024) P.probs[row * P.vocab + i] = s.bad ? __builtin_nanf("") : 0.f;
        if (P.ids && part == 0 && tid == 0) no_token(P, row, s.bad);
        return;
    }
    if (tid < TP_TABLE) S.table[tid] = ga_exp2(tid * (1.0 / TP_TABLE) + P.frac);
    __syncthreads();
    const Row R = {s.max, s.c, S.table};
    Bound bound;
    u64 total;
    bound_of_row(P, W, s, R, bound, total);
    if (P.ids || total == 0) {
        const u64 own = lane < P.parts ? W.sum[lane] : 0, upto = wave_scan(own);
        total = lane_u64(upto, 63);
        if (P.ids) {
            const u64 want = drawn_mass(P.r[row], total);
            if (lane_u64(upto, part) > want && lane_u64(upto - own, part) <= want)
                draw<1024>(P, L, R, S, bound, row, lane_u64(upto - own, part), want, total);
        }
    }
    if (P.probs) write_probs(P, L, R, bound, row, total);
}

template <typename LT> void go(const TpParams& P, int total, hipStream_t s) {
    if (P.work) {
        const dim3 grid(P.parts, total), block(1024);
        hipLaunchKernelGGL((part_max_kernel<LT>), grid, block, 0, s, P);
        if (P.top_k || P.top_p) {
            hipLaunchKernelGGL((part_hist_kernel<LT>), grid, block, 0, s, P);
            hipLaunchKernelGGL((part_list_kernel<LT>), grid, block, 0, s, P);
            hipLaunchKernelGGL((row_bound_kernel<LT>), dim3(total), block, 0, s, P);
        }
        hipLaunchKernelGGL((part_sum_kernel<LT>), grid, block, 0, s, P);
        hipLaunchKernelGGL((part_out_kernel<LT>), grid, block, 0, s, P);
    // (a workgroup per compute unit: all its threads; two: 512 each.  V 32000, top-p, us: 240 rows 34 with 1024 threads, 39 with 512, 300 rows 60 and 50)
    } else if (total <= 256) hipLaunchKernelGGL((target_probs_kernel<LT, 1024>), dim3(total), dim3(1024), 0, s, P);
    else hipLaunchKernelGGL((target_probs_kernel<LT, 512>), dim3(total), dim3(512), 0, s, P);
}

// tokens of a workgroup; 0: a row is one workgroup's
int part_of(const ps_target_probs_args* a) {
    const long long rows = (long long)a->batch * a->rows;
    if (a->vocab < TP_SPLIT_VOCAB || rows > TP_SPLIT_ROWS || (a->top_k && !a->top_p)) return 0;
    // about as many workgroups as there are compute units (8 x V 128256 top-p, draws: parts of 8192 42 us, 16384 47, 32768 62; 64 rows 70 with 16384, 64 with 32768)
    const long long least = std::max((a->vocab * rows + 255) / 256, (a->vocab + TP_MAX_PARTS - 1LL) / TP_MAX_PARTS);
    return (int)((least + TP_PART - 1) / TP_PART * TP_PART);
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
    return check(a) == PS_OK && part_of(a) ? a256((size_t)a->batch * a->rows * sizeof(Work)) : 0;
}

extern "C" int ps_target_probs(const ps_target_probs_args* a, void* stream) {
    const int st = check(a);
    if (st != PS_OK) return st;
    if (!a->logits || (!a->probs && !a->ids) || (a->ids && !a->r) || (a->id_probs && !a->ids)) return PS_ERR_NULL;
    if ((uintptr_t)a->logits & (a->dtype == PS_BF16 ? 1 : 3)) return PS_ERR_UNSUPPORTED;
    if (!aligned4(a->temperature) || !aligned4(a->top_k) || !aligned4(a->top_p) || !aligned4(a->min_p) || !aligned4(a->r) || !aligned4(a->probs) ||
        !aligned4(a->ids) || !aligned4(a->id_probs)) return PS_ERR_UNSUPPORTED;
    const size_t need = ps_target_probs_workspace_bytes(a);
    if (need && !a->workspace) return PS_ERR_NULL;
    if (need && (a->workspace_bytes < need || ((uintptr_t)a->workspace & 255))) return PS_ERR_WORKSPACE;
    TpParams P = {};
    P.logits = (const char*)a->logits; P.temperature = a->temperature; P.top_k = a->top_k; P.top_p = a->top_p; P.min_p = a->min_p; P.r = a->r;
    const int part = part_of(a);
    P.parts = part ? (a->vocab + part - 1) / part : 1;
    P.part_vecs = part / (a->dtype == PS_BF16 ? 8 : 4);
    P.work = part ? (char*)a->workspace : nullptr;
    P.probs = a->probs; P.ids = a->ids; P.id_probs = a->id_probs; P.rows = a->rows; P.vocab = a->vocab;
    int log = 0;
    while (1 << log < a->vocab) ++log;
    P.frac = std::min(51, 62 - log);
    const int total = a->batch * a->rows;
    if (a->dtype == PS_BF16) go<bf16_t>(P, total, (hipStream_t)stream);
    else go<float>(P, total, (hipStream_t)stream);
    return hipGetLastError() == hipSuccess ? PS_OK : PS_ERR_DEVICE;
}

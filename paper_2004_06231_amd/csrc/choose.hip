// One entry per row of logits, under temperature, top-k, top-p and min-p, from a given uniform.
//
// The entries are ordered by (logit descending, index ascending); each filter keeps a prefix of that order, so what is
// kept is one prefix: the entries whose order key is at least `cut`.  The order key of entry i has the logit's bits, made
// monotone, in its upper half and ~i in its lower half: no two are equal, and the larger comes first.
//
// Weights exp((logit - max) / T) are held as integers of 2^-shift, shift = 61 - ceil(log2 V): at most 2^61 in all, so
// that their sums are exact and the same in whatever order they are formed, by atomics too.  A weight is off by half a unit
// at most, 2^-61 of V times the largest; sums of float64 lose more where V is below 2^10, and no sum of float32 could tell
// the entries of a long row apart: a uniform falls between two of V running sums.
//
// The total of V weights is off by V^2 2^-62 of the largest: less than float32 resolves (2^-24) up to V = 2^19, but a quarter at
// 2^30, where every weight below 2^-32 would be lost.  Rows of more than FIXED_UNIT entries therefore get the unit that
// their own total allows: a launch before the others sums the weights in the coarse units above, which bounds the total by Z, and
// shift = 61 - ceil(log2 Z) then holds all of them: V weights are off by V 2^-60 of their total, 2^-30 at 2^30 entries.  (Kept ones
// of the total that is kept: n of them are off by n 2^-60 Z, and Z is at most their total and V times the least of them.)
#include "device_common.hpp"
#include "routing.hpp"

namespace einet_impl {

namespace {

typedef unsigned long long u64;

constexpr int FIXED_UNIT = 1 << 19;                              // entries up to which one unit does for every row

// ------------------------------------------------------------------------------------------------ keys and weights

// A logit's key: its bits, made monotone, without the low bits that a 16-bit type leaves empty; 0 for an entry that is
// left out (-inf, NaN).
template <class T> constexpr int KEY_SHIFT = 0;
template <> constexpr int KEY_SHIFT<__bf16> = 16;
template <> constexpr int KEY_SHIFT<_Float16> = 13;

template <class T>
__device__ __forceinline__ uint32_t logit_key(float v) {
    uint32_t b = __builtin_bit_cast(uint32_t, v);
    if (v == 0.f) b = 0u;                                        // -0 and 0 are equal
    const uint32_t k = ((b >> 31) ? ~b : b | 0x80000000u) >> KEY_SHIFT<T>;
    return v > -INFINITY ? k : 0u;
}
template <class T>
__device__ __forceinline__ float key_logit(uint32_t k) {
    constexpr int S = KEY_SHIFT<T>;
    const uint32_t b = k << S;
    return __builtin_bit_cast(float, (b >> 31) ? b & 0x7fffffffu : ~(b | ((1u << S) - 1u)));
}
__device__ __forceinline__ u64 order_key(uint32_t k, int i) { return ((u64)k << 32) | (uint32_t)~i; }

struct RowSettings {
    float t, inv_t;              // T and 1 / T in float32, for the bins
    double log2e_t;              // log2(e) / T
    int top_k;
    double top_p, min_p, u;
    bool greedy;
};
__device__ __forceinline__ RowSettings row_settings(const ChooseArgs& a, int row) {
    const float p = a.top_p.p ? a.top_p.p[row] : a.top_p.v, mp = a.min_p.p ? a.min_p.p[row] : a.min_p.v, u = a.u[row];
    RowSettings s;
    if (a.temperature.p) {
        s.t = a.temperature.p[row];
        s.inv_t = 1.f / s.t;
        s.log2e_t = 1.4426950408889634074 / (double)s.t;
    } else {
        s.t = a.temperature.v;
        s.inv_t = a.inv_t;                                       // (divided once, by the host)
        s.log2e_t = a.log2e_t;
    }
    s.greedy = !(s.t > 0.f);
    s.top_k = a.top_k.p ? a.top_k.p[row] : a.top_k.v;
    s.top_p = p >= 0.f ? (double)p : p < 0.f ? 0.0 : 1.0;       // (NaN: off)
    s.min_p = mp > 0.f ? fmin((double)mp, 1.0) : 0.0;
    s.u = u > 0.f ? (double)u : 0.0;
    return s;
}

// 2^y in units of 2^-shift, shift <= 61, rounded to the nearest, for y <= 0 (0 for NaN).  2^y = 2^n 2^f with n the nearest
// integer: the series of 2^f = exp(f ln 2) to the 12th power is good to 0.347^13 / 13! = 1.7e-16.  Added to 2 its last place
// is 2^-51, whole.  (The coefficients are kept in scalar registers: as literals each takes two moves before its
// multiplication.)
__device__ __forceinline__ double scalar_constant(double c) {
    asm("" : "+s"(c));
    return c;
}
struct Exp2Series {
    double c[12];
    __device__ __forceinline__ Exp2Series() {
        constexpr double L = 0.69314718055994530942;
        double term = 1.0;
#pragma unroll
        for (int i = 1; i <= 12; ++i) {
            term = term * L / i;
            c[i - 1] = scalar_constant(term);
        }
    }
};
__device__ __forceinline__ u64 exp2_fixed(double y, int shift, const Exp2Series& series) {
    y = fmax(y, -128.0);
    const double n = rint(y), f = y - n;
    double p = series.c[11];
#pragma unroll
    for (int i = 10; i >= 0; --i) p = fma(p, f, series.c[i]);
    p = fma(p, f, 1.0);
    const u64 whole = (__builtin_bit_cast(u64, p + 2.0) & 0xfffffffffffffull) << 10;      // p * 2^61
    const int down = min(61 - shift - (int)n, 63);               // (63: at most a quarter of a unit, which gives 0)
    return (whole + ((1ull << down) >> 1)) >> down;
}

// log x for a positive, normal x: x = 2^e m with m between sqrt(1/2) and sqrt(2), log m = 2 atanh r with r = (m - 1) / (m + 1),
// |r| <= 0.172: of the series in r^2 the terms up to r^19 are good to 2 * 0.172^21 / 21 = 8e-18.
__device__ __forceinline__ double log_of(double x) {
    const u64 b = __builtin_bit_cast(u64, x);
    int e = (int)(b >> 52) - 1023;
    double m = __builtin_bit_cast(double, (b & 0xfffffffffffffull) | 0x3ff0000000000000ull);
    if (m > 1.41421356237309505) m *= 0.5, e += 1;
    const double r = (m - 1.0) / (m + 1.0), q = r * r;
    double s = 1.0 / 19.0;
#pragma unroll
    for (int i = 17; i >= 1; i -= 2) s = fma(s, q, 1.0 / i);
    return fma((double)e, 0.69314718055994530942, 2.0 * r * s);
}

// What the weights of a row are computed from.
template <class T>
struct RowWeights {
    uint32_t kmax;
    float m;                     // the largest logit
    double log2e_t;
    int shift;
    // (a NaN has no weight; next to an entry at +inf the others are infinitely far)
    __device__ __forceinline__ double exponent(float v) const { return v == m ? 0.0 : ((double)v - (double)m) * log2e_t; }
    __device__ __forceinline__ u64 operator()(float v, const Exp2Series& series = Exp2Series()) const {
        return exp2_fixed(exponent(v), shift, series);
    }
    __device__ __forceinline__ u64 of_key(uint32_t k) const { return (*this)(key_logit<T>(k)); }
    __device__ __forceinline__ float log_share(float v, u64 total) const {
        return (float)(exponent(v) * 0.69314718055994530942 - log_of(ldexp((double)total, -shift)));
    }
    // the least weight that min_p keeps
    __device__ __forceinline__ u64 least(double min_p) const { return __double2ull_ru(min_p * (double)(1ull << shift)); }
};

// the first whole number above which lies a running sum that exceeds u * total
__device__ __forceinline__ u64 target_of(double u, u64 total) {
    const double t = u * (double)total;
    return t >= (double)total ? total - 1 : min((u64)t, total - 1);
}

// the mass that the entries kept by top_p reach, 1 .. total
__device__ __forceinline__ u64 mass_of(double top_p, u64 total) { return max((u64)1, __double2ull_ru(top_p * (double)total)); }

// N consecutive entries of a row, of which the first `count` exist (the others are -inf)
template <class T, int N>
__device__ __forceinline__ void load_logits(const T* x, int count, float (&v)[N]) {
    struct Pack { T v[N]; };
    if (count >= N) {
        const Pack q = load_bytes<Pack>(x);
#pragma unroll
        for (int c = 0; c < N; ++c) v[c] = (float)q.v[c];
    } else {
#pragma unroll
        for (int c = 0; c < N; ++c) v[c] = c < count ? (float)x[c] : -INFINITY;
    }
}

// ------------------------------------------------------------------------------------------- across the lanes of a wave

// Row shifts and broadcasts of the data-parallel primitives: after the four shifts every row of 16 lanes has its running
// results, the broadcasts add the last lane of the rows before.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xf, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 dpp(u64 v) {
    return ((u64)dpp<CTRL, ROWS>((uint32_t)(v >> 32)) << 32) | dpp<CTRL, ROWS>((uint32_t)v);
}
struct OpAdd {
    template <class V> __device__ V operator()(V a, V b) const { return a + b; }
};
struct OpMax {
    template <class V> __device__ V operator()(V a, V b) const { return a > b ? a : b; }
};
// running results over the lanes, each lane's own included; 0 is the neutral element
template <class V, class Op>
__device__ __forceinline__ V wave_scan(V v, Op op) {
    v = op(v, dpp<0x111, 0xf>(v));
    v = op(v, dpp<0x112, 0xf>(v));
    v = op(v, dpp<0x114, 0xf>(v));
    v = op(v, dpp<0x118, 0xf>(v));
    v = op(v, dpp<0x142, 0xa>(v));
    v = op(v, dpp<0x143, 0xc>(v));
    return v;
}
__device__ __forceinline__ uint32_t lane_value(uint32_t v, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); }
__device__ __forceinline__ u64 lane_value(u64 v, int lane) {
    return ((u64)lane_value((uint32_t)(v >> 32), lane) << 32) | lane_value((uint32_t)v, lane);
}
template <class V, class Op>
__device__ __forceinline__ V wave_reduce(V v, Op op) { return lane_value(wave_scan(v, op), 63); }

// ----------------------------------------------------------------------------------------------- a wave for every row
//
// Rows of up to 1024 entries stay in the registers of one wave: group g, lane l, place c is entry (g * 64 + l) * VEC + c.
// A cut is found by halving the range of keys: the entries above the middle are counted by ballots, their weights summed
// over the lanes.  The vector ALU bounds it: 50176 rows of 256 (51 MB) take 30 us without filters, 46 with top-k, 63 with
// top-p, some 700 instructions for a row, of which the float64 exponentials are 120 and a halving 28.  (A workgroup with bins for
// every row: 8192 rows of 500 45 us instead of 10, with top-p 90 instead of 21.)
template <class T, int VEC, int GROUPS>
__global__ __launch_bounds__(256) void k_choose_wave(ChooseArgs a, int shift) {
    constexpr int E = VEC * GROUPS;
    const int row = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)), lane = threadIdx.x & 63, V = a.V;
    if (row >= a.B) return;
    const T* const x = static_cast<const T*>(a.logits) + row * a.stride;
    const RowSettings st = row_settings(a, row);
    float v[E];
    uint32_t k[E];
    uint32_t best = 0;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        float part[VEC];
        const int i0 = (g * 64 + lane) * VEC;
        load_logits<T, VEC>(x + i0, V - i0, part);
#pragma unroll
        for (int c = 0; c < VEC; ++c) {
            v[g * VEC + c] = part[c];
            k[g * VEC + c] = logit_key<T>(part[c]);
            best = max(best, k[g * VEC + c]);
        }
    }
    const uint32_t kmax = wave_reduce(best, OpMax{});
    auto index_of = [&](int e) { return ((e / VEC) * 64 + lane) * VEC + e % VEC; };
    if (kmax == 0u || st.greedy) {
        uint32_t first = 0;                                      // (the lowest index as the largest complement)
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (kmax && k[e] == kmax) first = max(first, ~(uint32_t)index_of(e));
        first = wave_reduce(first, OpMax{});
        if (lane == 0) {
            a.index[row] = kmax ? (int)~first : -1;
            if (a.logq) a.logq[row] = kmax ? 0.f : -INFINITY;
        }
        return;
    }
    const RowWeights<T> weight{kmax, key_logit<T>(kmax), st.log2e_t, shift};
    u64 w[E];
    {
        const Exp2Series series;
#pragma unroll
        for (int e = 0; e < E; ++e) w[e] = weight(v[e], series);
    }
    // entries of key t beyond the first `keep` of them go, and all below t
    auto cut_at = [&](uint32_t t, int keep) {
        int before = 0;
        const u64 lower = (1ull << lane) - 1;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            int rank = before;
#pragma unroll
            for (int c = 0; c < VEC; ++c) {
                const u64 tied = __ballot(k[g * VEC + c] == t);
                rank += __popcll(tied & lower);
                before += __popcll(tied);
            }
#pragma unroll
            for (int c = 0; c < VEC; ++c) {
                const uint32_t kc = k[g * VEC + c];
                const bool tie = kc == t, out = kc < t || (tie && rank >= keep);
                rank += tie;
                if (out) k[g * VEC + c] = 0u, w[g * VEC + c] = 0;
            }
        }
    };
    auto count_from = [&](uint32_t t) {
        int n = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) n += __popcll(__ballot(k[e] >= t));
        return n;
    };
    auto mass_from = [&](uint32_t t) {
        u64 s = 0;
#pragma unroll
        for (int e = 0; e < E; ++e) s += k[e] >= t ? w[e] : 0;
        return wave_reduce(s, OpAdd{});
    };
    if (st.top_k > 0 && st.top_k < V) {
        uint32_t lo = 1, hi = kmax + 1;                          // at least top_k entries from lo on, fewer from hi on
        int n_lo = count_from(1), n_hi = 0;
        if (n_lo > st.top_k) {
            while (hi - lo > 1 && n_lo != st.top_k) {
                const uint32_t mid = lo + (hi - lo) / 2;
                const int n = count_from(mid);
                if (n >= st.top_k) lo = mid, n_lo = n;
                else hi = mid, n_hi = n;
            }
            if (n_lo == st.top_k) {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (k[e] < lo) k[e] = 0u, w[e] = 0;
            } else {
                cut_at(lo, st.top_k - n_hi);
            }
        }
    }
    if (st.top_p < 1.0) {
        // Sums of the weights' upper halves (2^31 units) decide where they can: what the lower halves add is below V of them.
        uint32_t upper[E];
#pragma unroll
        for (int e = 0; e < E; ++e) upper[e] = (uint32_t)(w[e] >> 31);
        const u64 mass = mass_of(st.top_p, mass_from(1));
        uint32_t lo = 1, hi = kmax + 1;                          // at least `mass` from lo on, less from hi on
        int n_lo = count_from(1), n_hi = 0;
        float guess = 2.f;                                       // the cut's distance from the largest in units of T, as a start
        for (int step = 0; hi - lo > 1 && n_lo - n_hi > 1; ++step) {
            uint32_t mid = lo + (hi - lo) / 2;
            if (step < 2) {
                const uint32_t near = __builtin_amdgcn_readfirstlane((int)logit_key<T>(weight.m - guess * st.t));
                if (near > lo && near < hi) mid = near;
            }
            uint32_t part = 0;
            int n = 0;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const bool in = k[e] >= mid;
                part += in ? upper[e] : 0u;
                n += __popcll(__ballot(in));
            }
            const u64 sum = wave_reduce(part, OpAdd{});
            const bool enough = (sum << 31) >= mass || (((sum + V) << 31) > mass && mass_from(mid) >= mass);
            if (enough) lo = mid, n_lo = n, guess = 0.5f;
            else hi = mid, n_hi = n, guess = 8.f;
        }
        if (n_lo - n_hi <= 1) {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (k[e] < lo) k[e] = 0u, w[e] = 0;
        } else {
            // several of one key: as many as it takes to reach the mass
            const u64 each = weight.of_key(lo), missing = mass - mass_from(hi);
            cut_at(lo, (int)((missing + each - 1) / each));
        }
    }
    if (st.min_p > 0.0) {
        const u64 least = weight.least(st.min_p);
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (w[e] < least) w[e] = 0;
    }
    u64 run[GROUPS], total = 0;                                  // running sums at the end of every lane's places
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        u64 s = 0;
#pragma unroll
        for (int c = 0; c < VEC; ++c) s += w[g * VEC + c];
        run[g] = wave_scan(s, OpAdd{}) + total;
        total = lane_value(run[g], 63);
    }
    const u64 target = target_of(st.u, total);
    bool done = false;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        const u64 above = __ballot(run[g] > target);
        if (!done && above) {
            done = true;
            if (lane == __ffsll(above) - 1) {
                u64 s = run[g];
                int at = VEC - 1;
#pragma unroll
                for (int c = VEC - 1; c > 0; --c) {
                    s -= w[g * VEC + c];                         // the running sum at place c - 1
                    if (s > target) at = c - 1;
                }
                uint32_t key = 0;
#pragma unroll
                for (int c = 0; c < VEC; ++c)
                    if (c == at) key = k[g * VEC + c];
                a.index[row] = (g * 64 + lane) * VEC + at;
                if (a.logq) a.logq[row] = weight.log_share(key_logit<T>(key), total);
            }
        }
    }
}

// ------------------------------------------------------------------------------------------ a workgroup for every row
//
// Wave w of the workgroup has a contiguous stretch of the row, in groups of 256 entries (four to a lane).  GROUPS > 0: the
// logits of the stretch stay in registers; 0: they are read again by every pass.
//
// A cut is found from the histogram of the entries over their distance from the largest logit in units of T (BINS equal bins
// to 32 units; their order is the entries' order): the bin that the cut lies in holds few entries of an ordinary row, and a
// radix search over the order keys of that bin's entries finds the very entry.  One row of 4000 takes 6 us without filters and
// 16 with all, most of it the latency of the some twenty steps between barriers; 4096 rows of 2048 (34 MB) 33 and 77 us.
template <class T, int NT, int GROUPS>
struct RowLogits {
    const T* x;
    int V, first, groups;        // of this thread's wave: its first group, the number of its groups
    float v[GROUPS > 0 ? GROUPS * 4 : 1];
    __device__ __forceinline__ void init(const T* row, int n) {
        x = row;
        V = n;
        const int wave = threadIdx.x >> 6;
        if constexpr (GROUPS > 0) {
            groups = GROUPS;
            first = wave * GROUPS;
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                float part[4];
                load_logits<T, 4>(x + index(g), V - index(g), part);
#pragma unroll
                for (int c = 0; c < 4; ++c) v[g * 4 + c] = part[c];
            }
        } else {
            groups = (V + NT * 4 - 1) / (NT * 4);
            first = wave * groups;
        }
    }
    __device__ __forceinline__ int index(int g) const { return (first + g) * 256 + (int)(threadIdx.x & 63) * 4; }
    // f(index, logit) for the four entries of a group
    template <class F>
    __device__ __forceinline__ void group(int g, F&& f) const {
        float part[4];
        load_logits<T, 4>(x + index(g), V - index(g), part);
#pragma unroll
        for (int c = 0; c < 4; ++c) f(index(g) + c, part[c]);
    }
    template <class F>
    __device__ __forceinline__ void each(F&& f) const {
        if constexpr (GROUPS > 0) {
#pragma unroll
            for (int g = 0; g < GROUPS; ++g)
#pragma unroll
                for (int c = 0; c < 4; ++c) f(index(g) + c, v[g * 4 + c]);
        } else {
            int g = 0;
            for (; g + 4 <= groups; g += 4) {                    // (four loads in flight)
                float part[4][4];
#pragma unroll
                for (int q = 0; q < 4; ++q) load_logits<T, 4>(x + index(g + q), V - index(g + q), part[q]);
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int c = 0; c < 4; ++c) f(index(g + q) + c, part[q][c]);
            }
            for (; g < groups; ++g) group(g, f);
        }
    }
};

// Bins per unit of the logits: over BIN_RANGE T (a weight beyond is below 2e-14 of the largest), or over the range of the
// row's logits where that is less, so that a flat row fills its bins too.
constexpr float BIN_RANGE = 32.f;
__device__ __forceinline__ float bins_per_unit(float highest, float lowest, float inv_t, int bins) {
    const float range = highest - lowest, by_t = inv_t * ((float)bins / BIN_RANGE);
    return range > 0.f ? fmaxf(by_t, (float)bins / range) : by_t;
}

template <int NT>
struct ChooseShared {
    static constexpr int BINS = 2 * NT;
    u64 mass[BINS];
    uint32_t count[BINS];
    u64 digit[256];
    uint32_t digit_count[256];
    u64 tmp[NT / 64], tmp2[NT / 64];
    u64 found[4];
};

template <int NT, class V, class Op>
__device__ __forceinline__ V block_reduce(V v, u64* tmp, Op op) {
    v = wave_reduce(v, op);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = v;
    __syncthreads();
    v = (V)tmp[0];
    for (int w = 1; w < NT / 64; ++w) v = op(v, (V)tmp[w]);
    return v;
}
// running sums over the threads, each thread's own included, and their total
template <int NT>
__device__ __forceinline__ u64 block_scan(u64 v, u64* tmp, u64& total) {
    v = wave_scan(v, OpAdd{});
    __syncthreads();
    if ((threadIdx.x & 63) == 63) tmp[threadIdx.x >> 6] = v;
    __syncthreads();
    total = 0;
    for (int w = 0; w < NT / 64; ++w) {
        if (w == (int)(threadIdx.x >> 6)) v += total;
        total += tmp[w];
    }
    return v;
}

// The bin in which the running sum of `bins` reaches target (1 .. their sum), and what is missing at its start.
template <int NT, class C>
__device__ __forceinline__ void find_bin(const C* bins, u64 target, ChooseShared<NT>& sh, int& bin, u64& missing) {
    const int b = 2 * threadIdx.x;
    const u64 v0 = bins[b], v1 = bins[b + 1];
    u64 total;
    const u64 run = block_scan<NT>(v0 + v1, sh.tmp, total), before = run - v0 - v1;
    if (before < target && target <= run) {
        const bool second = before + v0 < target;
        sh.found[0] = second ? b + 1 : b;
        sh.found[1] = target - (second ? before + v0 : before);
    }
    __syncthreads();
    bin = (int)sh.found[0];
    missing = sh.found[1];
}

// Of the entries that each(f) passes to f(order key, value): the one, in descending order, at which the running sum of the
// values reaches target.  A byte of the order key after the other, from the first in which the entries differ, until one
// entry is left.
template <int NT, class Each>
__device__ __forceinline__ u64 find_entry(Each&& each, u64 target, ChooseShared<NT>& sh) {
    u64 hi = 0, lo = 0;
    each([&](u64 o, u64) { hi = max(hi, o), lo = max(lo, ~o); });
    hi = wave_reduce(hi, OpMax{});
    lo = wave_reduce(lo, OpMax{});
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh.tmp[threadIdx.x >> 6] = hi, sh.tmp2[threadIdx.x >> 6] = lo;
    __syncthreads();
    for (int w = 0; w < NT / 64; ++w) hi = max(hi, sh.tmp[w]), lo = max(lo, sh.tmp2[w]);
    lo = ~lo;
    if (hi == lo) return hi;
    int top = 64 - __clzll(hi ^ lo);                             // bits in which they differ
    u64 prefix = top < 64 ? hi >> top : 0;
    while (top > 0) {
        const int shift = max(0, top - 8), n = 1 << (top - shift);
        __syncthreads();
        if (threadIdx.x < 256) sh.digit[threadIdx.x] = 0, sh.digit_count[threadIdx.x] = 0;
        __syncthreads();
        each([&](u64 o, u64 v) {
            if ((top < 64 ? o >> top : 0) == prefix && v) {
                atomicAdd(&sh.digit[(o >> shift) & (n - 1)], v);
                atomicAdd(&sh.digit_count[(o >> shift) & (n - 1)], 1u);
            }
        });
        __syncthreads();
        if (threadIdx.x < 64) {                                  // from the largest digit down, four to a lane
            u64 v[4], sum = 0;
#pragma unroll
            for (int c = 0; c < 4; ++c) v[c] = sh.digit[255 - (4 * threadIdx.x + c)], sum += v[c];
            u64 before = wave_scan(sum, OpAdd{}) - sum;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                if (before < target && target <= before + v[c]) {
                    const int d = 255 - (4 * threadIdx.x + c);
                    sh.found[0] = d;
                    sh.found[1] = target - before;
                    sh.found[2] = sh.digit_count[d];
                }
                before += v[c];
            }
        }
        __syncthreads();
        prefix = (prefix << (top - shift)) | sh.found[0];
        target = sh.found[1];
        top = shift;
        if (sh.found[2] == 1 && top > 0) {
            each([&](u64 o, u64 v) {
                if ((o >> top) == prefix && v) sh.found[3] = o;
            });
            __syncthreads();
            return sh.found[3];
        }
    }
    return prefix;
}

// The bin of a logit: its distance from the largest times bins_per_unit.
template <class T>
__device__ __forceinline__ int bin_of(const RowWeights<T>& weight, float v, float per_bin, int bins) {
    const float q = (weight.m - v) * per_bin;
    return v == weight.m ? 0 : q < (float)(bins - 1) ? (int)q : bins - 1;
}

// The largest order key of the entries and the complement of the lowest key, over the workgroup (0 without an entry).
template <class T, int NT, class Row>
__device__ __forceinline__ void row_ends(const Row& row, int origin, u64* tmp, u64* tmp2, u64& best, uint32_t& low) {
    best = 0;
    low = 0;
    row.each([&](int i, float v) {
        const uint32_t k = logit_key<T>(v);
        best = max(best, k ? order_key(k, origin + i) : 0);
        low = max(low, k ? ~k : 0u);
    });
    best = wave_reduce(best, OpMax{});
    low = wave_reduce(low, OpMax{});
    __syncthreads();
    if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = best, tmp2[threadIdx.x >> 6] = low;
    __syncthreads();
    for (int w = 0; w < NT / 64; ++w) best = max(best, tmp[w]), low = max(low, (uint32_t)tmp2[w]);
}

__device__ __forceinline__ void write_choice(const ChooseArgs& a, int row, int index, float logq) {
    a.index[row] = index;
    if (a.logq) a.logq[row] = logq;
}

// The choice among the entries of `keys` (those of the row from `origin` on), of which kept(index, logit) is the kept weight:
// the first at which the running sum, `before` at the start, exceeds target.  total: of all kept weights of the row.
template <class T, int NT, int GROUPS, class Kept>
__device__ __forceinline__ void choose_among(const ChooseArgs& a, int row, const RowLogits<T, NT, GROUPS>& keys, int origin, u64 before,
                                             u64 target, u64 total, u64 wave_sum, u64 wave_end, const RowWeights<T>& weight,
                                             Kept&& kept) {
    // the wave in whose stretch that is goes through its groups
    u64 run = before + wave_end - wave_sum;
    if (target < run || target >= run + wave_sum) return;
    for (int g = 0; g < keys.groups; ++g) {
        u64 w[4], sum = 0;
        float v4[4];
        int c = 0;
        keys.group(g, [&](int i, float v) {
            v4[c] = v;
            w[c] = kept(i, v);
            sum += w[c];
            ++c;
        });
        const u64 ends = wave_scan(sum, OpAdd{}) + run;
        const u64 above = __ballot(ends > target);
        if (above) {
            if ((int)(threadIdx.x & 63) == __ffsll(above) - 1) {
                u64 s = ends;
                int at = 3;
#pragma unroll
                for (int q = 3; q > 0; --q) {
                    s -= w[q];                                   // the running sum at place q - 1
                    if (s > target) at = q - 1;
                }
                const float v = at == 0 ? v4[0] : at == 1 ? v4[1] : at == 2 ? v4[2] : v4[3];
                write_choice(a, row, origin + keys.index(g) + at, weight.log_share(v, total));
            }
            return;
        }
        run = lane_value(ends, 63);
    }
}

template <class T, int NT, int GROUPS>
__device__ __forceinline__ void choose_block(const ChooseArgs& a, int row, int shift, ChooseShared<NT>& sh) {
    constexpr int BINS = ChooseShared<NT>::BINS;
    const int tid = threadIdx.x, V = a.V;
    const RowSettings st = row_settings(a, row);
    RowLogits<T, NT, GROUPS> keys;
    keys.init(static_cast<const T*>(a.logits) + row * a.stride, V);
    u64 best;
    uint32_t low;
    row_ends<T, NT>(keys, 0, sh.tmp, sh.tmp2, best, low);
    const uint32_t kmax = (uint32_t)(best >> 32);
    if (kmax == 0u || st.greedy) {
        if (tid == 0) write_choice(a, row, kmax ? (int)~(uint32_t)best : -1, kmax ? 0.f : -INFINITY);
        return;
    }
    const RowWeights<T> weight{kmax, key_logit<T>(kmax), st.log2e_t, shift};
    const float per_bin = bins_per_unit(weight.m, key_logit<T>(~low), st.inv_t, BINS);
    auto bin = [&](float v) { return bin_of(weight, v, per_bin, BINS); };
    u64 cut = 1ull << 32;                                        // everything that is not left out
    const bool by_count = st.top_k > 0 && st.top_k < V, by_mass = st.top_p < 1.0;
    if (by_count || by_mass) {
        for (int b = tid; b < BINS; b += NT) sh.count[b] = 0, sh.mass[b] = 0;
        __syncthreads();
        keys.each([&](int, float v) {
            if (!(v > -INFINITY)) return;
            const int b = bin(v);
            if (by_count) atomicAdd(&sh.count[b], 1u);
            if (by_mass) atomicAdd(&sh.mass[b], weight(v));
        });
        __syncthreads();
        // entries of a bin from the cut on, with their values
        auto of_bin = [&](int at, auto value) {
            return [&, at, value](auto f) {
                keys.each([&](int i, float v) {
                    if (!(v > -INFINITY) || bin(v) != at) return;
                    const u64 o = order_key(logit_key<T>(v), i);
                    if (o >= cut) f(o, value(v));
                });
            };
        };
        int at;
        u64 missing, total;
        if (by_count) {
            block_scan<NT>((u64)sh.count[2 * tid] + sh.count[2 * tid + 1], sh.tmp, total);
            if (total > (u64)st.top_k) {
                find_bin<NT>(sh.count, (u64)st.top_k, sh, at, missing);
                cut = find_entry<NT>(of_bin(at, [](float) -> u64 { return 1; }), missing, sh);
                if (by_mass) {
                    // the mass of that bin is what is kept of it, that of the bins behind it none
                    u64 rest = 0;
                    of_bin(at, weight)([&](u64, u64 v) { rest += v; });
                    rest = block_reduce<NT>(rest, sh.tmp, OpAdd{});
                    for (int b = tid; b < BINS; b += NT)
                        if (b >= at) sh.mass[b] = b == at ? rest : 0;
                    __syncthreads();
                }
            }
        }
        if (by_mass) {
            block_scan<NT>(sh.mass[2 * tid] + sh.mass[2 * tid + 1], sh.tmp, total);
            // kept: what has less than top_p of the total before it; the last one's own weight reaches that mass
            find_bin<NT>(sh.mass, mass_of(st.top_p, total), sh, at, missing);
            cut = find_entry<NT>(of_bin(at, weight), missing, sh);
        }
    }
    const u64 least = weight.least(st.min_p);
    auto kept = [&](int i, float v) {
        if (!(v > -INFINITY) || order_key(logit_key<T>(v), i) < cut) return (u64)0;
        const u64 w = weight(v);
        return w < least ? (u64)0 : w;
    };
    u64 mine = 0, total;
    keys.each([&](int i, float v) { mine += kept(i, v); });
    const u64 wave_sum = wave_reduce(mine, OpAdd{});
    const u64 end = lane_value(block_scan<NT>((tid & 63) == 63 ? wave_sum : 0, sh.tmp, total), 63);
    choose_among(a, row, keys, 0, 0, target_of(st.u, total), total, wave_sum, end, weight, kept);
}

template <class T, int NT, int GROUPS>
__global__ __launch_bounds__(NT, 4) void k_choose_block(ChooseArgs a, int shift) {
    __shared__ ChooseShared<NT> sh;
    choose_block<T, NT, GROUPS>(a, blockIdx.x, shift, sh);
}

// ------------------------------------------------------------------------------------ several workgroups for every row
//
// Long rows: `parts` workgroups of SPLIT_THREADS for every row, each with a stretch of `per` entries, in four launches (one
// less where no filter is on, one more for units of the row's own) for every batch of SPLIT_ROWS rows.
//   max      the largest order key of every part
//   scale    the weights of every part summed in coarse units, for rows of more than FIXED_UNIT entries
//   bins     the row's histogram over the distance from the largest logit, summed up by integer atomics (exact, in any
//            order); rows without top_k and top_p: the kept mass of every part instead
//   collect  the bin that the cut lies in, from the row's histogram.  With top_k: all entries up to that bin go to a list,
//            at most LIST of them.  With top_p alone: that bin's entries do, and every part's kept mass in the bins before it
//            is written down.
//   finish   one workgroup per row finds the cut among the list's entries, the choice among them (top_k) or in the part in
//            which the running sum exceeds the target.  A row whose list did not hold its entries (more than LIST in all or
//            PART_LIST of one part: nearly equal ones, or a large top_k of few parts, from some 1500 on of two) and one with
//            top_k above LIST are done as a workgroup for every row does it: right, but slow.
// One row of 131077 takes 14 us without filters and 25 with all, all of it launches and their latency; 64 rows (34 MB) 34 us (9
// largest keys, 16 masses, 10 finish) and 43 us (9 largest keys, 9 bins, 14 list, 11 finish); one row of 2^20 35 and 47 us, of which
// its own units cost 9 us.
constexpr int SPLIT_THREADS = 256, SPLIT_BINS = 2 * SPLIT_THREADS, LIST = 4096, PART_LIST = 1024, FINISH_THREADS = 256;
constexpr int SPLIT_PARTS = 64;                                  // at most (a lane each)
constexpr int STRETCHES = SPLIT_THREADS / 64;                    // of a part: its waves'

struct SplitRows {
    int parts, per;              // per: a multiple of 4 * SPLIT_THREADS
    u64* best;                   // [B][parts]
    uint32_t* low;               // [B][parts] complements of the lowest keys
    u64* coarse;                 // [B][parts] sums of the weights in coarse units, or nullptr (up to FIXED_UNIT entries)
    u64* mass;                   // [B][parts][STRETCHES] kept masses
    u64* bin_mass;               // [B][SPLIT_BINS]
    uint32_t* bin_count;         // [B][SPLIT_BINS]
    uint32_t* listed;            // [B] entries of the list, also those that it did not hold
    u64* list;                   // [B][LIST] order keys
};

enum SplitMode { SPLIT_NONE, SPLIT_ALL, SPLIT_COUNT, SPLIT_MASS, SPLIT_BLOCK };

// What a row's workgroups agree on from its settings and the largest keys of its parts.  OWN: the row has units of its own.
template <class T, bool OWN>
struct SplitRow {
    RowSettings st;
    u64 best;
    bool done;                   // no entry, or the largest one
    RowWeights<T> weight;
    float per_bin;
    __device__ __forceinline__ SplitRow(const ChooseArgs& a, const SplitRows& sp, int row, int shift) {
        st = row_settings(a, row);
        const int lane = threadIdx.x & 63;
        best = wave_reduce(lane < sp.parts ? sp.best[(size_t)row * sp.parts + lane] : 0, OpMax{});
        const uint32_t low = wave_reduce(lane < sp.parts ? sp.low[(size_t)row * sp.parts + lane] : 0u, OpMax{});
        const uint32_t kmax = (uint32_t)(best >> 32);
        done = kmax == 0u || st.greedy;
        if constexpr (OWN)
            if (!done) {
                // every weight is at most half a coarse unit above what it counts for: total <= (sum + V / 2) units, and one more
                const u64 sum = wave_reduce(lane < sp.parts ? sp.coarse[(size_t)row * sp.parts + lane] : 0, OpAdd{});
                shift += __clzll(sum + a.V / 2) - 3;             // 61 - ceil(log2(sum + V / 2 + 1))
            }
        weight = RowWeights<T>{kmax, key_logit<T>(kmax), st.log2e_t, shift};
        per_bin = bins_per_unit(weight.m, key_logit<T>(~low), st.inv_t, SPLIT_BINS);
    }
    __device__ __forceinline__ bool by_count(int V) const { return st.top_k > 0 && st.top_k < V; }
    __device__ __forceinline__ bool by_mass() const { return st.top_p < 1.0; }
    __device__ __forceinline__ int bin(float v) const { return bin_of(weight, v, per_bin, SPLIT_BINS); }
};

// the part's entries as RowLogits; index 0 of them is entry `origin` of the row
template <class T>
__device__ __forceinline__ int split_part(const ChooseArgs& a, const SplitRows& sp, int row, int part,
                                          RowLogits<T, SPLIT_THREADS, 0>& keys) {
    const int origin = part * sp.per;
    keys.init(static_cast<const T*>(a.logits) + row * a.stride + origin, min(sp.per, a.V - origin));
    keys.groups = sp.per / (4 * SPLIT_THREADS);                  // (of a whole part, also in a shorter last one)
    keys.first = (int)(threadIdx.x >> 6) * keys.groups;
    return origin;
}

template <class T>
__global__ __launch_bounds__(SPLIT_THREADS) void k_choose_split_max(ChooseArgs a, SplitRows sp) {
    __shared__ u64 tmp[SPLIT_THREADS / 64], tmp2[SPLIT_THREADS / 64];
    const int row = blockIdx.x / sp.parts, part = blockIdx.x - row * sp.parts, tid = threadIdx.x;
    for (int b = part * SPLIT_THREADS + tid; b < SPLIT_BINS; b += sp.parts * SPLIT_THREADS) {
        sp.bin_count[(size_t)row * SPLIT_BINS + b] = 0;
        sp.bin_mass[(size_t)row * SPLIT_BINS + b] = 0;
    }
    if (part == 0 && tid == 0) sp.listed[row] = 0;
    RowLogits<T, SPLIT_THREADS, 0> keys;
    const int origin = split_part(a, sp, row, part, keys);
    u64 best;
    uint32_t low;
    row_ends<T, SPLIT_THREADS>(keys, origin, tmp, tmp2, best, low);
    if (tid == 0) sp.best[(size_t)row * sp.parts + part] = best, sp.low[(size_t)row * sp.parts + part] = low;
}

__device__ __forceinline__ void write_stretch(const SplitRows& sp, int row, int part, u64 sum) {
    sum = wave_reduce(sum, OpAdd{});
    if ((threadIdx.x & 63) == 0) sp.mass[((size_t)row * sp.parts + part) * STRETCHES + (threadIdx.x >> 6)] = sum;
}

template <class T>
__global__ __launch_bounds__(SPLIT_THREADS) void k_choose_split_scale(ChooseArgs a, SplitRows sp, int shift) {
    __shared__ u64 tmp[SPLIT_THREADS / 64];
    const int row = blockIdx.x / sp.parts, part = blockIdx.x - row * sp.parts;
    const SplitRow<T, false> r(a, sp, row, shift);               // (the units that the row's length allows)
    if (r.done) return;
    RowLogits<T, SPLIT_THREADS, 0> keys;
    split_part(a, sp, row, part, keys);
    u64 sum = 0;
    keys.each([&](int, float v) { sum += r.weight(v); });
    sum = block_reduce<SPLIT_THREADS>(sum, tmp, OpAdd{});
    if (threadIdx.x == 0) sp.coarse[(size_t)row * sp.parts + part] = sum;
}

template <class T, bool OWN>
__global__ __launch_bounds__(SPLIT_THREADS) void k_choose_split_bins(ChooseArgs a, SplitRows sp, int shift) {
    __shared__ u64 mass[SPLIT_BINS];
    __shared__ uint32_t count[SPLIT_BINS];
    const int row = blockIdx.x / sp.parts, part = blockIdx.x - row * sp.parts, tid = threadIdx.x;
    const SplitRow<T, OWN> r(a, sp, row, shift);
    if (r.done) return;
    RowLogits<T, SPLIT_THREADS, 0> keys;
    split_part(a, sp, row, part, keys);
    const bool by_count = r.by_count(a.V), by_mass = r.by_mass();
    if (!by_count && !by_mass) {
        const u64 least = r.weight.least(r.st.min_p);
        u64 sum = 0;
        keys.each([&](int, float v) {
            const u64 w = r.weight(v);
            sum += w < least ? 0 : w;
        });
        write_stretch(sp, row, part, sum);
        return;
    }
    for (int b = tid; b < SPLIT_BINS; b += SPLIT_THREADS) count[b] = 0, mass[b] = 0;
    __syncthreads();
    // (with top_k the masses are those of the list's entries)
    keys.each([&](int, float v) {
        if (!(v > -INFINITY)) return;
        const int b = r.bin(v);
        if (by_count) atomicAdd(&count[b], 1u);
        else atomicAdd(&mass[b], r.weight(v));
    });
    __syncthreads();
    for (int b = tid; b < SPLIT_BINS; b += SPLIT_THREADS) {
        if (count[b]) atomicAdd(&sp.bin_count[(size_t)row * SPLIT_BINS + b], count[b]);
        if (mass[b]) atomicAdd(&sp.bin_mass[(size_t)row * SPLIT_BINS + b], mass[b]);
    }
}

// The row's mode and the bin that its cut lies in; missing: what is to be reached within that bin (top_p alone).
template <class T, bool OWN>
__device__ __forceinline__ SplitMode split_cut_bin(const ChooseArgs& a, const SplitRows& sp, const SplitRow<T, OWN>& r, int row,
                                                   ChooseShared<SPLIT_THREADS>& sh, int& bin, u64& missing) {
    const int tid = threadIdx.x, b = 2 * tid;
    if (r.done) return SPLIT_NONE;
    if (!r.by_count(a.V) && !r.by_mass()) return SPLIT_ALL;
    u64 total;
    if (r.by_count(a.V)) {
        sh.count[b] = sp.bin_count[(size_t)row * SPLIT_BINS + b];
        sh.count[b + 1] = sp.bin_count[(size_t)row * SPLIT_BINS + b + 1];
        block_scan<SPLIT_THREADS>((u64)sh.count[b] + sh.count[b + 1], sh.tmp, total);
        if (r.st.top_k > LIST) return SPLIT_BLOCK;
        find_bin<SPLIT_THREADS>(sh.count, min((u64)r.st.top_k, total), sh, bin, missing);
        return SPLIT_COUNT;
    }
    sh.mass[b] = sp.bin_mass[(size_t)row * SPLIT_BINS + b];
    sh.mass[b + 1] = sp.bin_mass[(size_t)row * SPLIT_BINS + b + 1];
    block_scan<SPLIT_THREADS>(sh.mass[b] + sh.mass[b + 1], sh.tmp, total);
    find_bin<SPLIT_THREADS>(sh.mass, mass_of(r.st.top_p, total), sh, bin, missing);
    return SPLIT_MASS;
}

template <class T, bool OWN>
__global__ __launch_bounds__(SPLIT_THREADS) void k_choose_split_collect(ChooseArgs a, SplitRows sp, int shift) {
    __shared__ ChooseShared<SPLIT_THREADS> sh;
    __shared__ u64 mine[PART_LIST];                              // the part's entries of the list, in any order
    __shared__ uint32_t n_mine, base;
    const int row = blockIdx.x / sp.parts, part = blockIdx.x - row * sp.parts, tid = threadIdx.x;
    if (tid == 0) n_mine = 0;                                    // (read behind the barriers of split_cut_bin)
    const SplitRow<T, OWN> r(a, sp, row, shift);
    int bin;
    u64 missing;
    const SplitMode mode = split_cut_bin(a, sp, r, row, sh, bin, missing);
    if (mode != SPLIT_COUNT && mode != SPLIT_MASS) return;
    RowLogits<T, SPLIT_THREADS, 0> keys;
    const int origin = split_part(a, sp, row, part, keys);
    const u64 least = r.weight.least(r.st.min_p);
    u64 sum = 0;
    keys.each([&](int i, float v) {
        const int b = v > -INFINITY ? r.bin(v) : SPLIT_BINS;
        const bool take = mode == SPLIT_COUNT ? b <= bin : b == bin;
        if (mode == SPLIT_MASS && b < bin) {
            const u64 w = r.weight(v);
            sum += w < least ? 0 : w;
        }
        if (take) {
            const uint32_t at = atomicAdd(&n_mine, 1u);
            if (at < PART_LIST) mine[at] = order_key(logit_key<T>(v), origin + i);
        }
    });
    __syncthreads();
    const uint32_t n = n_mine;
    if (n > 0) {
        // (more than this part can list are more than the list holds)
        if (tid == 0) base = atomicAdd(&sp.listed[row], n <= PART_LIST ? n : LIST + 1);
        __syncthreads();
        for (uint32_t i = tid; i < min(n, (uint32_t)PART_LIST); i += SPLIT_THREADS)
            if (base + i < LIST) sp.list[(size_t)row * LIST + base + i] = mine[i];
    }
    if (mode == SPLIT_MASS) write_stretch(sp, row, part, sum);
}

template <class T, bool OWN>
__global__ __launch_bounds__(FINISH_THREADS) void k_choose_split_finish(ChooseArgs a, SplitRows sp, int shift) {
    __shared__ ChooseShared<FINISH_THREADS> sh;
    __shared__ u64 list[LIST], stretch[SPLIT_PARTS * STRETCHES];
    const int row = blockIdx.x, tid = threadIdx.x;
    const SplitRow<T, OWN> r(a, sp, row, shift);
    if (r.done) {
        if (tid == 0) write_choice(a, row, r.weight.kmax ? (int)~(uint32_t)r.best : -1, r.weight.kmax ? 0.f : -INFINITY);
        return;
    }
    const bool by_count = r.by_count(a.V), by_mass = r.by_mass();
    const uint32_t listed = by_count || by_mass ? sp.listed[row] : 0;
    if (listed > LIST || (by_count && r.st.top_k > LIST)) {
        choose_block<T, FINISH_THREADS, 0>(a, row, r.weight.shift, sh);
        return;
    }
    for (uint32_t i = tid; i < listed; i += FINISH_THREADS) list[i] = sp.list[(size_t)row * LIST + i];
    const int stretches = sp.parts * STRETCHES, wide = sp.per / STRETCHES;
    for (int i = tid; i < SPLIT_PARTS * STRETCHES; i += FINISH_THREADS)
        stretch[i] = !by_count && i < stretches ? sp.mass[(size_t)row * stretches + i] : 0;
    __syncthreads();
    const u64 least = r.weight.least(r.st.min_p);
    u64 cut = 1ull << 32;
    auto logit = [&](u64 o) { return key_logit<T>((uint32_t)(o >> 32)); };
    auto weight = [&](u64 o) { return r.weight(logit(o)); };
    auto kept = [&](u64 o) {
        const u64 w = o < cut ? 0 : weight(o);
        return w < least ? (u64)0 : w;
    };
    // the list's entries from the cut on, with their values, in the order of `name`
    auto entries = [&](auto name, auto value) {
        return [&, name, value](auto f) {
            for (uint32_t i = tid; i < listed; i += FINISH_THREADS)
                if (list[i] >= cut) f(name(list[i]), value(list[i]));
        };
    };
    auto order = [](u64 o) { return o; };
    auto sum_of = [&](auto value) {
        u64 s = 0;
        entries(order, value)([&](u64, u64 v) { s += v; });
        return block_reduce<FINISH_THREADS>(s, sh.tmp, OpAdd{});
    };
    if (by_count) {
        if (listed > (uint32_t)r.st.top_k)
            cut = find_entry<FINISH_THREADS>(entries(order, [](u64) -> u64 { return 1; }), (u64)r.st.top_k, sh);
        if (by_mass) cut = find_entry<FINISH_THREADS>(entries(order, weight), mass_of(r.st.top_p, sum_of(weight)), sh);
        const u64 total = sum_of(kept), target = target_of(r.st.u, total);
        // (the lower half of an order key is the complement of the index: the largest is the lowest index)
        const u64 at = find_entry<FINISH_THREADS>(entries([](u64 o) { return o & 0xffffffffull; }, kept), target + 1, sh);
        for (uint32_t i = tid; i < listed; i += FINISH_THREADS)
            if ((list[i] & 0xffffffffull) == at)
                write_choice(a, row, (int)~(uint32_t)at, r.weight.log_share(logit(list[i]), total));
        return;
    }
    if (by_mass) {
        // what is missing of the mass in the list's bin: the bins before it hold the rest
        u64 total = 0, before = 0;
        const int bin = r.bin(logit(list[0]));
        for (int b = tid; b < SPLIT_BINS; b += FINISH_THREADS) {
            const u64 v = sp.bin_mass[(size_t)row * SPLIT_BINS + b];
            total += v;
            before += b < bin ? v : 0;
        }
        before = block_reduce<FINISH_THREADS>(before, sh.tmp, OpAdd{});
        total = block_reduce<FINISH_THREADS>(total, sh.tmp, OpAdd{});
        cut = find_entry<FINISH_THREADS>(entries(order, weight), mass_of(r.st.top_p, total) - before, sh);
        for (uint32_t i = tid; i < listed; i += FINISH_THREADS) {
            const u64 w = kept(list[i]);
            if (w) atomicAdd(&stretch[~(uint32_t)list[i] / (uint32_t)wide], w);
        }
        __syncthreads();
    }
    // the stretch in which the running sum exceeds the target
    static_assert(SPLIT_PARTS * STRETCHES == FINISH_THREADS, "a stretch to a thread");
    u64 total;
    const u64 mine = stretch[tid], run = block_scan<FINISH_THREADS>(mine, sh.tmp, total), target = target_of(r.st.u, total);
    if (run - mine <= target && target < run) sh.found[0] = tid, sh.found[1] = run - mine;
    __syncthreads();
    const int origin = (int)sh.found[0] * wide, lane = tid & 63;
    const u64 start = sh.found[1];
    RowLogits<T, FINISH_THREADS, 0> keys;
    keys.init(static_cast<const T*>(a.logits) + row * a.stride + origin, min(wide, a.V - origin));
    auto kept_at = [&](int i, float v) { return v > -INFINITY ? kept(order_key(logit_key<T>(v), origin + i)) : (u64)0; };
    u64 sum = 0, all;
    keys.each([&](int i, float v) { sum += kept_at(i, v); });
    const u64 wave_sum = wave_reduce(sum, OpAdd{});
    const u64 end = lane_value(block_scan<FINISH_THREADS>(lane == 63 ? wave_sum : 0, sh.tmp, all), 63);
    choose_among(a, row, keys, origin, start, target, total, wave_sum, end, r.weight, kept_at);
}

// Parts of a row, 0 for rows that a workgroup does alone: up to 4096 entries, and up to 8192 (it keeps their logits in its
// registers) as long as all rows run at once, two to a compute unit.  Measured with all filters, us, alone and split: 64 rows
// of 8000 26 and 29, 1000 of 8000 95 and 51, 300 of 25000 101 and 39, 500 of 16384 75 and 38.  A part has some 4096 entries
// of few rows, and as many more as fewer workgroups than that make of many rows (two for each beyond 512) or long ones.
constexpr int SPLIT_WORKGROUPS = 1024, SPLIT_ROWS = 1024;        // in a batch of rows; rows of a batch
int split_parts(int B, int V) {
    if (V <= 4096 || (V <= 8192 && B <= 2 * EINET_NUM_CUS)) return 0;
    return min(min((V + 4095) / 4096, max(2, SPLIT_WORKGROUPS / B)), SPLIT_PARTS);
}

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }
// lays the workspace of a batch out; p == nullptr: its size alone
size_t split_layout(int B, int V, char* p, SplitRows& sp) {
    sp.parts = split_parts(B, V);
    B = min(B, SPLIT_ROWS);
    if (sp.parts == 0) return 0;
    sp.per = ((V + sp.parts - 1) / sp.parts + 4 * SPLIT_THREADS - 1) / (4 * SPLIT_THREADS) * (4 * SPLIT_THREADS);
    sp.parts = (V + sp.per - 1) / sp.per;
    size_t n = 0;
    auto take = [&](auto*& field, size_t count) {
        field = reinterpret_cast<std::remove_reference_t<decltype(field)>>(p + n);
        n += align256(count * sizeof(*field));
    };
    take(sp.best, (size_t)B * sp.parts);
    take(sp.low, (size_t)B * sp.parts);
    if (V > FIXED_UNIT) take(sp.coarse, (size_t)B * sp.parts);
    else sp.coarse = nullptr;
    take(sp.mass, (size_t)B * sp.parts * STRETCHES);
    take(sp.bin_mass, (size_t)B * SPLIT_BINS);
    take(sp.bin_count, (size_t)B * SPLIT_BINS);
    take(sp.listed, (size_t)B);
    take(sp.list, (size_t)B * LIST);
    return n;
}

// the call for rows b0 .. b0 + n - 1
ChooseArgs rows_from(const ChooseArgs& a, int b0, int n) {
    ChooseArgs r = a;
    r.B = n;
    r.logits = static_cast<const char*>(a.logits) + (int64_t)b0 * a.stride * row_type_bytes(a.type);
    r.u += b0;
    r.index += b0;
    if (a.logq) r.logq += b0;
    if (a.temperature.p) r.temperature.p += b0;
    if (a.top_k.p) r.top_k.p += b0;
    if (a.top_p.p) r.top_p.p += b0;
    if (a.min_p.p) r.min_p.p += b0;
    return r;
}

template <class T, bool OWN>
void launch_choose_split(const ChooseArgs& a, const SplitRows& sp, int shift, hipStream_t s) {
    const dim3 parts(a.B * sp.parts), rows(a.B);
    hipLaunchKernelGGL(k_choose_split_max<T>, parts, dim3(SPLIT_THREADS), 0, s, a, sp);
    const bool weighted = a.temperature.p || a.temperature.v > 0.f;          // (else the largest entry it is)
    if (OWN && weighted) hipLaunchKernelGGL(k_choose_split_scale<T>, parts, dim3(SPLIT_THREADS), 0, s, a, sp, shift);
    if (weighted) hipLaunchKernelGGL((k_choose_split_bins<T, OWN>), parts, dim3(SPLIT_THREADS), 0, s, a, sp, shift);
    const bool filters = a.top_k.p || a.top_p.p || (a.top_k.v > 0 && a.top_k.v < a.V) || a.top_p.v < 1.f;
    if (weighted && filters) hipLaunchKernelGGL((k_choose_split_collect<T, OWN>), parts, dim3(SPLIT_THREADS), 0, s, a, sp, shift);
    hipLaunchKernelGGL((k_choose_split_finish<T, OWN>), rows, dim3(FINISH_THREADS), 0, s, a, sp, shift);
}

template <class T>
void launch_choose_rows(const ChooseArgs& a, int shift, hipStream_t s) {
    const int V = a.V;
    // `threads` to a workgroup, which has `per` rows
    auto go = [&](auto kernel, int threads, int per) {
        row_batches(a.B, threads / per, [&](int64_t b0, int64_t b) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)((b + per - 1) / per)), dim3(threads), 0, s, rows_from(a, (int)b0, (int)b), shift);
        });
    };
    SplitRows sp;
    if (V <= 64) go(k_choose_wave<T, 1, 1>, 256, 4);
    else if (V <= 128) go(k_choose_wave<T, 2, 1>, 256, 4);
    else if (V <= 256) go(k_choose_wave<T, 4, 1>, 256, 4);
    else if (V <= 512) go(k_choose_wave<T, 4, 2>, 256, 4);
    else if (V <= 1024) go(k_choose_wave<T, 4, 4>, 256, 4);
    else if (V <= 2048) go(k_choose_block<T, 256, 2>, 256, 1);
    else if (V <= 4096) go(k_choose_block<T, 512, 2>, 512, 1);
    else if (split_layout(a.B, V, static_cast<char*>(a.workspace), sp) == 0) go(k_choose_block<T, 1024, 2>, 1024, 1);
    else
        for (int64_t b0 = 0; b0 < a.B; b0 += SPLIT_ROWS) {
            const ChooseArgs rows = rows_from(a, (int)b0, min(a.B - (int)b0, SPLIT_ROWS));
            if (V > FIXED_UNIT) launch_choose_split<T, true>(rows, sp, shift, s);
            else launch_choose_split<T, false>(rows, sp, shift, s);
        }
}

}  // namespace

size_t choose_workspace(int B, int V) {
    SplitRows sp;
    return B > 0 ? split_layout(B, V, nullptr, sp) : 0;
}

void launch_choose(const ChooseArgs& args, hipStream_t s) {
    if (args.B == 0) return;
    int log_v = 0;
    while (((int64_t)1 << log_v) < args.V) ++log_v;
    const int shift = 61 - log_v;
    ChooseArgs a = args;
    a.inv_t = 1.f / a.temperature.v;
    a.log2e_t = 1.4426950408889634074 / (double)a.temperature.v;
    if (a.type == ROW_FLOAT32) launch_choose_rows<float>(a, shift, s);
    else if (a.type == ROW_BFLOAT16) launch_choose_rows<__bf16>(a, shift, s);
    else launch_choose_rows<_Float16>(a, shift, s);
}

}  // namespace einet_impl

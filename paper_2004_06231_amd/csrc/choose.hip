// One entry per row of logits, under temperature, top-k, top-p and min-p, from a given uniform.
//
// The entries are ordered by (logit descending, index ascending); each filter keeps a prefix of that order, so what is
// kept is one prefix: the entries whose order key is at least `cut`.  The order key of entry i has the logit's bits, made
// monotone, in its upper half and ~i in its lower half: no two are equal, and the larger comes first.
//
// Weights exp((logit - max) / T) are held as integers of 2^-shift, shift = 62 - ceil(log2 V): at most 2^62 in all, so
// that their sums are exact and the same in whatever order they are formed, by atomics too.  A weight is off by half a unit
// at most, 2^-63 of V times the largest; sums of float64 lose more where V is below 2^10, and no sum of float32 could tell
// the entries of a long row apart: a uniform falls between two of V running sums.
#include "device_common.hpp"
#include "routing.hpp"

namespace einet_impl {

namespace {

typedef unsigned long long u64;

// ------------------------------------------------------------------------------------------------ keys and weights

// A logit's key: its bits, made monotone, without the low bits that a 16-bit type leaves empty; 0 for an entry that is
// left out (-inf, NaN).
template <class T> constexpr int KEY_SHIFT = 0;
template <> constexpr int KEY_SHIFT<__bf16> = 16;
template <> constexpr int KEY_SHIFT<_Float16> = 13;

template <class T>
__device__ __forceinline__ uint32_t logit_key(T x) {
    const float v = (float)x;
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
    float inv_t;                 // 1 / T in float32, for the bins
    double log2e_t;              // log2(e) / T
    int top_k;
    double top_p, min_p, u;
    bool greedy;
};
__device__ __forceinline__ RowSettings row_settings(const ChooseArgs& a, int row) {
    const float t = a.temperature.p ? a.temperature.p[row] : a.temperature.v, p = a.top_p.p ? a.top_p.p[row] : a.top_p.v,
                mp = a.min_p.p ? a.min_p.p[row] : a.min_p.v, u = a.u[row];
    RowSettings s;
    s.greedy = !(t > 0.f);
    s.inv_t = s.greedy ? 1.f : 1.f / t;
    s.log2e_t = 1.4426950408889634074 / (s.greedy ? 1.0 : (double)t);
    s.top_k = a.top_k.p ? a.top_k.p[row] : a.top_k.v;
    s.top_p = p >= 0.f ? (double)p : p < 0.f ? 0.0 : 1.0;       // (NaN: off)
    s.min_p = mp > 0.f ? fmin((double)mp, 1.0) : 0.0;
    s.u = u > 0.f ? (double)u : 0.0;
    return s;
}

// 2^y in units of 2^-shift, rounded to the nearest, for y <= 0.  2^y = 2^n 2^f with n the nearest integer: the series of 2^f =
// exp(f ln 2) to the 12th power is good to 0.347^13 / 13! = 1.7e-16.  Added to 2 its last place is 2^-51, whole.
__device__ __forceinline__ u64 exp2_fixed(double y, int shift) {
    y = fmax(y, -128.0);
    const double n = rint(y), f = y - n;
    constexpr double L = 0.69314718055994530942;
    double p = L * L * L * L * L * L * L * L * L * L * L * L / 479001600.0;
    p = fma(p, f, L * L * L * L * L * L * L * L * L * L * L / 39916800.0);
    p = fma(p, f, L * L * L * L * L * L * L * L * L * L / 3628800.0);
    p = fma(p, f, L * L * L * L * L * L * L * L * L / 362880.0);
    p = fma(p, f, L * L * L * L * L * L * L * L / 40320.0);
    p = fma(p, f, L * L * L * L * L * L * L / 5040.0);
    p = fma(p, f, L * L * L * L * L * L / 720.0);
    p = fma(p, f, L * L * L * L * L / 120.0);
    p = fma(p, f, L * L * L * L / 24.0);
    p = fma(p, f, L * L * L / 6.0);
    p = fma(p, f, L * L / 2.0);
    p = fma(p, f, L);
    p = fma(p, f, 1.0);
    const u64 i = __builtin_bit_cast(u64, p + 2.0) & 0xfffffffffffffull;       // p * 2^51
    const int up = (int)n + shift - 51;
    const int down = min(-up, 63);
    return up >= 0 ? i << up : (i + (1ull << (down - 1))) >> down;
}

// What the weights of a row are computed from.
template <class T>
struct RowWeights {
    uint32_t kmax;
    float m;                     // the largest logit
    double log2e_t;
    int shift;
    // (only entries at +inf have weight next to one)
    __device__ __forceinline__ u64 operator()(uint32_t k) const {
        if (k == 0u || (m == INFINITY && k != kmax)) return 0;
        return exp2_fixed(k == kmax ? 0.0 : ((double)key_logit<T>(k) - (double)m) * log2e_t, shift);
    }
    __device__ __forceinline__ float log_share(uint32_t k, u64 total) const {
        const double d = k == kmax ? 0.0 : ((double)key_logit<T>(k) - (double)m) * log2e_t * 0.69314718055994530942;
        return (float)(d - log((double)total * exp2((double)-shift)));
    }
    // the least weight that min_p keeps
    __device__ __forceinline__ u64 least(double min_p) const { return __double2ull_ru(min_p * (double)(1ull << shift)); }
};

// the first whole number above which lies a running sum that exceeds u * total
__device__ __forceinline__ u64 target_of(double u, u64 total) {
    const double t = u * (double)total;
    return t >= (double)total ? total - 1 : min((u64)t, total - 1);
}

// N consecutive entries of a row, of which the first `count` exist; the hardware loads them at any alignment at once
template <class T, int N>
__device__ __forceinline__ void load_keys(const T* x, int count, uint32_t (&k)[N]) {
    struct Pack { T v[N]; };
    if (count >= N) {
        const Pack q = load_bytes<Pack>(x);
#pragma unroll
        for (int c = 0; c < N; ++c) k[c] = logit_key(q.v[c]);
    } else {
#pragma unroll
        for (int c = 0; c < N; ++c) k[c] = c < count ? logit_key(x[c]) : 0u;
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
// over the lanes.
template <class T, int VEC, int GROUPS>
__global__ __launch_bounds__(256) void k_choose_wave(ChooseArgs a, int shift) {
    constexpr int E = VEC * GROUPS;
    const int row = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6)), lane = threadIdx.x & 63, V = a.V;
    if (row >= a.B) return;
    const T* const x = static_cast<const T*>(a.logits) + row * a.stride;
    const RowSettings st = row_settings(a, row);
    uint32_t k[E];
    uint32_t best = 0;
#pragma unroll
    for (int g = 0; g < GROUPS; ++g) {
        uint32_t part[VEC];
        const int i0 = (g * 64 + lane) * VEC;
        load_keys<T, VEC>(x + i0, V - i0, part);
#pragma unroll
        for (int c = 0; c < VEC; ++c) k[g * VEC + c] = part[c], best = max(best, part[c]);
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
#pragma unroll
    for (int e = 0; e < E; ++e) w[e] = weight(k[e]);
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
        const u64 total = mass_from(1), mass = max((u64)1, __double2ull_ru(st.top_p * (double)total));
        uint32_t lo = 1, hi = kmax + 1;                          // at least `mass` from lo on, less from hi on
        int n_lo = count_from(1), n_hi = 0;
        u64 m_hi = 0;
        while (hi - lo > 1 && n_lo - n_hi > 1) {
            const uint32_t mid = lo + (hi - lo) / 2;
            const u64 m = mass_from(mid);
            const int n = count_from(mid);
            if (m >= mass) lo = mid, n_lo = n;
            else hi = mid, n_hi = n, m_hi = m;
        }
        if (n_lo - n_hi <= 1) {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (k[e] < lo) k[e] = 0u, w[e] = 0;
        } else {
            // several of one key: as many as it takes to reach the mass
            const u64 each = weight(lo), missing = mass - m_hi;
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
                if (a.logq) a.logq[row] = weight.log_share(key, total);
            }
        }
    }
}

// ------------------------------------------------------------------------------------------ a workgroup for every row
//
// Wave w of the workgroup has a contiguous stretch of the row, in groups of 256 entries (four to a lane).  GROUPS > 0: the
// keys of the stretch stay in registers; 0: they are read again by every pass.
//
// A cut is found from the histogram of the entries over their distance from the largest logit in units of T (BINS equal bins
// to 32 units; their order is the entries' order): the bin that the cut lies in holds few entries of an ordinary row, and a
// radix search over the order keys of that bin's entries finds the very entry.
template <class T, int NT, int GROUPS>
struct RowKeys {
    const T* x;
    int V, first, groups;        // of this thread's wave: its first group, the number of its groups
    uint32_t k[GROUPS > 0 ? GROUPS * 4 : 1];
    __device__ void init(const T* row, int n) {
        x = row;
        V = n;
        const int wave = threadIdx.x >> 6;
        if constexpr (GROUPS > 0) {
            groups = GROUPS;
            first = wave * GROUPS;
#pragma unroll
            for (int g = 0; g < GROUPS; ++g) {
                uint32_t part[4];
                const int i0 = (first + g) * 256 + (int)(threadIdx.x & 63) * 4;
                load_keys<T, 4>(x + i0, V - i0, part);
#pragma unroll
                for (int c = 0; c < 4; ++c) k[g * 4 + c] = part[c];
            }
        } else {
            groups = (V + NT * 4 - 1) / (NT * 4);
            first = wave * groups;
        }
    }
    // f(index, key) for the four entries of a group
    template <class F>
    __device__ __forceinline__ void group(int g, F&& f) const {
        const int i0 = (first + g) * 256 + (int)(threadIdx.x & 63) * 4;
        uint32_t part[4];
        load_keys<T, 4>(x + i0, V - i0, part);
#pragma unroll
        for (int c = 0; c < 4; ++c) f(i0 + c, part[c]);
    }
    template <class F>
    __device__ __forceinline__ void each(F&& f) const {
        if constexpr (GROUPS > 0) {
#pragma unroll
            for (int g = 0; g < GROUPS; ++g)
#pragma unroll
                for (int c = 0; c < 4; ++c) f((first + g) * 256 + (int)(threadIdx.x & 63) * 4 + c, k[g * 4 + c]);
        } else {
            for (int g = 0; g < groups; ++g) group(g, f);
        }
    }
};

template <int NT>
struct ChooseShared {
    static constexpr int BINS = 2 * NT;
    u64 mass[BINS];
    uint32_t count[BINS];
    u64 digit[256];
    u64 tmp[NT / 64];
    u64 found[2];
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
// values reaches target.  A byte of the order key after the other, from the first in which the entries differ.
template <int NT, class Each>
__device__ __forceinline__ u64 find_entry(Each&& each, u64 target, ChooseShared<NT>& sh) {
    u64 hi = 0, lo = 0;
    each([&](u64 o, u64) { hi = max(hi, o), lo = max(lo, ~o); });
    hi = block_reduce<NT>(hi, sh.tmp, OpMax{});
    lo = ~block_reduce<NT>(lo, sh.tmp, OpMax{});
    int top = 64 - __clzll(hi ^ lo);                             // bits in which they differ (0: one entry)
    if (hi == lo) return hi;
    u64 prefix = top < 64 ? hi >> top : 0;
    while (top > 0) {
        const int shift = max(0, top - 8), n = 1 << (top - shift);
        __syncthreads();
        if (threadIdx.x < 256) sh.digit[threadIdx.x] = 0;
        __syncthreads();
        each([&](u64 o, u64 v) {
            if ((top < 64 ? o >> top : 0) == prefix && v) atomicAdd(&sh.digit[(o >> shift) & (n - 1)], v);
        });
        __syncthreads();
        if (threadIdx.x < 64) {                                  // from the largest digit down, four to a lane
            u64 v[4], sum = 0;
#pragma unroll
            for (int c = 0; c < 4; ++c) v[c] = sh.digit[255 - (4 * threadIdx.x + c)], sum += v[c];
            u64 before = wave_scan(sum, OpAdd{}) - sum;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                if (before < target && target <= before + v[c]) sh.found[0] = 255 - (4 * threadIdx.x + c), sh.found[1] = target - before;
                before += v[c];
            }
        }
        __syncthreads();
        prefix = (prefix << (top - shift)) | sh.found[0];
        target = sh.found[1];
        top = shift;
    }
    return prefix;
}

template <class T, int NT, int GROUPS>
__global__ __launch_bounds__(NT) void k_choose_block(ChooseArgs a, int shift) {
    __shared__ ChooseShared<NT> sh;
    constexpr int BINS = ChooseShared<NT>::BINS;
    const int row = blockIdx.x, tid = threadIdx.x, V = a.V;
    const RowSettings st = row_settings(a, row);
    RowKeys<T, NT, GROUPS> keys;
    keys.init(static_cast<const T*>(a.logits) + row * a.stride, V);
    u64 best = 0;
    keys.each([&](int i, uint32_t k) { best = max(best, k ? order_key(k, i) : 0); });
    best = block_reduce<NT>(best, sh.tmp, OpMax{});
    const uint32_t kmax = (uint32_t)(best >> 32);
    if (kmax == 0u || st.greedy) {
        if (tid == 0) {
            a.index[row] = kmax ? (int)~(uint32_t)best : -1;
            if (a.logq) a.logq[row] = kmax ? 0.f : -INFINITY;
        }
        return;
    }
    const RowWeights<T> weight{kmax, key_logit<T>(kmax), st.log2e_t, shift};
    const float per_bin = st.inv_t * (float)(BINS / 32);
    auto bin_of = [&](uint32_t k) {
        const float q = (weight.m - key_logit<T>(k)) * per_bin;
        return k == kmax ? 0 : q < (float)(BINS - 1) ? (int)q : BINS - 1;
    };
    u64 cut = 1ull << 32;                                        // everything that is not left out
    const bool by_count = st.top_k > 0 && st.top_k < V, by_mass = st.top_p < 1.0;
    if (by_count || by_mass) {
        for (int b = tid; b < BINS; b += NT) sh.count[b] = 0, sh.mass[b] = 0;
        __syncthreads();
        keys.each([&](int, uint32_t k) {
            if (k == 0u) return;
            const int b = bin_of(k);
            if (by_count) atomicAdd(&sh.count[b], 1u);
            if (by_mass) atomicAdd(&sh.mass[b], weight(k));
        });
        __syncthreads();
        // entries of a bin from the cut on, with their values
        auto of_bin = [&](int bin, auto value) {
            return [&, bin, value](auto f) {
                keys.each([&](int i, uint32_t k) {
                    if (k == 0u || bin_of(k) != bin) return;
                    const u64 o = order_key(k, i);
                    if (o >= cut) f(o, value(k));
                });
            };
        };
        int bin;
        u64 missing, total;
        if (by_count) {
            block_scan<NT>((u64)sh.count[2 * tid] + sh.count[2 * tid + 1], sh.tmp, total);
            if (total > (u64)st.top_k) {
                find_bin<NT>(sh.count, (u64)st.top_k, sh, bin, missing);
                cut = find_entry<NT>(of_bin(bin, [](uint32_t) -> u64 { return 1; }), missing, sh);
                if (by_mass) {
                    // the mass of that bin is what is kept of it, that of the bins behind it none
                    u64 rest = 0;
                    of_bin(bin, weight)([&](u64, u64 v) { rest += v; });
                    rest = block_reduce<NT>(rest, sh.tmp, OpAdd{});
                    for (int b = tid; b < BINS; b += NT)
                        if (b >= bin) sh.mass[b] = b == bin ? rest : 0;
                    __syncthreads();
                }
            }
        }
        if (by_mass) {
            block_scan<NT>(sh.mass[2 * tid] + sh.mass[2 * tid + 1], sh.tmp, total);
            // kept: what has less than top_p of the total before it; the last one's own weight reaches that mass
            find_bin<NT>(sh.mass, max((u64)1, __double2ull_ru(st.top_p * (double)total)), sh, bin, missing);
            cut = find_entry<NT>(of_bin(bin, weight), missing, sh);
        }
    }
    const u64 least = weight.least(st.min_p);
    auto kept = [&](int i, uint32_t k) {
        if (k == 0u || order_key(k, i) < cut) return (u64)0;
        const u64 w = weight(k);
        return w < least ? (u64)0 : w;
    };
    u64 mine = 0, total;
    keys.each([&](int i, uint32_t k) { mine += kept(i, k); });
    const u64 wave_sum = wave_reduce(mine, OpAdd{});
    const u64 end = block_scan<NT>((tid & 63) == 63 ? wave_sum : 0, sh.tmp, total);
    const u64 target = target_of(st.u, total);
    // the wave in whose stretch the running sum exceeds the target goes through its groups
    u64 run = lane_value(end, 63) - wave_sum;
    if (target < run || target >= run + wave_sum) return;
    for (int g = 0; g < keys.groups; ++g) {
        u64 w[4], sum = 0;
        uint32_t k4[4];
        int c = 0;
        keys.group(g, [&](int i, uint32_t k) {
            k4[c] = k;
            w[c] = kept(i, k);
            sum += w[c];
            ++c;
        });
        const u64 ends = wave_scan(sum, OpAdd{}) + run;
        const u64 above = __ballot(ends > target);
        if (above) {
            if ((tid & 63) == __ffsll(above) - 1) {
                u64 s = ends;
                int at = 3;
#pragma unroll
                for (int c = 3; c > 0; --c) {
                    s -= w[c];
                    if (s > target) at = c - 1;
                }
                a.index[row] = (keys.first + g) * 256 + (tid & 63) * 4 + at;
                if (a.logq) a.logq[row] = weight.log_share(at == 0 ? k4[0] : at == 1 ? k4[1] : at == 2 ? k4[2] : k4[3], total);
            }
            return;
        }
        run = lane_value(ends, 63);
    }
}

template <class T>
void launch_choose_rows(const ChooseArgs& a, int shift, hipStream_t s) {
    const int V = a.V;
    const dim3 waves((a.B + 3) / 4), rows(a.B);
    if (V <= 64) hipLaunchKernelGGL((k_choose_wave<T, 1, 1>), waves, dim3(256), 0, s, a, shift);
    else if (V <= 128) hipLaunchKernelGGL((k_choose_wave<T, 2, 1>), waves, dim3(256), 0, s, a, shift);
    else if (V <= 256) hipLaunchKernelGGL((k_choose_wave<T, 4, 1>), waves, dim3(256), 0, s, a, shift);
    else if (V <= 512) hipLaunchKernelGGL((k_choose_wave<T, 4, 2>), waves, dim3(256), 0, s, a, shift);
    else if (V <= 1024) hipLaunchKernelGGL((k_choose_wave<T, 4, 4>), waves, dim3(256), 0, s, a, shift);
    else if (V <= 2048) hipLaunchKernelGGL((k_choose_block<T, 256, 2>), rows, dim3(256), 0, s, a, shift);
    else if (V <= 8192) hipLaunchKernelGGL((k_choose_block<T, 1024, 2>), rows, dim3(1024), 0, s, a, shift);
    else hipLaunchKernelGGL((k_choose_block<T, 1024, 0>), rows, dim3(1024), 0, s, a, shift);
}

}  // namespace

size_t choose_workspace(int, int) { return 0; }

void launch_choose(const ChooseArgs& a, hipStream_t s) {
    if (a.B == 0) return;
    int log_v = 0;
    while (((int64_t)1 << log_v) < a.V) ++log_v;
    const int shift = 62 - log_v;
    if (a.type == ROW_FLOAT32) launch_choose_rows<float>(a, shift, s);
    else if (a.type == ROW_BFLOAT16) launch_choose_rows<__bf16>(a, shift, s);
    else launch_choose_rows<_Float16>(a, shift, s);
}

}  // namespace einet_impl

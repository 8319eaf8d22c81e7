// One entry per row of logits, under temperature, top-k, top-p and min-p, from a given uniform.
//
// The entries are ordered by (logit descending, index ascending); each filter keeps a prefix of that order, so what is
// kept is one prefix: the entries whose order key is at least `cut`.  The order key of entry i has the logit's bits, made
// monotone, in its upper half and ~i in its lower half: no two are equal, and the larger comes first.
//
// Weights exp((logit - max) / T) are held as integers of 2^-shift, shift = 62 - ceil(log2 V): at most 2^62 in all, so
// that their sums are exact and the same in whatever order they are formed, by atomics too.  What such a weight loses,
// 2^-(shift + 1), is 2^-63 of V times the largest weight; sums of float64 lose more where V is below 2^10 and no sum of
// float32 could tell the entries of a long row apart: a uniform falls between two of V running sums.
#include "device_common.hpp"
#include "routing.hpp"

namespace einet_impl {

namespace {

typedef unsigned long long u64;

// 0 for an entry that is left out (-inf, NaN)
__device__ __forceinline__ uint32_t logit_key(float v) {
    if (!(v > -INFINITY)) return 0u;
    if (v == 0.f) v = 0.f;                                       // -0 and 0 are equal
    const uint32_t b = __builtin_bit_cast(uint32_t, v);
    return (b >> 31) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_logit(uint32_t k) {
    return __builtin_bit_cast(float, (k >> 31) ? k & 0x7fffffffu : ~k);
}
__device__ __forceinline__ u64 order_key(uint32_t k, int i) { return ((u64)k << 32) | (uint32_t)~i; }

struct RowSettings {
    double inv_t;
    int top_k;
    double top_p, min_p, u;
    bool greedy;
};
__device__ __forceinline__ RowSettings row_settings(const ChooseArgs& a, int row) {
    const float t = a.temperature.p ? a.temperature.p[row] : a.temperature.v, p = a.top_p.p ? a.top_p.p[row] : a.top_p.v,
                mp = a.min_p.p ? a.min_p.p[row] : a.min_p.v, u = a.u[row];
    RowSettings s;
    s.greedy = !(t > 0.f);
    s.inv_t = s.greedy ? 1.0 : 1.0 / (double)t;
    s.top_k = a.top_k.p ? a.top_k.p[row] : a.top_k.v;
    s.top_p = p >= 0.f ? (double)p : p < 0.f ? 0.0 : 1.0;       // (NaN: off)
    s.min_p = mp > 0.f ? fmin((double)mp, 1.0) : 0.0;
    s.u = u > 0.f ? (double)u : 0.0;
    return s;
}

// weight of a key in units of 2^-shift; scale = 2^shift.  Nothing but the maximum has weight next to an infinite one.
__device__ __forceinline__ u64 weight_of(uint32_t k, uint32_t kmax, double m, double inv_t, double scale) {
    if (k == kmax) return (u64)scale;
    if (k == 0u || m == INFINITY) return 0;
    return __double2ull_rn(exp(((double)key_logit(k) - m) * inv_t) * scale);
}

constexpr int CHOOSE_THREADS = 1024;

template <class V>
__device__ V block_reduce(V v, V* tmp, V (*op)(V, V)) {
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) v = op(v, __shfl_xor(v, o, 64));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) tmp[threadIdx.x >> 6] = v;
    __syncthreads();
    v = tmp[0];
    for (int w = 1; w < CHOOSE_THREADS / 64; ++w) v = op(v, tmp[w]);
    return v;
}
__device__ u64 op_add(u64 a, u64 b) { return a + b; }
__device__ u64 op_max(u64 a, u64 b) { return a > b ? a : b; }

template <class T>
__global__ __launch_bounds__(CHOOSE_THREADS) void k_choose(ChooseArgs a, double scale) {
    __shared__ u64 tmp[CHOOSE_THREADS / 64], hist[256], found[2];
    const int row = blockIdx.x, tid = threadIdx.x, V = a.V;
    const T* const x = static_cast<const T*>(a.logits) + row * a.stride;
    const RowSettings st = row_settings(a, row);
    auto key = [&](int i) { return logit_key((float)x[i]); };
    u64 best = 0;
    for (int i = tid; i < V; i += CHOOSE_THREADS) best = op_max(best, order_key(key(i), i));
    best = block_reduce<u64>(best, tmp, op_max);
    const uint32_t kmax = (uint32_t)(best >> 32);
    if (kmax == 0u || st.greedy) {
        if (tid == 0) {
            a.index[row] = kmax ? (int)~(uint32_t)best : -1;
            if (a.logq) a.logq[row] = kmax ? 0.f : -INFINITY;
        }
        return;
    }
    const double m = (double)key_logit(kmax);
    u64 cut = 1ull << 32;                                        // everything that is not left out
    // The entry before whose end in the order lies `target` (1, 2, ..): from the top byte of the order key down, the
    // byte's sums over the entries that agree with what is found of it so far.
    auto last_of = [&](u64 target, auto value) {
        u64 prefix = 0;
        for (int shift = 56; shift >= 0; shift -= 8) {
            __syncthreads();
            if (tid < 256) hist[tid] = 0;
            __syncthreads();
            for (int i = tid; i < V; i += CHOOSE_THREADS) {
                const u64 o = order_key(key(i), i);
                if (o < cut || (shift < 56 && (o >> (shift + 8)) != prefix)) continue;
                const u64 v = value(o);
                if (v) atomicAdd(&hist[(o >> shift) & 255], v);
            }
            __syncthreads();
            if (tid == 0) {
                u64 before = 0;
                int b = 255;
                for (; b > 0 && before + hist[b] < target; --b) before += hist[b];
                found[0] = b;
                found[1] = before;
            }
            __syncthreads();
            prefix = (prefix << 8) | found[0];
            target -= found[1];
        }
        return prefix;
    };
    auto sum_of = [&](auto value) {
        u64 s = 0;
        for (int i = tid; i < V; i += CHOOSE_THREADS) {
            const u64 o = order_key(key(i), i);
            if (o >= cut) s += value(o);
        }
        return block_reduce<u64>(s, tmp, op_add);
    };
    auto one = [](u64) -> u64 { return 1; };
    auto weight = [&](u64 o) { return weight_of((uint32_t)(o >> 32), kmax, m, st.inv_t, scale); };
    if (st.top_k > 0 && st.top_k < V && sum_of(one) > (u64)st.top_k) cut = last_of((u64)st.top_k, one);
    if (st.top_p < 1.0) {
        // kept: what has less than top_p of the total before it; the last one's own weight reaches that mass
        const u64 total = sum_of(weight), mass = __double2ull_ru(st.top_p * (double)total);
        cut = mass == 0 ? best : last_of(mass, weight);
    }
    // the choice: running sums over the index, every thread a stretch of the row
    auto kept = [&](int i) {
        const u64 o = order_key(key(i), i);
        if (o < cut) return (u64)0;
        const u64 w = weight(o);
        return st.min_p > 0.0 && (uint32_t)(o >> 32) != kmax &&
                       exp(((double)key_logit((uint32_t)(o >> 32)) - m) * st.inv_t) < st.min_p
                   ? (u64)0 : w;
    };
    const int per = (V + CHOOSE_THREADS - 1) / CHOOSE_THREADS, lo = min(V, tid * per), hi = min(V, lo + per);
    u64 mine = 0;
    for (int i = lo; i < hi; ++i) mine += kept(i);
    u64 run = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const u64 v = __shfl_up(run, o, 64);
        if ((tid & 63) >= o) run += v;
    }
    __syncthreads();
    if ((tid & 63) == 63) tmp[tid >> 6] = run;
    __syncthreads();
    u64 total = 0;
    for (int w = 0; w < CHOOSE_THREADS / 64; ++w) {
        if (w == tid >> 6) run += total;
        total += tmp[w];
    }
    u64 target = (u64)(st.u * (double)total);
    if (target >= total) target = total - 1;
    if (run - mine <= target && target < run) {
        u64 sum = run - mine;
        for (int i = lo; i < hi; ++i) {
            sum += kept(i);
            if (sum > target) {
                a.index[row] = i;
                if (a.logq) {
                    const uint32_t k = key(i);
                    const double d = k == kmax ? 0.0 : ((double)key_logit(k) - m) * st.inv_t;
                    a.logq[row] = (float)(d - log((double)total / scale));
                }
                break;
            }
        }
    }
}

}  // namespace

size_t choose_workspace(int, int) { return 0; }

void launch_choose(const ChooseArgs& a, hipStream_t s) {
    if (a.B == 0) return;
    int log_v = 0;
    while (((int64_t)1 << log_v) < a.V) ++log_v;
    const double scale = (double)(1ull << (62 - log_v));
    if (a.type == ROW_FLOAT32) hipLaunchKernelGGL(k_choose<float>, dim3(a.B), dim3(CHOOSE_THREADS), 0, s, a, scale);
    else if (a.type == ROW_BFLOAT16) hipLaunchKernelGGL(k_choose<__bf16>, dim3(a.B), dim3(CHOOSE_THREADS), 0, s, a, scale);
    else hipLaunchKernelGGL(k_choose<_Float16>, dim3(a.B), dim3(CHOOSE_THREADS), 0, s, a, scale);
}

}  // namespace einet_impl

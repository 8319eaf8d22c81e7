// Routing samples to the components of a mixture: the most probable components of every sample with their weights, a
// stable counting sort of the (sample, choice) slots by component, and rows carried to their components and back.
#include "device_common.hpp"
#include "routing.hpp"

namespace einet_impl {

namespace {

template <class T>
__device__ __forceinline__ float to_float(T v) { return (float)v; }

// ---------------------------------------------------------------------------------------------------- routing
//
// With t[c] = score[c] + coef[c], m = max t and z = sum exp(t[c] - m): logp = m + log z, p[c] = exp(t[c] - m) / z.  The
// sums t are formed in float64 (type K): log-densities are in the hundreds and thousands and differ by little, and which
// of two is larger must not depend on a rounding.  Without coefficients t is the score, and K float.  A component whose t
// is -inf or NaN is left out.

// All lanes of a group of G get op over the group: lanes that differ in one, then in two bits, mirrored halves of 8 and 16.
template <int CTRL>
__device__ __forceinline__ float lane_of(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
template <int CTRL>
__device__ __forceinline__ int lane_of(int v) { return __builtin_amdgcn_mov_dpp(v, CTRL, 0xf, 0xf, true); }
template <int CTRL>
__device__ __forceinline__ double lane_of(double v) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)lane_of<CTRL>((int)(uint32_t)b), hi = (uint32_t)lane_of<CTRL>((int)(uint32_t)(b >> 32));
    return __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}
template <int G, class V, class Op>
__device__ __forceinline__ V group_reduce(V v, Op op) {
    if constexpr (G >= 2) v = op(v, lane_of<0xB1>(v));
    if constexpr (G >= 4) v = op(v, lane_of<0x4E>(v));
    if constexpr (G >= 8) v = op(v, lane_of<0x141>(v));
    if constexpr (G >= 16) v = op(v, lane_of<0x140>(v));
    if constexpr (G >= 32) v = op(v, __shfl_xor(v, 16, 64));
    if constexpr (G >= 64) v = op(v, __shfl_xor(v, 32, 64));
    return v;
}
struct Larger {
    __device__ float operator()(float a, float b) const { return fmaxf(a, b); }
    __device__ double operator()(double a, double b) const { return fmax(a, b); }
};
struct Smaller {
    __device__ int operator()(int a, int b) const { return min(a, b); }
};
struct Plus {
    __device__ float operator()(float a, float b) const { return a + b; }
};

// exp(t - m) of a component, 1 at the maximum (also where both are infinite), 0 for one that is left out.  The argument is
// rounded to float32 once: of the product with log2(e) what its rounding took is added back to first order.
__device__ __forceinline__ float route_exp(double t, double m) {
    const float y = (float)fmax((t - m) * 1.4426950408889634074, -200.0);
    return t == m ? 1.f : __builtin_amdgcn_exp2f(y);
}
__device__ __forceinline__ float route_exp(float t, float m) {
    constexpr float L = 1.44269502f, L_REST = 1.92596299e-8f;
    const float d = fmaxf(t - m, -150.f), y = d * L, e = __builtin_amdgcn_exp2f(y);
    const float rest = fmaf(d, L_REST, fmaf(d, L, -y));
    return t == m ? 1.f : fmaf(e, rest * 0.693147182f, e);
}

template <class K, class T>
__device__ __forceinline__ K route_sum(T score, const float* coef, int c) {
    K t = (K)to_float(score);
    if constexpr (sizeof(K) == 8) t += (K)coef[c];
    return t > (K)-INFINITY ? t : (K)-INFINITY;                 // (NaN too)
}

// G lanes share a sample, each with E components in registers: VEC neighbours of every G * VEC, which are one load where
// the components of a sample are next to each other.  16001 rows of 128 bf16 logits, eight selections: 7.3 us, 0.6 TB/s; the
// vector ALU bounds it, whose instructions are the eight selections (some 50 each for the wave's four samples) and the
// exponentials.
template <class T, int E> constexpr int ROUTE_VEC = E < 16 / (int)sizeof(T) ? E : 16 / (int)sizeof(T);
template <class T, int G, int E>
__device__ __forceinline__ int route_component(int e, int j) {
    constexpr int VEC = ROUTE_VEC<T, E>;
    return ((e / VEC) * G + j) * VEC + e % VEC;
}

template <class T, class K, int G, int E>
__device__ __forceinline__ K route_load(const T* __restrict__ p, int64_t sc, int64_t sn, const float* __restrict__ coef, int M,
                                        int64_t n, int j, K (&t)[E]) {
    constexpr int VEC = ROUTE_VEC<T, E>;
    struct Pack { T v[VEC]; };
    const T* const row = p + n * sn;
    K m = (K)-INFINITY;
#pragma unroll
    for (int v = 0; v < E / VEC; ++v) {
        const int c0 = route_component<T, G, E>(v * VEC, j);
        if (sc == 1 && c0 + VEC <= M) {
            const Pack q = load_bytes<Pack>(row + c0);
#pragma unroll
            for (int i = 0; i < VEC; ++i) t[v * VEC + i] = route_sum<K>(q.v[i], coef, c0 + i);
        } else {
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                t[v * VEC + i] = c0 + i < M ? route_sum<K>(row[(c0 + i) * sc], coef, c0 + i) : (K)-INFINITY;
        }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) m = Larger{}(m, t[e]);
    return group_reduce<G>(m, Larger{});
}

// Where the samples of a component are next to each other, the scores of ROUTE_STAGE samples come through LDS: read along the
// samples, handed out along the components.  Rows of M | 1 floats: neither way meets a bank twice.
template <int G> constexpr int ROUTE_STAGE = G == 64 ? 8 : 32;
template <int G, bool STAGED> constexpr int ROUTE_THREADS = STAGED ? ROUTE_STAGE<G> * G : 256;

template <class T, int G>
__device__ __forceinline__ void stage_scores(const T* __restrict__ p, int64_t sc, int M, int64_t n0, int64_t N, float* tile) {
    constexpr int S = ROUTE_STAGE<G>;
    const int s = threadIdx.x % S, wide = M | 1;
    const bool there = n0 + s < N;
#pragma unroll 4
    for (int c = threadIdx.x / S; c < M; c += G) tile[s * wide + c] = there ? to_float(p[c * sc + n0 + s]) : -INFINITY;
    __syncthreads();
}
template <class T, class K, int G, int E>
__device__ __forceinline__ K staged_load(const float* tile, const float* __restrict__ coef, int M, int j, K (&t)[E]) {
    const float* const row = tile + threadIdx.x / G * (M | 1);
    K m = (K)-INFINITY;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int c = route_component<T, G, E>(e, j);
        t[e] = c < M ? route_sum<K>(row[c], coef, c) : (K)-INFINITY;
        m = Larger{}(m, t[e]);
    }
    return group_reduce<G>(m, Larger{});
}

template <class T, class K, int G, int E, bool STAGED>
__global__ __launch_bounds__((ROUTE_THREADS<G, STAGED>))
void k_route(const T* __restrict__ p, int64_t sc, int64_t sn, const float* __restrict__ coef, int M, int64_t N, int top,
             int renormalise, int32_t* __restrict__ ids, float* __restrict__ weights, float* __restrict__ logp) {
    constexpr int S = ROUTE_THREADS<G, STAGED> / G;
    const int j = threadIdx.x % G;
    const int64_t n = (int64_t)blockIdx.x * S + threadIdx.x / G;
    extern __shared__ float tile[];
    if constexpr (STAGED) stage_scores<T, G>(p, sc, M, (int64_t)blockIdx.x * S, N, tile);
    if (n >= N) return;
    K t[E];
    K m;
    if constexpr (STAGED) m = staged_load<T, K, G, E>(tile, coef, M, j, t);
    else m = route_load<T, K, G, E>(p, sc, sn, coef, M, n, j, t);
    const bool dead = !(m > (K)-INFINITY);
    float z = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) z += dead ? 0.f : route_exp(t[e], m);
    z = group_reduce<G>(z, Plus{});
    // one selection after the other, the largest of what is left; lane s of the group keeps selection s
    int my_id = -1;
    float my_e = 0.f;
    K best = m;
    for (int s = 0; s < top; ++s) {
        if (s > 0) {
            best = (K)-INFINITY;
#pragma unroll
            for (int e = 0; e < E; ++e) best = Larger{}(best, t[e]);
            best = group_reduce<G>(best, Larger{});
        }
        if (!(best > (K)-INFINITY)) break;
        int c = 0x7fffffff;
#pragma unroll
        for (int e = E - 1; e >= 0; --e) c = t[e] == best ? route_component<T, G, E>(e, j) : c;
        c = group_reduce<G>(c, Smaller{});
        if (j == s) my_id = c, my_e = route_exp(best, m);
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (c == route_component<T, G, E>(e, j)) t[e] = (K)-INFINITY;
    }
    const float total = renormalise ? group_reduce<G>(my_e, Plus{}) : z;
    if (j < top) {
        ids[n * top + j] = my_id;
        weights[n * top + j] = my_id >= 0 ? my_e / total : 0.f;
    }
    if (j == 0) logp[n] = dead ? -INFINITY : (float)((double)m + (double)logf(z));
}

// A sample to a lane, for components whose samples are next to each other: the loads of a component are contiguous over
// the lanes, and up to MOST components of a sample are in registers.  262144 samples of 64 components: 17 us with one
// selection and no coefficients (4.1 TB/s), 24 us with two and coefficients: the loads of all components come first, then two
// float64 sums of each, so neither memory (2.9 TB/s) nor the vector ALU (busy 57 % of the time) is full.
constexpr int ROUTE_COLUMNS_MOST = 64;
template <class T, class K, int TOP, int MOST>
__global__ __launch_bounds__(256) void k_route_columns(const T* __restrict__ p, int64_t sc, const float* __restrict__ coef, int M,
                                                       int64_t N, int top, int renormalise, int32_t* __restrict__ ids,
                                                       float* __restrict__ weights, float* __restrict__ logp) {
    const int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (n >= N) return;
    T x[MOST];
#pragma unroll
    for (int c = 0; c < MOST; ++c) x[c] = p[n + min(c, M - 1) * sc];
    // f(component, one of eight, score) for all components
    auto each = [&](auto f) {
#pragma unroll
        for (int c0 = 0; c0 < MOST; c0 += 8) {
            if (c0 >= M) break;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (c0 + i < M) f(c0 + i, i, x[c0 + i]);
        }
    };
    K best[TOP];
    int id[TOP];
#pragma unroll
    for (int s = 0; s < TOP; ++s) best[s] = (K)-INFINITY, id[s] = -1;
    each([&](int c, int, T score) {
        const K t = route_sum<K>(score, coef, c);
        if (!(t > best[TOP - 1])) return;                    // (equal ones stay behind the lower component)
        best[TOP - 1] = t;
        id[TOP - 1] = c;
#pragma unroll
        for (int s = TOP - 1; s > 0; --s)
            if (best[s] > best[s - 1]) {
                const K b = best[s];
                const int k = id[s];
                best[s] = best[s - 1], id[s] = id[s - 1];
                best[s - 1] = b, id[s - 1] = k;
            }
    });
    const K m = best[0];
    const bool dead = !(m > (K)-INFINITY);
    float sums[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sums[i] = 0.f;
    if (!dead) each([&](int c, int i, T score) { sums[i] += route_exp(route_sum<K>(score, coef, c), m); });
    const float z = ((sums[0] + sums[1]) + (sums[2] + sums[3])) + ((sums[4] + sums[5]) + (sums[6] + sums[7]));
    float e[TOP], total = 0.f;
#pragma unroll
    for (int s = 0; s < TOP; ++s) {
        e[s] = s < top && best[s] > (K)-INFINITY ? route_exp(best[s], m) : 0.f;
        total += e[s];
    }
    if (!renormalise) total = z;
#pragma unroll
    for (int s = 0; s < TOP; ++s)
        if (s < top) {
            ids[n * top + s] = id[s];
            weights[n * top + s] = id[s] >= 0 ? e[s] / total : 0.f;
        }
    logp[n] = dead ? -INFINITY : (float)((double)m + (double)logf(z));
}

// Sums of the gradients of the coefficients, a row for every wave of the workgroup.
template <int G, int E, bool STAGED> constexpr size_t route_sums_bytes = sizeof(float) * (ROUTE_THREADS<G, STAGED> / 64) * G * E;

// With a = sum_s dw[s] w[s]:
//   d t[c] = p[c] (dlogp - a) + sum_{s: id[s] = c} dw[s] w[s]            (weights p)
//   d t[c] = p[c] dlogp + sum_{s: id[s] = c} w[s] (dw[s] - a)            (weights that sum to one)
// The log-density and the weights are differences and quotients of numbers rounded to float32; m and z come from the
// scores again.  d coef[c] = sum_n d t[c][n]: a lane has the same components for all its samples and adds their gradients
// up in registers; the workgroup's sums go to a row of the workspace, which the second kernel adds up in a fixed order.
template <class T, class K, int G, int E, bool STAGED>
__global__ __launch_bounds__((ROUTE_THREADS<G, STAGED>)) void k_route_backward(const T* __restrict__ p, int64_t sc, int64_t sn,
                                                        const float* __restrict__ coef, int M, int64_t N, int top,
                                                        int renormalise, const int32_t* __restrict__ ids,
                                                        const float* __restrict__ weights, const float* __restrict__ dweights,
                                                        const float* __restrict__ dlogp, T* __restrict__ dscores, int64_t dsc,
                                                        int64_t dsn, float* __restrict__ partial) {
    constexpr int NT = ROUTE_THREADS<G, STAGED>, S = NT / G, VEC = ROUTE_VEC<T, E>;
    struct Pack { T v[VEC]; };
    extern __shared__ float tile[];
    const int j = threadIdx.x % G;
    float acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.f;
    for (int64_t n0 = (int64_t)blockIdx.x * S; n0 < N; n0 += (int64_t)gridDim.x * S) {
        if constexpr (STAGED) stage_scores<T, G>(p, sc, M, n0, N, tile);
        // (the samples behind the last one are the last one again, and count for nothing)
        const bool there = n0 + threadIdx.x / G < N;
        const int64_t n = there ? n0 + threadIdx.x / G : N - 1;
        K t[E];
        K m;
        if constexpr (STAGED) m = staged_load<T, K, G, E>(tile, coef, M, j, t);
        else m = route_load<T, K, G, E>(p, sc, sn, coef, M, n, j, t);
        const bool dead = !(m > (K)-INFINITY);
        float z = 0.f;
        float d[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            d[e] = dead ? 0.f : route_exp(t[e], m);
            z += d[e];
        }
        z = group_reduce<G>(z, Plus{});
        int id = -1;
        float w = 0.f, dw = 0.f;
        if (j < top && dweights) {
            id = ids[n * top + j];
            w = weights[n * top + j];
            dw = dweights[n * top + j];
            if (id < 0) w = dw = 0.f;
        }
        const float a = group_reduce<G>(w * dw, Plus{}), dl = dlogp ? dlogp[n] : 0.f;
        const float scale = dead ? 0.f : (renormalise ? dl : dl - a) / z, add = w * (renormalise ? dw - a : dw);
#pragma unroll
        for (int e = 0; e < E; ++e) d[e] *= scale;
        if (dweights)
            for (int s = 0; s < top; ++s) {
                const int c = __shfl(id, s, G);
                const float v = __shfl(add, s, G);
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (c == route_component<T, G, E>(e, j)) d[e] += v;
            }
        if constexpr (STAGED) {
            float* const mine = tile + threadIdx.x / G * (M | 1);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const int c = route_component<T, G, E>(e, j);
                if (c < M) mine[c] = d[e];
                if (there) acc[e] += d[e];
            }
            __syncthreads();
            const int s = threadIdx.x % S;
            if (n0 + s < N)
                for (int c = threadIdx.x / S; c < M; c += G) dscores[c * dsc + n0 + s] = (T)tile[s * (M | 1) + c];
            __syncthreads();
            continue;
        }
        if (!there) continue;
        T* const row = dscores + n * dsn;
#pragma unroll
        for (int v = 0; v < E / VEC; ++v) {
            const int c0 = route_component<T, G, E>(v * VEC, j);
            if (dsc == 1 && c0 + VEC <= M) {
                Pack q;
#pragma unroll
                for (int i = 0; i < VEC; ++i) q.v[i] = (T)d[v * VEC + i];
                store_bytes(row + c0, q);
            } else {
#pragma unroll
                for (int i = 0; i < VEC; ++i)
                    if (c0 + i < M) row[(c0 + i) * dsc] = (T)d[v * VEC + i];
            }
        }
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] += d[e];
    }
    if (!partial) return;
    constexpr int WAVES = NT / 64;
    __shared__ float sums[WAVES][G * E];
    static_assert(sizeof(sums) == route_sums_bytes<G, E, STAGED>, "what the launch allows for");
#pragma unroll
    for (int e = 0; e < E; ++e) {
        float v = acc[e];
#pragma unroll
        for (int o = 32; o >= G; o >>= 1) v += __shfl_xor(v, o, 64);
        if ((threadIdx.x & 63) < G) sums[threadIdx.x >> 6][route_component<T, G, E>(e, j)] = v;
    }
    __syncthreads();
    for (int c = threadIdx.x; c < M; c += NT) {
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v += sums[w][c];
        partial[(size_t)blockIdx.x * M + c] = v;
    }
}

// The same with a sample to a lane and up to MOST components in registers.  The gradients of a component are summed over the
// lanes by folding: a step adds two halves of the lanes and keeps of every pair of components one in each half, so that 64
// components take 63 additions, not 64 times 6, and lane l is left with the sum of component l (16: with that of l % 16).
// 262144 samples of 64 components: 45 to 47 us, 3.0 TB/s read and written.
template <int CTRL>
__device__ __forceinline__ float fold(float a, float b, bool second) {
    return (second ? b : a) + lane_of<CTRL>(second ? a : b);
}
template <int MOST>
__device__ __forceinline__ float fold_lanes(float (&d)[MOST]) {
    const int lane = threadIdx.x & 63;
    if constexpr (MOST == 64) {
#pragma unroll
        for (int c = 0; c < 32; ++c) {
            const uint32_t a = __builtin_bit_cast(uint32_t, d[c]), b = __builtin_bit_cast(uint32_t, d[c + 32]);
            const auto v = __builtin_amdgcn_permlane32_swap(a, b, false, false);
            const uint32_t v0 = v[0], v1 = v[1];
            d[c] = __builtin_bit_cast(float, v0) + __builtin_bit_cast(float, v1);
        }
#pragma unroll
        for (int c = 0; c < 16; ++c) {
            const uint32_t a = __builtin_bit_cast(uint32_t, d[c]), b = __builtin_bit_cast(uint32_t, d[c + 16]);
            const auto v = __builtin_amdgcn_permlane16_swap(a, b, false, false);
            const uint32_t v0 = v[0], v1 = v[1];
            d[c] = __builtin_bit_cast(float, v0) + __builtin_bit_cast(float, v1);
        }
    }
    // (partners: rotated by eight, mirrored in eight, mirrored in four, neighbours)
#pragma unroll
    for (int c = 0; c < 8; ++c) d[c] = fold<0x128>(d[c], d[c + 8], lane & 8);
#pragma unroll
    for (int c = 0; c < 4; ++c) d[c] = fold<0x141>(d[c], d[c + 4], lane & 4);
#pragma unroll
    for (int c = 0; c < 2; ++c) d[c] = fold<0x1B>(d[c], d[c + 2], lane & 2);
    float r = fold<0xB1>(d[0], d[1], lane & 1);
    if constexpr (MOST == 16) {
        r += __shfl_xor(r, 16, 64);
        r += __shfl_xor(r, 32, 64);
    }
    return r;
}

template <class T, class K, int TOP, int MOST>
__global__ __launch_bounds__(256) void k_route_backward_columns(const T* __restrict__ p, int64_t sc, const float* __restrict__ coef,
                                                                int M, int64_t N, int top, int renormalise,
                                                                const int32_t* __restrict__ ids, const float* __restrict__ weights,
                                                                const float* __restrict__ dweights, const float* __restrict__ dlogp,
                                                                T* __restrict__ dscores, int64_t dsc, float* __restrict__ partial) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float acc = 0.f;                                            // of component lane % MOST, over the wave's samples
    for (int64_t n0 = (int64_t)blockIdx.x * 256; n0 < N; n0 += (int64_t)gridDim.x * 256) {
        const bool there = n0 + threadIdx.x < N;
        const int64_t n = there ? n0 + threadIdx.x : N - 1;
        float d[MOST];
#pragma unroll
        for (int c = 0; c < MOST; ++c) d[c] = to_float(p[n + min(c, M - 1) * sc]);
        K m = (K)-INFINITY;
#pragma unroll
        for (int c = 0; c < MOST; ++c)
            if (c < M) m = Larger{}(m, route_sum<K>(d[c], coef, c));
        const bool dead = !(m > (K)-INFINITY);
        float part[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) part[i] = 0.f;
#pragma unroll
        for (int c = 0; c < MOST; ++c) {
            d[c] = c < M ? route_exp(route_sum<K>(d[c], coef, c), m) : 0.f;
            part[c % 8] += d[c];
        }
        const float z = ((part[0] + part[1]) + (part[2] + part[3])) + ((part[4] + part[5]) + (part[6] + part[7]));
        int id[TOP];
        float add[TOP], a = 0.f;
#pragma unroll
        for (int s = 0; s < TOP; ++s) {
            id[s] = s < top && dweights ? ids[n * top + s] : -1;
            add[s] = id[s] >= 0 ? weights[n * top + s] * dweights[n * top + s] : 0.f;
            a += add[s];
        }
        if (renormalise) {
#pragma unroll
            for (int s = 0; s < TOP; ++s)
                if (id[s] >= 0) add[s] = weights[n * top + s] * (dweights[n * top + s] - a);
        }
        const float dl = dlogp ? dlogp[n] : 0.f;
        const float scale = (renormalise ? dl : dl - a) / z;
#pragma unroll
        for (int c = 0; c < MOST; ++c) {
            float v = d[c] * scale;
#pragma unroll
            for (int s = 0; s < TOP; ++s) v += id[s] == c ? add[s] : 0.f;
            d[c] = dead || !there ? 0.f : v;
            if (there && c < M) dscores[n + c * dsc] = (T)d[c];
        }
        if (partial) acc += fold_lanes<MOST>(d);
    }
    if (!partial) return;
    __shared__ float sums[4][MOST];
    if (lane < MOST) sums[wave][lane] = acc;
    __syncthreads();
    for (int c = threadIdx.x; c < M; c += 256)
        partial[(size_t)blockIdx.x * M + c] = (sums[0][c] + sums[1][c]) + (sums[2][c] + sums[3][c]);
}

// dcoef[c] = sum of the rows of `partial`, in float64: a workgroup has 32 columns and 32 interleaved shares of the rows
__global__ __launch_bounds__(1024) void k_route_coef(const float* __restrict__ partial, int rows, int M,
                                                    float* __restrict__ dcoef) {
    __shared__ double sums[32][33];
    const int x = threadIdx.x & 31, share = threadIdx.x >> 5, c = blockIdx.x * 32 + x;
    double v = 0.0;
    if (c < M) {
#pragma unroll 8
        for (int r = share; r < rows; r += 32) v += (double)partial[(size_t)r * M + c];
    }
    sums[share][x] = v;
    __syncthreads();
    if (share == 0 && c < M) {
        double d = 0.0;
        for (int r = 0; r < 32; ++r) d += sums[r][x];
        dcoef[c] = (float)d;
    }
}

// Lanes per sample: as many as selections at least, and at most 16 components to a lane.  Measured with rows of float32 scores
// and coefficients, four selections, us without / with gradient, by components to a lane,
//                  16000 samples                                       500 samples
//   components     2           4           8           16              2          4          8          16
//   32             4.1 / 7.1   3.8 / 6.6   4.1 / 7.6   4.0 / 7.9       3.1 / 5.7  3.3 / 6.1  3.7 / 6.9  3.7 / 7.1
//   64             6.0 / 10.2  4.7 / 8.2   4.5 / 7.9   5.7 / 10.4      3.5 / 6.0  3.3 / 6.5  3.9 / 7.3  5.2 / 9.7
//   128            10.1 / 16.2 7.2 / 11.7  6.0 / 10.2  6.5 / 11.3      3.8 / 6.3  3.8 / 6.9  4.0 / 7.4  5.5 / 9.7
//   256            12.5 / 20.3 12.0 / 20.1 9.7 / 15.5  9.1 / 15.2      4.2 / 6.8  4.4 / 6.7  4.6 / 7.3  5.6 / 9.3
// The rule is that of many samples; a few hundred of more than 64 components would do better with fewer to a lane.
int route_lanes(int M, int top) {
    const int most = M <= 64 ? 4 : M <= 128 ? 8 : 16;                 // components to a lane
    int G = 4;
    while (G < 64 && (G < top || G * most < M)) G *= 2;
    return G;
}

// Which kernel takes scores whose samples are next to each other (sn = 1).  Measured with log coefficients and two selections, us
// without / with gradient (of weights and log-density),
//   components                     samples: 8192       65536         131072         262144
//   16     groups of lanes, directly      3.5 / 6.7    4.5 / 9.2     5.9 / 11.5     9.1 / 18.2
//          a lane per sample              4.4 / 8.8    4.6 / 9.7     5.5 / 10.8     7.2 / 17.2
//   24     groups of lanes, directly      3.4 / 6.5    6.1 / 11.6    9.2 / 16.0     15.7 / 30.6
//          groups of lanes, through LDS   3.6 / 7.0    5.8 / 14.0    9.3 / 21.6     15.7 / 50.5
//          a lane per sample              6.3 / 18.8   6.6 / 19.7    7.9 / 22.9     11.9 / 36.5
//   64     groups of lanes, directly      4.2 / 8.0    14.5 / 28.1   27.5 / 53.4    49.4 / 93.4
//          groups of lanes, through LDS   4.3 / 7.9    10.7 / 21.5   21.9 / 39.7    41.7 / 71.7
//          a lane per sample              11.3 / 22.8  11.2 / 25.1   13.7 / 30.3    23.3 / 47.4
//   256    groups of lanes, directly      9.5 / 17.9   52 / 101      98 / 203       200 / 546
//          groups of lanes, through LDS   8.1 / 14.3   44 / 60       83 / 127       173 / 291
//   1024   groups of lanes, directly      56 / 99      357 / 1067
//          groups of lanes, through LDS   35 / 46      223 / 451
// A lane per sample waits for one chain of loads and needs every compute unit full of waves; a wide row of few components
// is read well enough directly.  The rule is the same with gradient and without; of 17 to 32 components, whose lane per sample
// goes through 64, the gradient alone would do better directly at any number of samples.
bool route_by_columns(const Scores& a, int top) {
    return a.sn == 1 && a.M <= ROUTE_COLUMNS_MOST && top <= 4 && a.N >= (a.M <= 16 ? 256 : 512) * EINET_NUM_CUS;
}
bool route_staged(const Scores& a) { return a.sn == 1 && a.sc != 1 && a.M > 16 && a.N >= 32 * EINET_NUM_CUS; }
template <int G> constexpr bool ROUTE_CAN_STAGE = G > 4;               // (four lanes have up to 16 components)
template <int G> size_t route_tile_bytes(int M) { return sizeof(float) * ROUTE_STAGE<G> * (size_t)(M | 1); }
// Dynamic LDS of a workgroup that has `own` bytes besides: beyond 64 KiB in all the kernel has to be allowed it (the scores of
// 512 components, their gradient for 257 to 512 and for 1024).
template <class Kernel>
void allow_tile(Kernel kernel, size_t tile, size_t own) {
    if (tile + own > 65536) allow_dynamic_lds(kernel, tile);
}

// Workgroups of the gradient, which is the rows of its workspace.  A handful of samples are one workgroup's, whose sums are
// the gradient of the coefficients: no second launch and no workspace.  Two to a compute unit, four where many samples are read
// directly: the loads of a wave's next samples wait for its last ones there (262144 rows of 64: 35 us instead of 54, 100000 of 128
// 25 instead of 35; through LDS 262144 x 100 took 103 instead of 98).
int route_backward_groups(int M, int64_t N, bool directly) {
    if (N <= (M <= 64 ? 32 : 8)) return 1;
    const int64_t tiles = (N + 3) / 4;               // (a workgroup has four samples at least)
    const int most = (directly && N >= 256 * EINET_NUM_CUS ? 4 : 2) * EINET_NUM_CUS;
    return (int)(tiles < most ? tiles : most);
}

// f(std::integral_constant<int, G>, std::integral_constant<int, E>) for the lanes and components per lane of M, top
template <class F>
void route_variant(int M, int top, F&& f) {
    const int G = route_lanes(M, top), E = (M + G - 1) / G;
#define EINET_E(GG, EE) if (E <= EE) { f(std::integral_constant<int, GG>{}, std::integral_constant<int, EE>{}); return; }
    switch (G) {
    case 4: EINET_E(4, 2) EINET_E(4, 4) return;
    case 8: EINET_E(8, 4) return;
    case 16: EINET_E(16, 4) EINET_E(16, 8) EINET_E(16, 16) return;
    case 32: EINET_E(32, 16) return;
    case 64: EINET_E(64, 16) return;
    }
#undef EINET_E
}

// f(T{}) for an element type
template <class F>
void with_type(int type, F&& f) {
    if (type == ROW_FLOAT32) f(float{});
    else if (type == ROW_BFLOAT16) f(__bf16{});
    else f(_Float16{});
}

// ------------------------------------------------------------------------------------------------------- sorting
//
// Stable counting sort of slots by component: first[c] slots belong to components below c, place[i] is slot i's position,
// -1 for a slot without a component.  Block b has the b-th stretch of the slots and wave w of it the w-th stretch of that.
// A slot's position: the slots of lower components, those of its own in the blocks and waves before, and its rank among
// those of the wave.  Few slots are one workgroup's; more are counted in a first launch, one row of counts per block.
// Latency bounds both: 1024 slots of 128 components take 4.4 us, 32768 8.3 us (30 in one workgroup), a million 25 us, where
// the 64 workgroups do.
// One workgroup against two launches: 4096 slots 6.1 and 6.5 us, 6000 slots 7.5 and 6.9.  At most 64, 128 and 256 workgroups (64
// components): 131072 slots 9.8, 11.7 and 11.6 us, 262144 11.7, 12.7 and 17.4, a million 23, 19 and 21, four million 72, 48 and 36:
// every workgroup reads the counts of all, which 64 keep short for up to some half a million slots.
constexpr int SORT_WAVES = 16;
constexpr int SORT_ONE_BLOCK = 4096, SORT_MOST_BLOCKS = 64;

int sort_blocks(int64_t slots) {
    if (slots <= SORT_ONE_BLOCK) return 1;
    const int64_t b = (slots + 1023) / 1024;
    return (int)(b < SORT_MOST_BLOCKS ? b : SORT_MOST_BLOCKS);
}
// slots of a block and of a wave: whole steps of a wave
__host__ __device__ inline int64_t sort_per_wave(int64_t slots, int blocks) {
    const int64_t waves = (int64_t)blocks * SORT_WAVES;
    return ((slots + waves - 1) / waves + 63) & ~(int64_t)63;
}

__device__ __forceinline__ uint64_t same_key_lanes(int key, int bits) {
    uint64_t same = ~0ull;
    for (int b = 0; b < bits; ++b) {
        const bool bit = (key >> b) & 1;
        const uint64_t set = __ballot(bit);
        same &= bit ? set : ~set;
    }
    return same;
}

// Orders the LDS accesses of one wave's lanes: what a lane has read or written before is done for the others behind it.
__device__ __forceinline__ void wave_lds_fence() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

__global__ __launch_bounds__(64 * SORT_WAVES) void k_sort_count(const int32_t* __restrict__ ids, int64_t slots, int M,
                                                                int32_t* __restrict__ counts) {
    __shared__ int32_t count[ROUTE_MAX_COMPONENTS];
    for (int c = threadIdx.x; c < M; c += 64 * SORT_WAVES) count[c] = 0;
    __syncthreads();
    const int64_t per = sort_per_wave(slots, gridDim.x) * SORT_WAVES, lo = blockIdx.x * per, hi = lo + per < slots ? lo + per : slots;
    for (int64_t i = lo + threadIdx.x; i < hi; i += 64 * SORT_WAVES) {
        const int c = ids[i];
        if ((unsigned)c < (unsigned)M) atomicAdd(&count[c], 1);
    }
    __syncthreads();
    for (int c = threadIdx.x; c < M; c += 64 * SORT_WAVES) counts[blockIdx.x * M + c] = count[c];
}

// counts: [gridDim.x][M], not read by a single block
__global__ __launch_bounds__(64 * SORT_WAVES) void k_sort(const int32_t* __restrict__ ids, int64_t slots, int M, int bits,
                                                          const int32_t* __restrict__ counts, int32_t* __restrict__ first,
                                                          int32_t* __restrict__ place) {
    extern __shared__ int32_t count[];                       // [SORT_WAVES][M], then [SORT_WAVES] sums of the scan
    int32_t* const wave_total = count + SORT_WAVES * M;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, blocks = gridDim.x;
    for (int i = tid; i < SORT_WAVES * M; i += blockDim.x) count[i] = 0;
    __syncthreads();
    const int64_t per = sort_per_wave(slots, blocks), at0 = (blockIdx.x * (int64_t)SORT_WAVES + wave) * per;
    const int64_t lo = at0 < slots ? at0 : slots, hi = lo + per < slots ? lo + per : slots;
    for (int64_t i = lo + lane; i < hi; i += 64) {
        const int c = ids[i];
        if ((unsigned)c < (unsigned)M) atomicAdd(&count[wave * M + c], 1);
    }
    // thread c: the slots of component c, in all blocks and in those before this one
    int total = 0, before_block = 0;
    if (blocks > 1 && tid < M) {
#pragma unroll 8
        for (int b = 0; b < blocks; ++b) {
            const int v = counts[b * M + tid];
            total += v;
            before_block += b < (int)blockIdx.x ? v : 0;
        }
    }
    __syncthreads();
    if (blocks == 1 && tid < M)
        for (int w = 0; w < SORT_WAVES; ++w) total += count[w * M + tid];
    int run = total;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const int v = __shfl_up(run, o, 64);
        if (lane >= o) run += v;
    }
    if (lane == 63) wave_total[wave] = run;
    __syncthreads();
    int before = 0;
    for (int w = 0; w < wave; ++w) before += wave_total[w];
    run += before;
    if (tid < M) {
        if (blockIdx.x == 0) {
            first[tid] = run - total;
            if (tid == M - 1) first[M] = run;
        }
        int at = run - total + before_block;
        for (int w = 0; w < SORT_WAVES; ++w) {
            const int v = count[w * M + tid];
            count[w * M + tid] = at;
            at += v;
        }
    }
    __syncthreads();
    for (int64_t i0 = lo; i0 < hi; i0 += 64) {
        const int64_t i = i0 + lane;
        int c = i < hi ? ids[i] : -1;
        if ((unsigned)c >= (unsigned)M) c = M;               // (a key of its own: bits covers 0 .. M)
        const uint64_t same = same_key_lanes(c, bits);
        const int rank = __popcll(same & ((1ull << lane) - 1));
        int at = -1;
        if (c < M) at = count[wave * M + c] + rank;
        wave_lds_fence();
        if (c < M && rank == 0) count[wave * M + c] += __popcll(same);
        wave_lds_fence();
        if (i < hi) place[i] = at;
    }
}

// ------------------------------------------------------------------------------------------- rows there and back
//
// A row is a number of units of up to 16 bytes (the last may be shorter; loads and stores of 16 bytes need no more than the
// elements' alignment).  L lanes share a sample, each with one unit of every L: a tile.  A tile's work is one item, so that
// a few long rows spread over many workgroups too; rows shorter than half a wave's units share a wave.  Memory bounds all
// three kernels: 8192 samples with four rows of 2048 bf16 each, with gradients, take 177 us for 672 MB (3.8 TB/s; a copy
// reaches 4.9).  Two units to a lane of longer rows: 187 us, four 193; four slots in flight instead of two: 3 us less.
template <class T> constexpr int UNIT = 16 / (int)sizeof(T);
template <class T> struct Unit { T v[UNIT<T>]; };

template <class T>
__device__ __forceinline__ Unit<T> load_unit(const T* p, int64_t left) {
    if (left >= UNIT<T>) return load_bytes<Unit<T>>(p);
    Unit<T> u;
#pragma unroll
    for (int i = 0; i < UNIT<T>; ++i) u.v[i] = i < left ? p[i] : T{};
    return u;
}
template <class T>
__device__ __forceinline__ void store_unit(T* p, int64_t left, const Unit<T>& u) {
    if (left >= UNIT<T>) {
        store_bytes(p, u);
        return;
    }
#pragma unroll
    for (int i = 0; i < UNIT<T>; ++i)
        if (i < left) p[i] = u.v[i];
}

// The item of a lane: its sample and the column of its unit.
template <class T, int L>
__device__ __forceinline__ bool row_item(int64_t N, int64_t H, int tiles, int64_t& n, int64_t& k) {
    uint32_t item = blockIdx.x * (256 / L) + threadIdx.x / L;        // (a launch has fewer than 2^32 lanes)
    if constexpr (L == 64) item = (uint32_t)__builtin_amdgcn_readfirstlane((int)item);
    const uint32_t i = tiles == 1 ? item : item / (uint32_t)tiles;
    n = i;
    k = ((int64_t)(item - i * (uint32_t)tiles) * L + threadIdx.x % L) * UNIT<T>;
    return n < N && k < H;
}

template <class T, int L>
__global__ __launch_bounds__(256) void k_dispatch(const T* __restrict__ x, int64_t H, int64_t x_stride, int64_t N, int tiles, int top,
                                                  const int32_t* __restrict__ place, T* __restrict__ out, int64_t out_stride,
                                                  int64_t out_rows) {
    int64_t n, k;
    if (!row_item<T, L>(N, H, tiles, n, k)) return;
    const Unit<T> u = load_unit(x + n * x_stride + k, H - k);
    for (int s = 0; s < top; ++s) {
        const int64_t at = place[n * top + s];
        if (at >= 0 && at < out_rows) store_unit(out + at * out_stride + k, H - k, u);
    }
}

// Slots are taken S at a time, their loads in flight together.
template <class T, int L, int S>
__global__ __launch_bounds__(256) void k_combine(const T* __restrict__ rows, int64_t H, int64_t stride, int64_t n_rows,
                                                 const int32_t* __restrict__ place, const float* __restrict__ weights, int64_t N,
                                                 int tiles, int top, T* __restrict__ out, int64_t out_stride) {
    int64_t n, k;
    if (!row_item<T, L>(N, H, tiles, n, k)) return;
    float acc[UNIT<T>];
#pragma unroll
    for (int c = 0; c < UNIT<T>; ++c) acc[c] = 0.f;
    for (int s0 = 0; s0 < top; s0 += S) {
        Unit<T> u[S];
        float w[S];
        bool has[S];
#pragma unroll
        for (int q = 0; q < S; ++q) {
            const int64_t slot = n * top + min(s0 + q, top - 1);
            const int64_t at = place[slot];
            has[q] = s0 + q < top && at >= 0 && at < n_rows;
            w[q] = weights ? weights[slot] : 1.f;
            if (has[q]) u[q] = load_unit(rows + at * stride + k, H - k);
        }
#pragma unroll
        for (int q = 0; q < S; ++q)
            if (has[q]) {
#pragma unroll
                for (int c = 0; c < UNIT<T>; ++c) acc[c] = fmaf(w[q], to_float(u[q].v[c]), acc[c]);
            }
    }
    Unit<T> o;
#pragma unroll
    for (int c = 0; c < UNIT<T>; ++c) o.v[c] = (T)acc[c];
    store_unit(out + n * out_stride + k, H - k, o);
}

// The rows of a sample are gone through by L lanes (256: the whole workgroup), S slots at a time: the gradient of the
// output is read once for them, every row once.  A workgroup for rows of more than 64 units instead of a wave: 8192 x 4 rows of
// 2048 bf16 57 us instead of 61.
template <class T, int L, int S>
__global__ __launch_bounds__(256) void k_combine_backward(const T* __restrict__ dout, int64_t dout_stride,
                                                          const T* __restrict__ rows, int64_t H, int64_t stride, int64_t n_rows,
                                                          const int32_t* __restrict__ place, const float* __restrict__ weights,
                                                          int64_t N, int top, T* __restrict__ drows, int64_t drows_stride,
                                                          float* __restrict__ dweights) {
    const int64_t n = (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L;
    const int j = threadIdx.x % L;
    if (n >= N) return;
    const T* const g = dout + n * dout_stride;
    for (int s0 = 0; s0 < top; s0 += S) {
        int64_t at[S];
        float w[S], dot[S];
        bool has[S];
#pragma unroll
        for (int q = 0; q < S; ++q) {
            const int64_t slot = n * top + min(s0 + q, top - 1);
            at[q] = place[slot];
            has[q] = s0 + q < top && at[q] >= 0 && at[q] < n_rows;
            w[q] = weights[slot];
            dot[q] = 0.f;
        }
        for (int64_t k = (int64_t)j * UNIT<T>; k < H; k += L * UNIT<T>) {
            const Unit<T> d = load_unit(g + k, H - k);
            Unit<T> u[S];
#pragma unroll
            for (int q = 0; q < S; ++q)
                if (has[q]) u[q] = load_unit(rows + at[q] * stride + k, H - k);
#pragma unroll
            for (int q = 0; q < S; ++q)
                if (has[q]) {
                    Unit<T> o;
#pragma unroll
                    for (int c = 0; c < UNIT<T>; ++c) {
                        const float v = to_float(d.v[c]);
                        dot[q] = fmaf(v, to_float(u[q].v[c]), dot[q]);
                        o.v[c] = (T)(w[q] * v);
                    }
                    store_unit(drows + at[q] * drows_stride + k, H - k, o);
                }
        }
#pragma unroll
        for (int q = 0; q < S; ++q) dot[q] = group_reduce<(L < 64 ? L : 64)>(dot[q], Plus{});
        if constexpr (L == 256) {
            __shared__ float part[4][S];
            __syncthreads();
            if ((threadIdx.x & 63) == 0) {
#pragma unroll
                for (int q = 0; q < S; ++q) part[threadIdx.x >> 6][q] = dot[q];
            }
            __syncthreads();
#pragma unroll
            for (int q = 0; q < S; ++q) dot[q] = (part[0][q] + part[1][q]) + (part[2][q] + part[3][q]);
        }
        if (j == 0) {
#pragma unroll
            for (int q = 0; q < S; ++q)
                if (s0 + q < top) dweights[n * top + s0 + q] = dot[q];
        }
    }
}

// f(integral_constant<L>) for rows of `units` units
template <class F>
void row_lanes(int64_t units, F&& f) {
    if (units <= 1) f(std::integral_constant<int, 1>{});
    else if (units <= 2) f(std::integral_constant<int, 2>{});
    else if (units <= 4) f(std::integral_constant<int, 4>{});
    else if (units <= 8) f(std::integral_constant<int, 8>{});
    else if (units <= 16) f(std::integral_constant<int, 16>{});
    else if (units <= 32) f(std::integral_constant<int, 32>{});
    else f(std::integral_constant<int, 64>{});
}

}  // namespace

// f(integral_constant<TOP>, integral_constant<MOST>) for the selections and components of a lane's sample
template <class F>
void columns_variant(int M, int top, F&& f) {
    auto with = [&](auto most) {
        if (top == 1) f(std::integral_constant<int, 1>{}, most);
        else if (top == 2) f(std::integral_constant<int, 2>{}, most);
        else f(std::integral_constant<int, 4>{}, most);
    };
    if (M <= 16) with(std::integral_constant<int, 16>{});
    else with(std::integral_constant<int, ROUTE_COLUMNS_MOST>{});
}

// f(T{}, K{}) for the types of the scores and of their sums with the coefficients
template <class F>
void route_types(const Scores& a, F&& f) {
    with_type(a.type, [&](auto t) {
        if (a.coef) f(t, double{});
        else f(t, float{});
    });
}

void launch_route(const Scores& a, int top, bool renormalise, int32_t* ids, float* weights, float* logp, hipStream_t s) {
    if (a.N == 0) return;
    const int re = renormalise ? 1 : 0;
    route_types(a, [&](auto t, auto k) {
        using T = decltype(t);
        using K = decltype(k);
        const T* const p = static_cast<const T*>(a.p);
        if (route_by_columns(a, top)) {
            const dim3 grid((unsigned)((a.N + 255) / 256));
            columns_variant(a.M, top, [&](auto most, auto components) {
                hipLaunchKernelGGL((k_route_columns<T, K, decltype(most)::value, decltype(components)::value>), grid, dim3(256), 0, s, p,
                                   a.sc, a.coef, a.M, a.N, top, re, ids, weights, logp);
            });
            return;
        }
        route_variant(a.M, top, [&](auto g, auto e) {
            constexpr int G = decltype(g)::value, E = decltype(e)::value;
            auto go = [&](auto staged) {
                constexpr bool STAGED = decltype(staged)::value;
                constexpr int NT = ROUTE_THREADS<G, STAGED>, S = NT / G;
                if constexpr (STAGED) allow_tile(k_route<T, K, G, E, STAGED>, route_tile_bytes<G>(a.M), 0);
                row_batches(a.N, G, [&](int64_t n0, int64_t n) {
                    hipLaunchKernelGGL((k_route<T, K, G, E, STAGED>), dim3((unsigned)((n + S - 1) / S)), dim3(NT),
                                       STAGED ? route_tile_bytes<G>(a.M) : 0, s, p + n0 * a.sn, a.sc, a.sn, a.coef, a.M, n, top, re,
                                       ids + n0 * top, weights + n0 * top, logp + n0);
                });
            };
            if constexpr (ROUTE_CAN_STAGE<G>)
                if (route_staged(a)) return go(std::true_type{});
            go(std::false_type{});
        });
    });
}

size_t route_backward_workspace(int M, int64_t N) {
    const int groups = route_backward_groups(M, N, true);
    return groups > 1 ? sizeof(float) * (size_t)groups * M : 0;
}

void launch_route_backward(const Scores& a, int top, bool renormalise, const int32_t* ids, const float* weights,
                           const float* dweights, const float* dlogp, void* dscores, int64_t dsc, int64_t dsn, float* dcoef,
                           void* workspace, hipStream_t s) {
    const bool by_columns = route_by_columns(a, top) && dsn == 1, staged_rows = route_staged(a) && dsn == 1;
    const int groups = route_backward_groups(a.M, a.N, !by_columns && !staged_rows), re = renormalise ? 1 : 0;
    float* const partial = !dcoef ? nullptr : groups > 1 ? static_cast<float*>(workspace) : dcoef;
    if (a.N > 0)
        route_types(a, [&](auto t, auto k) {
            using T = decltype(t);
            using K = decltype(k);
            const T* const p = static_cast<const T*>(a.p);
            T* const d = static_cast<T*>(dscores);
            if (by_columns) {
                columns_variant(a.M, top, [&](auto most, auto components) {
                    hipLaunchKernelGGL((k_route_backward_columns<T, K, decltype(most)::value, decltype(components)::value>), dim3(groups),
                                       dim3(256), 0, s, p, a.sc, a.coef, a.M, a.N, top, re, ids, weights, dweights, dlogp, d, dsc, partial);
                });
                return;
            }
            route_variant(a.M, top, [&](auto g, auto e) {
                constexpr int G = decltype(g)::value, E = decltype(e)::value;
                auto go = [&](auto staged) {
                    constexpr bool STAGED = decltype(staged)::value;
                    if constexpr (STAGED)
                        allow_tile(k_route_backward<T, K, G, E, STAGED>, route_tile_bytes<G>(a.M), route_sums_bytes<G, E, STAGED>);
                    hipLaunchKernelGGL((k_route_backward<T, K, G, E, STAGED>), dim3(groups), dim3(ROUTE_THREADS<G, STAGED>),
                                       STAGED ? route_tile_bytes<G>(a.M) : 0, s, p, a.sc, a.sn, a.coef, a.M, a.N, top, re, ids, weights,
                                       dweights, dlogp, d, dsc, dsn, partial);
                };
                if constexpr (ROUTE_CAN_STAGE<G>)
                    if (staged_rows) return go(std::true_type{});
                go(std::false_type{});
            });
        });
    if (dcoef && (groups > 1 || a.N == 0))
        hipLaunchKernelGGL(k_route_coef, dim3((a.M + 31) / 32), dim3(1024), 0, s, partial, a.N > 0 ? groups : 0, a.M, dcoef);
}

size_t sort_workspace(int64_t slots, int M) {
    const int blocks = sort_blocks(slots);
    return blocks > 1 ? sizeof(int32_t) * (size_t)blocks * M : 0;
}

void launch_sort(const int32_t* ids, int64_t slots, int M, int32_t* first, int32_t* place, void* workspace, hipStream_t s) {
    int bits = 1;
    while ((1 << bits) <= M) ++bits;
    const int blocks = sort_blocks(slots);
    int32_t* const counts = static_cast<int32_t*>(workspace);
    if (blocks > 1) hipLaunchKernelGGL(k_sort_count, dim3(blocks), dim3(64 * SORT_WAVES), 0, s, ids, slots, M, counts);
    const size_t lds = sizeof(int32_t) * (size_t)(SORT_WAVES * M + SORT_WAVES);
    if (lds > 65536) allow_dynamic_lds(k_sort, lds);
    hipLaunchKernelGGL(k_sort, dim3(blocks), dim3(64 * SORT_WAVES), lds, s, ids, slots, M, bits, counts, first, place);
}

void launch_dispatch(const void* x, int64_t row_bytes, int64_t x_stride, int64_t N, int top, const int32_t* place, void* out,
                     int64_t out_stride, int64_t out_rows, hipStream_t s) {
    if (N == 0 || row_bytes == 0 || out_rows == 0) return;
    const uint64_t any = (uint64_t)row_bytes | (uint64_t)x_stride | (uint64_t)out_stride | reinterpret_cast<uintptr_t>(x) |
                         reinterpret_cast<uintptr_t>(out);
    auto go = [&](auto t) {
        using T = decltype(t);
        constexpr int64_t e = sizeof(T);
        const int64_t H = row_bytes / e, units = (H + UNIT<T> - 1) / UNIT<T>;
        row_lanes(units, [&](auto l) {
            constexpr int L = decltype(l)::value;
            const int64_t tiles = (units + L - 1) / L;
            row_batches(N, tiles * L, [&](int64_t n0, int64_t n) {
                hipLaunchKernelGGL((k_dispatch<T, L>), dim3((unsigned)((n * tiles + 256 / L - 1) / (256 / L))), dim3(256), 0, s,
                                   static_cast<const T*>(x) + n0 * (x_stride / e), H, x_stride / e, n, (int)tiles, top,
                                   place + n0 * top, static_cast<T*>(out), out_stride / e, out_rows);
            });
        });
    };
    if (any % 4 == 0) go(uint32_t{});
    else if (any % 2 == 0) go(uint16_t{});
    else go(uint8_t{});
}

// f(integral_constant<S>) for the slots whose rows are in flight together
template <class F>
void slots_together(int top, F&& f) {
    if (top == 1) f(std::integral_constant<int, 1>{});
    else if (top == 2) f(std::integral_constant<int, 2>{});
    else f(std::integral_constant<int, 4>{});
}

void launch_combine(const void* rows, int type, int64_t H, int64_t stride, int64_t n_rows, const int32_t* place,
                    const float* weights, int64_t N, int top, void* out, int64_t out_stride, hipStream_t s) {
    if (N == 0 || H == 0) return;
    with_type(type, [&](auto t) {
        using T = decltype(t);
        const int64_t units = (H + UNIT<T> - 1) / UNIT<T>;
        row_lanes(units, [&](auto l) {
            constexpr int L = decltype(l)::value;
            const int64_t tiles = (units + L - 1) / L;
            row_batches(N, tiles * L, [&](int64_t n0, int64_t n) {
                slots_together(top, [&](auto q) {
                    hipLaunchKernelGGL((k_combine<T, L, decltype(q)::value>), dim3((unsigned)((n * tiles + 256 / L - 1) / (256 / L))),
                                       dim3(256), 0, s, static_cast<const T*>(rows), H, stride, n_rows, place + n0 * top,
                                       weights ? weights + n0 * top : nullptr, n, (int)tiles, top,
                                       static_cast<T*>(out) + n0 * out_stride, out_stride);
                });
            });
        });
    });
}

void launch_combine_backward(const void* dout, int64_t dout_stride, const void* rows, int type, int64_t H, int64_t stride,
                             int64_t n_rows, const int32_t* place, const float* weights, int64_t N, int top, void* drows,
                             int64_t drows_stride, float* dweights, hipStream_t s) {
    if (N == 0) return;
    with_type(type, [&](auto t) {
        using T = decltype(t);
        const int64_t units = (H + UNIT<T> - 1) / UNIT<T>;
        auto go = [&](auto l) {
            constexpr int L = decltype(l)::value;
            row_batches(N, L, [&](int64_t n0, int64_t n) {
                slots_together(top, [&](auto q) {
                    hipLaunchKernelGGL((k_combine_backward<T, L, decltype(q)::value>), dim3((unsigned)((n + 256 / L - 1) / (256 / L))),
                                       dim3(256), 0, s, static_cast<const T*>(dout) + n0 * dout_stride, dout_stride,
                                       static_cast<const T*>(rows), H, stride, n_rows, place + n0 * top, weights + n0 * top, n, top,
                                       static_cast<T*>(drows), drows_stride, dweights + n0 * top);
                });
            });
        };
        if (units > 64) go(std::integral_constant<int, 256>{});
        else row_lanes(units, go);
    });
}

}  // namespace einet_impl

// Routing samples to the components of a mixture: the most probable components of every sample with their weights, a
// stable counting sort of the (sample, choice) slots by component, and rows carried to their components and back.
#include "device_common.hpp"
#include "routing.hpp"

namespace einet_impl {

namespace {

template <class T>
__device__ __forceinline__ float to_float(T v) { return (float)v; }

template <int G>
__device__ __forceinline__ double group_max(double v) {
#pragma unroll
    for (int o = G / 2; o >= 1; o >>= 1) v = fmax(v, __shfl_xor(v, o, G));
    return v;
}
template <int G>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
    for (int o = G / 2; o >= 1; o >>= 1) v += __shfl_xor(v, o, G);
    return v;
}

// ---------------------------------------------------------------------------------------------------- routing
//
// With t[c] = score[c] + coef[c], m = max t and z = sum exp(t[c] - m): logp = m + log z, p[c] = exp(t[c] - m) / z.  The
// sums t are formed in float64: log-densities are in the hundreds and thousands and differ by little, and which of two
// is larger must not depend on a rounding.  A component whose t is -inf or NaN is left out.
//
// G lanes share a sample, each with E components in registers (component e * G + lane).

template <class T, int G, int E>
__device__ __forceinline__ double route_load(const T* __restrict__ p, int64_t sc, int64_t sn, const float* __restrict__ coef,
                                             int M, int64_t n, int j, double (&t)[E]) {
    double m = -INFINITY;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const int c = e * G + j;
        double v = -INFINITY;
        if (c < M) {
            v = (double)to_float(p[c * sc + n * sn]);
            if (coef) v += (double)coef[c];
            if (!(v > -INFINITY)) v = -INFINITY;
        }
        t[e] = v;
        m = fmax(m, v);
    }
    return group_max<G>(m);
}

// exp(t - m) of a component, 1 at the maximum (also where both are infinite)
__device__ __forceinline__ float route_exp(double t, double m) { return t == m ? 1.f : expf((float)(t - m)); }

template <class T, int G, int E>
__global__ __launch_bounds__(256) void k_route(const T* __restrict__ p, int64_t sc, int64_t sn, const float* __restrict__ coef,
                                               int M, int64_t N, int top, int renormalise, int32_t* __restrict__ ids,
                                               float* __restrict__ weights, float* __restrict__ logp) {
    const int j = threadIdx.x % G;
    const int64_t n = (int64_t)blockIdx.x * (256 / G) + threadIdx.x / G;
    if (n >= N) return;
    double t[E];
    const double m = route_load<T, G, E>(p, sc, sn, coef, M, n, j, t);
    const bool dead = !(m > -INFINITY);
    float z = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) z += dead ? 0.f : route_exp(t[e], m);
    z = group_sum<G>(z);
    // one selection after the other, the largest of what is left; lane s of the group keeps selection s
    int my_id = -1;
    float my_e = 0.f;
    for (int s = 0; s < top; ++s) {
        double best = -INFINITY;
        int c = 0x7fffffff;
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (t[e] > best) best = t[e], c = e * G + j;
#pragma unroll
        for (int o = G / 2; o >= 1; o >>= 1) {
            const double ob = __shfl_xor(best, o, G);
            const int oc = __shfl_xor(c, o, G);
            if (ob > best || (ob == best && oc < c)) best = ob, c = oc;
        }
        if (!(best > -INFINITY)) break;
        if (j == s) my_id = c, my_e = route_exp(best, m);
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (c == e * G + j) t[e] = -INFINITY;
    }
    const float total = renormalise ? group_sum<G>(my_e) : z;
    if (j < top) {
        ids[n * top + j] = my_id;
        weights[n * top + j] = my_id >= 0 ? my_e / total : 0.f;
    }
    if (j == 0) logp[n] = dead ? -INFINITY : (float)(m + (double)logf(z));
}

// With a = sum_s dw[s] w[s]:
//   d t[c] = p[c] (dlogp - a) + sum_{s: id[s] = c} dw[s] w[s]            (weights p)
//   d t[c] = p[c] dlogp + sum_{s: id[s] = c} w[s] (dw[s] - a)            (weights that sum to one)
// The log-density and the weights are differences and quotients of numbers rounded to float32; m and z come from the
// scores again.  d coef[c] = sum_n d t[c][n]: a lane has the same components for all its samples and adds their gradients
// up in registers; the workgroup's sums go to a row of the workspace, which the second kernel adds up in a fixed order.
template <class T, int G, int E>
__global__ __launch_bounds__(256) void k_route_backward(const T* __restrict__ p, int64_t sc, int64_t sn,
                                                        const float* __restrict__ coef, int M, int64_t N, int top,
                                                        int renormalise, const int32_t* __restrict__ ids,
                                                        const float* __restrict__ weights, const float* __restrict__ dweights,
                                                        const float* __restrict__ dlogp, T* __restrict__ dscores, int64_t dsc,
                                                        int64_t dsn, float* __restrict__ partial) {
    constexpr int S = 256 / G;
    const int j = threadIdx.x % G;
    float acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.f;
    for (int64_t n0 = (int64_t)blockIdx.x * S; n0 < N; n0 += (int64_t)gridDim.x * S) {
        const int64_t n = n0 + threadIdx.x / G;
        if (n >= N) continue;                                   // (whole groups leave together)
        double t[E];
        const double m = route_load<T, G, E>(p, sc, sn, coef, M, n, j, t);
        const bool dead = !(m > -INFINITY);
        float z = 0.f;
        float d[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            d[e] = dead ? 0.f : route_exp(t[e], m);
            z += d[e];
        }
        z = group_sum<G>(z);
        int id = -1;
        float w = 0.f, dw = 0.f;
        if (j < top && dweights) {
            id = ids[n * top + j];
            w = weights[n * top + j];
            dw = dweights[n * top + j];
            if (id < 0) w = dw = 0.f;
        }
        const float a = group_sum<G>(w * dw), dl = dlogp ? dlogp[n] : 0.f;
        const float scale = dead ? 0.f : (renormalise ? dl : dl - a) / z, add = w * (renormalise ? dw - a : dw);
#pragma unroll
        for (int e = 0; e < E; ++e) d[e] *= scale;
        if (dweights)
            for (int s = 0; s < top; ++s) {
                const int c = __shfl(id, s, G);
                const float v = __shfl(add, s, G);
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (c == e * G + j) d[e] += v;
            }
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int c = e * G + j;
            if (c < M) dscores[c * dsc + n * dsn] = (T)d[e];
            acc[e] += d[e];
        }
    }
    if (!partial) return;
    __shared__ float sums[4][G * E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        float v = acc[e];
#pragma unroll
        for (int o = 32; o >= G; o >>= 1) v += __shfl_xor(v, o, 64);
        if ((threadIdx.x & 63) < G) sums[threadIdx.x >> 6][e * G + j] = v;
    }
    __syncthreads();
    for (int c = threadIdx.x; c < M; c += 256)
        partial[(size_t)blockIdx.x * M + c] = (sums[0][c] + sums[1][c]) + (sums[2][c] + sums[3][c]);
}

// dcoef[c] = sum of the rows of `partial`, in float64: 64 columns and four interleaved shares of the rows per workgroup
__global__ __launch_bounds__(256) void k_route_coef(const float* __restrict__ partial, int rows, int M, float* __restrict__ dcoef) {
    __shared__ double sums[4][64];
    const int c = blockIdx.x * 64 + (threadIdx.x & 63), share = threadIdx.x >> 6;
    double v = 0.0;
    if (c < M)
        for (int r = share; r < rows; r += 4) v += (double)partial[(size_t)r * M + c];
    sums[share][threadIdx.x & 63] = v;
    __syncthreads();
    if (share == 0 && c < M) dcoef[c] = (float)((sums[0][threadIdx.x] + sums[1][threadIdx.x]) + (sums[2][threadIdx.x] + sums[3][threadIdx.x]));
}

// Lanes per sample: as many as selections at least, and at most 16 components to a lane.
int route_lanes(int M, int top) {
    int G = 4;
    while (G < 64 && (G < top || G * 4 < M)) G *= 2;
    return G;
}

constexpr int ROUTE_BACKWARD_GROUPS = 1024;          // workgroups of the gradient, which is the rows of its workspace
int route_backward_groups(int M, int64_t N) {
    const int64_t tiles = (N + 3) / 4;               // (a workgroup has four samples at least)
    (void)M;
    return (int)(tiles < ROUTE_BACKWARD_GROUPS ? tiles : ROUTE_BACKWARD_GROUPS);
}

// f(std::integral_constant<int, G>, std::integral_constant<int, E>) for the lanes and components per lane of M, top
template <class F>
void route_variant(int M, int top, F&& f) {
    const int G = route_lanes(M, top), E = (M + G - 1) / G;
#define EINET_E(GG, EE) if (E <= EE) { f(std::integral_constant<int, GG>{}, std::integral_constant<int, EE>{}); return; }
    switch (G) {
    case 4: EINET_E(4, 2) EINET_E(4, 4) return;
    case 8: EINET_E(8, 1) EINET_E(8, 4) return;
    case 16: EINET_E(16, 1) EINET_E(16, 4) return;
    case 32: EINET_E(32, 4) return;
    case 64: EINET_E(64, 4) EINET_E(64, 8) EINET_E(64, 16) return;
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
// -1 for a slot without a component.  Wave w of the workgroup has the w-th stretch of the slots.
constexpr int SORT_WAVES = 16;

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

__global__ __launch_bounds__(64 * SORT_WAVES) void k_sort(const int32_t* __restrict__ ids, int64_t slots, int M, int bits,
                                                          int32_t* __restrict__ first, int32_t* __restrict__ place) {
    extern __shared__ int32_t count[];                       // [SORT_WAVES][M], then [SORT_WAVES] sums of the scan
    int32_t* const wave_total = count + SORT_WAVES * M;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    for (int i = tid; i < SORT_WAVES * M; i += blockDim.x) count[i] = 0;
    __syncthreads();
    const int64_t per = ((slots + SORT_WAVES - 1) / SORT_WAVES + 63) & ~(int64_t)63;
    const int64_t lo = wave * per < slots ? wave * per : slots, hi = lo + per < slots ? lo + per : slots;
    for (int64_t i = lo + lane; i < hi; i += 64) {
        const int c = ids[i];
        if ((unsigned)c < (unsigned)M) atomicAdd(&count[wave * M + c], 1);
    }
    __syncthreads();
    // thread c: components' totals, their running sum over c, then the first position of every wave's share
    int total = 0;
    if (tid < M)
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
        first[tid] = run - total;
        if (tid == M - 1) first[M] = run;
        int at = run - total;
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

template <class U>
__global__ __launch_bounds__(256) void k_dispatch(const char* __restrict__ x, int64_t units, int64_t x_stride, int64_t N, int top,
                                                  const int32_t* __restrict__ place, char* __restrict__ out, int64_t out_stride,
                                                  int64_t out_rows) {
    const int64_t all = N * units;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int64_t n = i / units, k = i - n * units;
        const U v = *reinterpret_cast<const U*>(x + n * x_stride + k * (int64_t)sizeof(U));
        for (int s = 0; s < top; ++s) {
            const int64_t at = place[n * top + s];
            if (at >= 0 && at < out_rows) *reinterpret_cast<U*>(out + at * out_stride + k * (int64_t)sizeof(U)) = v;
        }
    }
}

template <class T>
__global__ __launch_bounds__(256) void k_combine(const T* __restrict__ rows, int64_t H, int64_t stride, int64_t n_rows,
                                                 const int32_t* __restrict__ place, const float* __restrict__ weights, int64_t N,
                                                 int top, T* __restrict__ out, int64_t out_stride) {
    const int64_t all = N * H;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < all; i += (int64_t)gridDim.x * 256) {
        const int64_t n = i / H, k = i - n * H;
        float v = 0.f;
        for (int s = 0; s < top; ++s) {
            const int64_t at = place[n * top + s];
            if (at >= 0 && at < n_rows) v += (weights ? weights[n * top + s] : 1.f) * to_float(rows[at * stride + k]);
        }
        out[n * out_stride + k] = (T)v;
    }
}

template <class T>
__global__ __launch_bounds__(256) void k_combine_backward(const T* __restrict__ dout, int64_t dout_stride,
                                                          const T* __restrict__ rows, int64_t H, int64_t stride, int64_t n_rows,
                                                          const int32_t* __restrict__ place, const float* __restrict__ weights,
                                                          int64_t slots, int top, T* __restrict__ drows, int64_t drows_stride,
                                                          float* __restrict__ dweights) {
    const int lane = threadIdx.x & 63;
    for (int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); i < slots; i += (int64_t)gridDim.x * 4) {
        const int64_t n = i / top, at = place[i];
        float dot = 0.f;
        if (at >= 0 && at < n_rows) {
            const float w = weights[i];
            for (int64_t k = lane; k < H; k += 64) {
                const float g = to_float(dout[n * dout_stride + k]);
                dot += g * to_float(rows[at * stride + k]);
                drows[at * drows_stride + k] = (T)(w * g);
            }
        }
        dot = wave_sum(dot);
        if (lane == 0) dweights[i] = dot;
    }
}

unsigned blocks_for(int64_t work, int64_t per, int64_t most) {
    const int64_t b = (work + per - 1) / per;
    return (unsigned)(b < most ? b : most);
}

}  // namespace

void launch_route(const Scores& a, int top, bool renormalise, int32_t* ids, float* weights, float* logp, hipStream_t s) {
    if (a.N == 0) return;
    with_type(a.type, [&](auto t) {
        using T = decltype(t);
        route_variant(a.M, top, [&](auto g, auto e) {
            constexpr int G = decltype(g)::value, E = decltype(e)::value;
            hipLaunchKernelGGL((k_route<T, G, E>), dim3((unsigned)((a.N + 256 / G - 1) / (256 / G))), dim3(256), 0, s,
                               static_cast<const T*>(a.p), a.sc, a.sn, a.coef, a.M, a.N, top, renormalise ? 1 : 0, ids, weights,
                               logp);
        });
    });
}

size_t route_backward_workspace(int M, int64_t N) { return sizeof(float) * (size_t)route_backward_groups(M, N) * M; }

void launch_route_backward(const Scores& a, int top, bool renormalise, const int32_t* ids, const float* weights,
                           const float* dweights, const float* dlogp, void* dscores, int64_t dsc, int64_t dsn, float* dcoef,
                           void* workspace, hipStream_t s) {
    const int groups = route_backward_groups(a.M, a.N);
    float* const partial = dcoef ? static_cast<float*>(workspace) : nullptr;
    if (a.N > 0)
        with_type(a.type, [&](auto t) {
            using T = decltype(t);
            route_variant(a.M, top, [&](auto g, auto e) {
                constexpr int G = decltype(g)::value, E = decltype(e)::value;
                hipLaunchKernelGGL((k_route_backward<T, G, E>), dim3(groups), dim3(256), 0, s, static_cast<const T*>(a.p), a.sc,
                                   a.sn, a.coef, a.M, a.N, top, renormalise ? 1 : 0, ids, weights, dweights, dlogp,
                                   static_cast<T*>(dscores), dsc, dsn, partial);
            });
        });
    if (dcoef) hipLaunchKernelGGL(k_route_coef, dim3((a.M + 63) / 64), dim3(256), 0, s, partial, groups, a.M, dcoef);
}

size_t sort_workspace(int64_t, int) { return 0; }

void launch_sort(const int32_t* ids, int64_t slots, int M, int32_t* first, int32_t* place, void*, hipStream_t s) {
    int bits = 1;
    while ((1 << bits) <= M) ++bits;
    const size_t lds = sizeof(int32_t) * (size_t)(SORT_WAVES * M + SORT_WAVES);
    allow_dynamic_lds(k_sort, lds);
    hipLaunchKernelGGL(k_sort, dim3(1), dim3(64 * SORT_WAVES), lds, s, ids, slots, M, bits, first, place);
}

void launch_dispatch(const void* x, int64_t row_bytes, int64_t x_stride, int64_t N, int top, const int32_t* place, void* out,
                     int64_t out_stride, int64_t out_rows, hipStream_t s) {
    if (N == 0 || row_bytes == 0) return;
    const uint64_t any = (uint64_t)row_bytes | (uint64_t)x_stride | (uint64_t)out_stride | reinterpret_cast<uintptr_t>(x) |
                         reinterpret_cast<uintptr_t>(out);
    auto go = [&](auto u) {
        using U = decltype(u);
        const int64_t units = row_bytes / (int64_t)sizeof(U);
        hipLaunchKernelGGL(k_dispatch<U>, dim3(blocks_for(N * units, 256, 16384)), dim3(256), 0, s, static_cast<const char*>(x),
                           units, x_stride, N, top, place, static_cast<char*>(out), out_stride, out_rows);
    };
    if (any % 16 == 0) go(uint4{});
    else if (any % 4 == 0) go(uint32_t{});
    else if (any % 2 == 0) go(uint16_t{});
    else go(uint8_t{});
}

void launch_combine(const void* rows, int type, int64_t H, int64_t stride, int64_t n_rows, const int32_t* place,
                    const float* weights, int64_t N, int top, void* out, int64_t out_stride, hipStream_t s) {
    if (N == 0 || H == 0) return;
    with_type(type, [&](auto t) {
        using T = decltype(t);
        hipLaunchKernelGGL(k_combine<T>, dim3(blocks_for(N * H, 256, 16384)), dim3(256), 0, s, static_cast<const T*>(rows), H,
                           stride, n_rows, place, weights, N, top, static_cast<T*>(out), out_stride);
    });
}

void launch_combine_backward(const void* dout, int64_t dout_stride, const void* rows, int type, int64_t H, int64_t stride,
                             int64_t n_rows, const int32_t* place, const float* weights, int64_t N, int top, void* drows,
                             int64_t drows_stride, float* dweights, hipStream_t s) {
    if (N == 0) return;
    with_type(type, [&](auto t) {
        using T = decltype(t);
        hipLaunchKernelGGL(k_combine_backward<T>, dim3(blocks_for(N * top, 4, 16384)), dim3(256), 0, s,
                           static_cast<const T*>(dout), dout_stride, static_cast<const T*>(rows), H, stride, n_rows, place,
                           weights, N * top, top, static_cast<T*>(drows), drows_stride, dweights);
    });
}

}  // namespace einet_impl

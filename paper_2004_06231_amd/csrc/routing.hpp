// Launchers of the operators around a mixture whose samples are routed to its components (routing.hip, choose.hip), and
// the sizes that their host checks and workspaces go by.
#ifndef EINET_ROUTING_HPP
#define EINET_ROUTING_HPP

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace einet_impl {

enum RowType { ROW_FLOAT32 = 0, ROW_BFLOAT16 = 1, ROW_FLOAT16 = 2 };      // EINET_FLOAT32, ...
inline int row_type_bytes(int t) { return t == ROW_FLOAT32 ? 4 : 2; }

constexpr int ROUTE_MAX_COMPONENTS = 1024, ROUTE_MAX_TOP = 16;

// A launch holds fewer than 2^32 work-items: rows of `items` work-items each, in launches of as many rows as fit.
// f(first row, rows)
template <class F>
void row_batches(int64_t rows, int64_t items, F&& f) {
    const int64_t most = std::max<int64_t>((0xffffffffll - 1023) / items, 1);      // (1023: up to a whole workgroup)
    for (int64_t r = 0; r < rows; r += most) f(r, std::min(rows - r, most));
}
constexpr int64_t ROW_MOST_BYTES = 1ll << 35;                                      // 2^31 units of 16 bytes

// scores: entry (component c, sample n) at c * sc + n * sn
struct Scores {
    const void* p;
    int type;
    int64_t sc, sn;
    const float* coef;        // [M] or nullptr
    int M;
    int64_t N;
};
void launch_route(const Scores& a, int top, bool renormalise, int32_t* ids, float* weights, float* logp, hipStream_t s);
size_t route_backward_workspace(int M, int64_t N);
void launch_route_backward(const Scores& a, int top, bool renormalise, const int32_t* ids, const float* weights,
                           const float* dweights, const float* dlogp, void* dscores, int64_t dsc, int64_t dsn, float* dcoef,
                           void* workspace, hipStream_t s);

size_t sort_workspace(int64_t slots, int M);
void launch_sort(const int32_t* ids, int64_t slots, int M, int32_t* first, int32_t* place, void* workspace, hipStream_t s);

void launch_dispatch(const void* x, int64_t row_bytes, int64_t x_stride, int64_t N, int top, const int32_t* place, void* out,
                     int64_t out_stride, int64_t out_rows, hipStream_t s);
void launch_combine(const void* rows, int type, int64_t H, int64_t stride, int64_t n_rows, const int32_t* place,
                    const float* weights, int64_t N, int top, void* out, int64_t out_stride, hipStream_t s);
void launch_combine_backward(const void* dout, int64_t dout_stride, const void* rows, int type, int64_t H, int64_t stride,
                             int64_t n_rows, const int32_t* place, const float* weights, int64_t N, int top, void* drows,
                             int64_t drows_stride, float* dweights, hipStream_t s);

// a setting of every row (p) or one for all of them (v, where p is nullptr)
template <class X>
struct Setting {
    const X* p;
    X v;
};
struct ChooseArgs {
    const void* logits;
    int type;
    int64_t stride;
    int B, V;
    const float* u;
    Setting<float> temperature, top_p, min_p;
    Setting<int32_t> top_k;
    int32_t* index;
    float* logq;              // or nullptr
    void* workspace;
    float inv_t;              // 1 / T and log2(e) / T where T holds for all rows: filled in by launch_choose
    double log2e_t;
};
size_t choose_workspace(int B, int V);
void launch_choose(const ChooseArgs& a, hipStream_t s);

}  // namespace einet_impl

#endif

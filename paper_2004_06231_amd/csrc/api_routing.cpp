// C ABI of the operators around a mixture whose samples are routed to its components (see include/einet.h): argument
// checks and launches.  No device memory is allocated here.
#include <hip/hip_runtime.h>

#include <string>

#include "../../include/einet.h"
#include "kernels.hpp"
#include "routing.hpp"

using namespace einet_impl;

static_assert(EINET_ROUTE_MAX_COMPONENTS == ROUTE_MAX_COMPONENTS && EINET_ROUTE_MAX_TOP == ROUTE_MAX_TOP, "limits of the header");
static_assert(EINET_FLOAT32 == ROW_FLOAT32 && EINET_BFLOAT16 == ROW_BFLOAT16 && EINET_FLOAT16 == ROW_FLOAT16, "types of the header");

namespace {

int invalid(const char* call, const char* what) { return fail_without_handle(EINET_ERR_INVALID_ARG, std::string(call) + ": " + what); }

int check_hip(const char* call) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail_without_handle(EINET_ERR_HIP, std::string(call) + ": " + hipGetErrorString(e));
    return EINET_OK;
}

bool known_type(int t) { return t == EINET_FLOAT32 || t == EINET_BFLOAT16 || t == EINET_FLOAT16; }
bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
constexpr int64_t MOST_SLOTS = 0x7fffffff;
const char* const MISALIGNED = "a pointer is not aligned to its elements";

const char* route_problem(const void* score, int dtype, int64_t sc, int64_t sn, const float* coef, int M, int64_t n, int top) {
    if (!known_type(dtype)) return "unknown dtype";
    if (M < 1 || M > EINET_ROUTE_MAX_COMPONENTS) return "n_components must be in 1..EINET_ROUTE_MAX_COMPONENTS";
    if (top < 1 || top > EINET_ROUTE_MAX_TOP || top > M) return "top must be in 1..min(n_components, EINET_ROUTE_MAX_TOP)";
    if (n < 0 || n > MOST_SLOTS / top) return "n must be at least 0 and n * top below 2^31";
    if (sc < 0 || sn < 0) return "strides must not be negative";
    if (!score && n > 0) return "score_dev is NULL";
    if (!aligned(score, row_type_bytes(dtype)) || !aligned(coef, 4)) return MISALIGNED;
    return nullptr;
}

// what the calls that carry rows have in common
const char* slots_problem(int64_t n, int top, int64_t n_rows, int64_t width, int64_t element_bytes) {
    if (top < 1) return "top must be at least 1";
    if (n < 0 || n > MOST_SLOTS / top) return "n must be at least 0 and n * top below 2^31";
    if (n_rows < 0) return "the number of sorted rows must not be negative";
    if (width > ROW_MOST_BYTES / element_bytes) return "a row must not have more than 2^35 bytes";
    return nullptr;
}

}  // namespace

extern "C" {

int einet_route(const void* score_dev, int dtype, int64_t component_stride, int64_t sample_stride, const float* log_coef_dev,
                int n_components, int64_t n, int top, int renormalise, int32_t* id_dev, float* weight_dev, float* logp_dev,
                void* stream) {
    const char* const call = "einet_route";
    if (const char* e = route_problem(score_dev, dtype, component_stride, sample_stride, log_coef_dev, n_components, n, top))
        return invalid(call, e);
    if (n == 0) return EINET_OK;
    if (!id_dev || !weight_dev || !logp_dev) return invalid(call, "NULL pointer");
    if (!aligned(id_dev, 4) || !aligned(weight_dev, 4) || !aligned(logp_dev, 4)) return invalid(call, MISALIGNED);
    launch_route(Scores{score_dev, dtype, component_stride, sample_stride, log_coef_dev, n_components, n}, top, renormalise != 0,
                 id_dev, weight_dev, logp_dev, static_cast<hipStream_t>(stream));
    return check_hip(call);
}

int einet_route_workspace(int n_components, int64_t n, size_t* bytes) {
    if (!bytes || n_components < 1 || n_components > EINET_ROUTE_MAX_COMPONENTS || n < 0)
        return invalid("einet_route_workspace", "n_components must be in 1..EINET_ROUTE_MAX_COMPONENTS, n at least 0, bytes not NULL");
    *bytes = route_backward_workspace(n_components, n);
    return EINET_OK;
}

int einet_route_backward(const void* score_dev, int dtype, int64_t component_stride, int64_t sample_stride,
                         const float* log_coef_dev, int n_components, int64_t n, int top, int renormalise, const int32_t* id_dev,
                         const float* weight_dev, const float* dweight_dev, const float* dlogp_dev, void* dscore_dev,
                         int64_t dcomponent_stride, int64_t dsample_stride, float* dlog_coef_dev, void* workspace_dev,
                         size_t workspace_bytes, void* stream) {
    const char* const call = "einet_route_backward";
    if (const char* e = route_problem(score_dev, dtype, component_stride, sample_stride, log_coef_dev, n_components, n, top))
        return invalid(call, e);
    if (dcomponent_stride < 0 || dsample_stride < 0) return invalid(call, "strides must not be negative");
    if (n > 0 && (!dscore_dev || (dweight_dev && (!id_dev || !weight_dev)))) return invalid(call, "NULL pointer");
    if (!aligned(dscore_dev, row_type_bytes(dtype)) || !aligned(id_dev, 4) || !aligned(weight_dev, 4) || !aligned(dweight_dev, 4) ||
        !aligned(dlogp_dev, 4) || !aligned(dlog_coef_dev, 4))
        return invalid(call, MISALIGNED);
    const size_t need = route_backward_workspace(n_components, n);
    if (dlog_coef_dev && need > 0 && (!workspace_dev || !aligned(workspace_dev, 16) || workspace_bytes < need))
        return invalid(call, "dlog_coef_dev needs a workspace of einet_route_workspace bytes, 16-byte aligned");
    launch_route_backward(Scores{score_dev, dtype, component_stride, sample_stride, log_coef_dev, n_components, n}, top,
                          renormalise != 0, id_dev, weight_dev, dweight_dev, dlogp_dev, dscore_dev, dcomponent_stride,
                          dsample_stride, dlog_coef_dev, workspace_dev, static_cast<hipStream_t>(stream));
    return check_hip(call);
}

int einet_sort_workspace(int64_t n_slots, int n_components, size_t* bytes) {
    if (!bytes || n_components < 1 || n_components > EINET_ROUTE_MAX_COMPONENTS || n_slots < 0 || n_slots > MOST_SLOTS)
        return invalid("einet_sort_workspace", "n_components must be in 1..EINET_ROUTE_MAX_COMPONENTS, n_slots in 0..2^31-1, bytes not NULL");
    *bytes = sort_workspace(n_slots, n_components);
    return EINET_OK;
}

int einet_sort(const int32_t* id_dev, int64_t n_slots, int n_components, int32_t* first_dev, int32_t* place_dev,
               void* workspace_dev, size_t workspace_bytes, void* stream) {
    const char* const call = "einet_sort";
    if (n_components < 1 || n_components > EINET_ROUTE_MAX_COMPONENTS)
        return invalid(call, "n_components must be in 1..EINET_ROUTE_MAX_COMPONENTS");
    if (n_slots < 0 || n_slots > MOST_SLOTS) return invalid(call, "n_slots must be in 0..2^31-1");
    if (!first_dev || (n_slots > 0 && (!id_dev || !place_dev))) return invalid(call, "NULL pointer");
    if (!aligned(id_dev, 4) || !aligned(first_dev, 4) || !aligned(place_dev, 4)) return invalid(call, MISALIGNED);
    const size_t need = sort_workspace(n_slots, n_components);
    if (need > 0 && (!workspace_dev || !aligned(workspace_dev, 16) || workspace_bytes < need))
        return invalid(call, "needs a workspace of einet_sort_workspace bytes, 16-byte aligned");
    launch_sort(id_dev, n_slots, n_components, first_dev, place_dev, workspace_dev, static_cast<hipStream_t>(stream));
    return check_hip(call);
}

int einet_dispatch(const void* row_dev, int64_t row_bytes, int64_t row_stride_bytes, int64_t n, int top, const int32_t* place_dev,
                   void* out_dev, int64_t out_stride_bytes, int64_t out_rows, void* stream) {
    const char* const call = "einet_dispatch";
    if (const char* e = slots_problem(n, top, out_rows, row_bytes, 1)) return invalid(call, e);
    if (row_bytes < 0 || row_stride_bytes < 0) return invalid(call, "row_bytes and the strides must not be negative");
    if (out_stride_bytes < row_bytes) return invalid(call, "rows of out_dev would overlap");
    if (n == 0 || row_bytes == 0 || out_rows == 0) return EINET_OK;
    if (!row_dev || !place_dev || !out_dev) return invalid(call, "NULL pointer");
    if (!aligned(place_dev, 4)) return invalid(call, MISALIGNED);
    launch_dispatch(row_dev, row_bytes, row_stride_bytes, n, top, place_dev, out_dev, out_stride_bytes, out_rows,
                    static_cast<hipStream_t>(stream));
    return check_hip(call);
}

int einet_combine(const void* row_dev, int dtype, int64_t width, int64_t row_stride, int64_t n_rows, const int32_t* place_dev,
                  const float* weight_dev, int64_t n, int top, void* out_dev, int64_t out_stride, void* stream) {
    const char* const call = "einet_combine";
    if (!known_type(dtype)) return invalid(call, "unknown dtype");
    if (const char* e = slots_problem(n, top, n_rows, width, row_type_bytes(dtype))) return invalid(call, e);
    if (width < 0 || row_stride < 0) return invalid(call, "width and the strides must not be negative");
    if (out_stride < width) return invalid(call, "rows of out_dev would overlap");
    if (n == 0 || width == 0) return EINET_OK;
    if ((!row_dev && n_rows > 0) || !place_dev || !out_dev) return invalid(call, "NULL pointer");
    const size_t e = row_type_bytes(dtype);
    if (!aligned(row_dev, e) || !aligned(out_dev, e) || !aligned(place_dev, 4) || !aligned(weight_dev, 4))
        return invalid(call, MISALIGNED);
    launch_combine(row_dev, dtype, width, row_stride, n_rows, place_dev, weight_dev, n, top, out_dev, out_stride,
                   static_cast<hipStream_t>(stream));
    return check_hip(call);
}

int einet_combine_backward(const void* dout_dev, int64_t dout_stride, const void* row_dev, int dtype, int64_t width,
                           int64_t row_stride, int64_t n_rows, const int32_t* place_dev, const float* weight_dev, int64_t n, int top,
                           void* drow_dev, int64_t drow_stride, float* dweight_dev, void* stream) {
    const char* const call = "einet_combine_backward";
    if (!known_type(dtype)) return invalid(call, "unknown dtype");
    if (const char* e = slots_problem(n, top, n_rows, width, row_type_bytes(dtype))) return invalid(call, e);
    if (width < 0 || row_stride < 0 || dout_stride < 0) return invalid(call, "width and the strides must not be negative");
    if (drow_stride < width) return invalid(call, "rows of drow_dev would overlap");
    if (n == 0) return EINET_OK;
    if (!place_dev || !weight_dev || !dweight_dev || (width > 0 && !dout_dev) || (width > 0 && n_rows > 0 && (!row_dev || !drow_dev)))
        return invalid(call, "NULL pointer");
    const size_t e = row_type_bytes(dtype);
    if (!aligned(dout_dev, e) || !aligned(row_dev, e) || !aligned(drow_dev, e) || !aligned(place_dev, 4) || !aligned(weight_dev, 4) ||
        !aligned(dweight_dev, 4))
        return invalid(call, MISALIGNED);
    launch_combine_backward(dout_dev, dout_stride, row_dev, dtype, width, row_stride, n_rows, place_dev, weight_dev, n, top, drow_dev,
                            drow_stride, dweight_dev, static_cast<hipStream_t>(stream));
    return check_hip(call);
}

int einet_choose_workspace(int n_rows, int n_entries, size_t* bytes) {
    if (!bytes || n_rows < 0 || n_entries < 1 || n_entries > EINET_CHOOSE_MAX_ENTRIES)
        return invalid("einet_choose_workspace", "n_rows must be at least 0, n_entries in 1..EINET_CHOOSE_MAX_ENTRIES, bytes not NULL");
    *bytes = choose_workspace(n_rows, n_entries);
    return EINET_OK;
}

int einet_choose(const void* logit_dev, int dtype, int64_t row_stride, int n_rows, int n_entries, const float* u_dev,
                 const float* temperature_dev, float temperature, const int32_t* top_k_dev, int top_k, const float* top_p_dev,
                 float top_p, const float* min_p_dev, float min_p, int32_t* index_dev, float* logq_dev, void* workspace_dev,
                 size_t workspace_bytes, void* stream) {
    const char* const call = "einet_choose";
    if (!known_type(dtype)) return invalid(call, "unknown dtype");
    if (n_rows < 0 || n_entries < 1 || n_entries > EINET_CHOOSE_MAX_ENTRIES)
        return invalid(call, "n_rows must be at least 0 and n_entries in 1..EINET_CHOOSE_MAX_ENTRIES");
    if (row_stride < 0) return invalid(call, "row_stride must not be negative");
    if (!temperature_dev && !(temperature >= 0.f)) return invalid(call, "temperature must be at least 0");
    if (!top_k_dev && top_k < 0) return invalid(call, "top_k must be at least 0");
    if (!top_p_dev && !(top_p >= 0.f && top_p <= 1.f)) return invalid(call, "top_p must be in [0, 1]");
    if (!min_p_dev && !(min_p >= 0.f && min_p <= 1.f)) return invalid(call, "min_p must be in [0, 1]");
    if (n_rows == 0) return EINET_OK;
    if (!logit_dev || !u_dev || !index_dev) return invalid(call, "NULL pointer");
    if (!aligned(logit_dev, row_type_bytes(dtype)) || !aligned(u_dev, 4) || !aligned(temperature_dev, 4) || !aligned(top_k_dev, 4) ||
        !aligned(top_p_dev, 4) || !aligned(min_p_dev, 4) || !aligned(index_dev, 4) || !aligned(logq_dev, 4))
        return invalid(call, MISALIGNED);
    const size_t need = choose_workspace(n_rows, n_entries);
    if (need > 0 && (!workspace_dev || !aligned(workspace_dev, 256) || workspace_bytes < need))
        return invalid(call, "needs a workspace of einet_choose_workspace bytes, 256-byte aligned");
    launch_choose(ChooseArgs{logit_dev, dtype, row_stride, n_rows, n_entries, u_dev, {temperature_dev, temperature},
                             {top_p_dev, top_p}, {min_p_dev, min_p}, {top_k_dev, top_k}, index_dev, logq_dev, workspace_dev, 0.f, 0.0},
                  static_cast<hipStream_t>(stream));
    return check_hip(call);
}

}  // extern "C"

// fff_operators.hpp -- parameters and launchers of the operators around the layer, between
// fff_api.cpp and their kernels.  Apart from fff_internal.hpp: the layer's kernels are not built from it.
#pragma once

#include "fff_internal.hpp"

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

namespace fff {

// Dropout's generator (fff_dropout_rng) as the kernels take it.
struct DropRng {
    uint32_t on;             // p > 0
    uint32_t threshold;      // kept where the generator's word is at least this
    float scale;             // 1 / (1 - p)
    uint32_t k0, k1;         // seed
    uint64_t offset;
    const int64_t* offset_dev;  // added to offset when set
};

struct NormParams {
    const void* x;
    const void* residual;    // or null
    const float* gamma;      // or null
    const float* beta;       // or null
    void* y;
    void* s;                 // or null
    float* mean;             // or null
    float* rstd;             // or null
    int64_t n_tokens;
    int32_t hidden;
    int32_t x_bf16, s_bf16, y_bf16;
    float eps;
    DropRng drop;
};
hipError_t run_layer_norm(const NormParams& p, const DeviceInfo& dev, hipStream_t stream);

struct NormBwdParams {
    const void* dy;
    const void* s;
    const float* mean;
    const float* rstd;
    const float* gamma;      // or null
    const void* ds_in;       // or null
    void* ds;                // or null
    void* dx;                // or null
    float* dgamma;           // or null
    float* dbeta;            // or null
    float* part;             // [parts, 2, hidden] partial sums of dgamma and dbeta
    int64_t n_tokens;
    int32_t hidden;
    int32_t x_bf16, s_bf16, y_bf16;
    int32_t accumulate;
    DropRng drop;
};
size_t norm_bwd_workspace_bytes(int64_t n_tokens, int32_t hidden);
hipError_t run_layer_norm_backward(const NormBwdParams& p, const DeviceInfo& dev, hipStream_t stream);

struct DropoutParams {
    const void* x;
    const void* residual;    // or null
    void* y;
    int64_t n_tokens;
    int32_t hidden;
    int32_t x_bf16, r_bf16, y_bf16;
    DropRng drop;
};
hipError_t run_dropout(const DropoutParams& p, const DeviceInfo& dev, hipStream_t stream);

struct GroupParams {
    const int32_t* ids;
    int32_t* order;
    int32_t* offsets;
    int32_t* bad;            // or null
    int64_t n_entries;
    int32_t n_ids, n_trees, first;
    int32_t n_groups;        // n_ids * n_trees
    void* workspace;
};
constexpr int32_t MAX_GROUPS = 32768;
size_t group_workspace_bytes(int64_t n_entries, int32_t n_groups);
hipError_t run_group_rows(const GroupParams& p, hipStream_t stream);

// Rows of the grouped products: entry i of group g (offsets[g] <= i < offsets[g + 1]).
struct GroupedParams {
    const void* x;           // [x_rows, k]
    const void* w;           // [n_groups, n, k] or (w_transposed) [n_groups, k, n]
    const int32_t* offsets;
    const int32_t* x_index;  // or null
    const int32_t* y_index;  // or null
    void* y;                 // [y_rows, n]
    void* z_out;             // or null
    const void* z_in;        // or null
    int64_t n_entries, x_rows, y_rows;
    int32_t n_groups, k, n, x_div;
    int32_t w_transposed;
    int32_t bf16;            // x and w
    int32_t y_bf16, z_bf16;
    int32_t act;
};
// *status: ST_OK, or FFF_ERR_UNSUPPORTED's value when the grid would be too large (nothing enqueued).
// With buf nothing is enqueued: the kernel and its launch are named there (describe).
hipError_t run_grouped_matmul(const GroupedParams& p, const DeviceInfo& dev, hipStream_t stream, int* status,
                              char* buf = nullptr, size_t len = 0);

struct GroupedGradParams {
    const void* dy;          // [dy_rows, n]
    const void* x;           // [x_rows, k]
    const int32_t* offsets;
    const int32_t* dy_index; // or null
    const int32_t* x_index;  // or null
    float* dw;               // [n_groups, n, k]
    int64_t n_entries, dy_rows, x_rows;
    int32_t n_groups, k, n, x_div;
    int32_t bf16;
    int32_t accumulate;
    float* part;             // partial sums, or null
};
size_t grouped_grad_workspace_bytes(int64_t n_entries, int32_t n_groups, int32_t k, int32_t n);
hipError_t run_grouped_weight_grad(const GroupedGradParams& p, hipStream_t stream, int* status, char* buf = nullptr,
                                   size_t len = 0);

// ---- a routed expert block --------------------------------------------------

enum { SCORE_SOFTMAX = 0, SCORE_SIGMOID = 1 };
enum { GROUP_MAX = 0, GROUP_TOP2 = 1 };
constexpr int32_t MAX_TOP_K = 64, MAX_ROUTE_GROUPS = 1024;

struct RouteParams {
    const void* logits;
    const float* bias;       // or null
    int32_t* ids;
    float* weights;
    int64_t n_tokens;
    int32_t n_experts, top_k, n_groups, top_groups;
    int32_t group_size;      // n_experts / n_groups
    int32_t bf16;
    int32_t score, group_score, renormalise;
    float scale;
};
hipError_t run_route(const RouteParams& p, const DeviceInfo& dev, hipStream_t stream);

struct RouteBwdParams {
    const float* dweights;
    const void* logits;
    const int32_t* ids;
    void* dlogits;
    int64_t n_tokens;
    int32_t n_experts, top_k;
    int32_t bf16, d_bf16;
    int32_t score, renormalise;
    float scale;
};
hipError_t run_route_backward(const RouteBwdParams& p, const DeviceInfo& dev, hipStream_t stream);

struct CombineParams {
    const void* rows;
    const float* weights;    // or null
    const int32_t* ids;      // or null
    const void* residual;    // or null
    void* y;
    int64_t n_tokens;
    int32_t hidden, top_k;
    int32_t rows_bf16, y_bf16;
};
hipError_t run_combine(const CombineParams& p, const DeviceInfo& dev, hipStream_t stream);

struct CombineBwdParams {
    const void* dy;
    const void* rows;        // or null
    const float* weights;    // or null
    const int32_t* ids;      // or null
    void* drows;             // or null
    float* dweights;         // or null
    int64_t n_tokens;
    int32_t hidden, top_k;
    int32_t y_bf16, rows_bf16, drows_bf16;
};
hipError_t run_combine_backward(const CombineBwdParams& p, const DeviceInfo& dev, hipStream_t stream);

struct RmsParams {
    const void* x;
    const void* residual;    // or null
    const float* gamma;      // or null
    void* y;                 // or null
    void* s;                 // or null
    float* rstd;             // or null
    uint8_t* q;              // or null
    uint8_t* q_scale;
    int64_t n_tokens;
    int32_t hidden;
    int32_t x_bf16, s_bf16, y_bf16;
    float eps;
};
hipError_t run_rms_norm(const RmsParams& p, const DeviceInfo& dev, hipStream_t stream);

struct RmsBwdParams {
    const void* dy;
    const void* s;
    const float* rstd;
    const float* gamma;      // or null
    const void* ds_in;       // or null
    void* ds;                // or null
    void* dx;                // or null
    float* dgamma;           // or null
    float* part;             // [parts, hidden] partial sums of dgamma
    int64_t n_tokens;
    int32_t hidden;
    int32_t x_bf16, s_bf16, y_bf16;
    int32_t accumulate;
};
size_t rms_bwd_workspace_bytes(int64_t n_tokens, int32_t hidden);
hipError_t run_rms_norm_backward(const RmsBwdParams& p, const DeviceInfo& dev, hipStream_t stream);

struct PackParams {
    const void* x;
    uint8_t* q;
    uint8_t* q_scale;
    int64_t n_rows;
    int32_t hidden;
    int32_t x_bf16;
};
hipError_t run_pack_rows(const PackParams& p, const DeviceInfo& dev, hipStream_t stream);

struct UnpackParams {
    const uint8_t* q;
    const uint8_t* q_scale;
    const void* dy;          // with dx
    void* y;                 // or null
    void* dx;                // or null
    int64_t n_rows;
    int32_t hidden;
    int32_t dy_bf16, y_bf16, dx_bf16;
    int32_t act;
};
hipError_t run_unpack_rows(const UnpackParams& p, const DeviceInfo& dev, hipStream_t stream);

}  // namespace fff

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

}  // namespace fff

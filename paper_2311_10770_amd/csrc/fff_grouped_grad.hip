// fff_grouped_grad.hip -- weight gradients of the grouped products
// (fff_grouped_weight_grad): dW_g = sum over group g's entries of dy_i^T x_i.
#include "fff_grouped.hpp"

namespace fff {

namespace {

enum { ST_OK_ = 0, ST_UNSUPPORTED_ = -2 };

// Any sizes and types: a workgroup per 64 x 64 tile of one group's dW, its entries sixteen at a time.
__global__ __launch_bounds__(256) void grouped_grad_any_kernel(GroupedGradParams p) {
    __shared__ float sa[16][65], sb[16][65];
    const int tn = (p.n + 63) / 64, tk = (p.k + 63) / 64;
    const int64_t b = blockIdx.x;
    const int g = int(b / (int64_t(tn) * tk)), rest = int(b % (int64_t(tn) * tk));
    const int n0 = rest / tk * 64, k0 = rest % tk * 64, tid = threadIdx.x;
    int64_t lo = 0, hi = 0;
    if (p.n_entries > 0) group_range(p.offsets, p.n_entries, g, &lo, &hi);
    float acc[4][4] = {};
    const int tm = tid / 16, tc = tid % 16;
    for (int64_t e0 = lo; e0 < hi; e0 += 16) {
        for (int v = tid; v < 1024; v += 256) {
            const int c = v % 64, r = v / 64;
            const int64_t i = e0 + r;
            const int64_t d = i < hi ? entry_row(p.dy_index, 1, p.dy_rows, i) : -1;
            const int64_t s = i < hi ? entry_row(p.x_index, p.x_div, p.x_rows, i) : -1;
            sa[r][c] = d >= 0 && n0 + c < p.n ? load_elem(p.dy, p.bf16, d * p.n + n0 + c) : 0.0f;
            sb[r][c] = s >= 0 && k0 + c < p.k ? load_elem(p.x, p.bf16, s * p.k + k0 + c) : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < 16; ++r)
#pragma unroll
            for (int a = 0; a < 4; ++a)
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    acc[a][c] = __builtin_fmaf(sa[r][tm * 4 + a], sb[r][tc * 4 + c], acc[a][c]);
        __syncthreads();
    }
    if (hi == lo && p.accumulate) return;
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int n = n0 + tm * 4 + a, k = k0 + tc * 4 + c;
            if (n >= p.n || k >= p.k) continue;
            float* d = p.dw + (int64_t(g) * p.n + n) * p.k + k;
            *d = p.accumulate ? *d + acc[a][c] : acc[a][c];
        }
}

}  // namespace

size_t grouped_grad_workspace_bytes(int64_t, int32_t, int32_t, int32_t) { return 0; }

hipError_t run_grouped_weight_grad(const GroupedGradParams& p, const DeviceInfo&, hipStream_t stream, int* status) {
    const int64_t grid = int64_t(p.n_groups) * ((int64_t(p.n) + 63) / 64) * ((int64_t(p.k) + 63) / 64);
    *status = grid > INT32_MAX ? ST_UNSUPPORTED_ : ST_OK_;
    if (*status != ST_OK_) return hipSuccess;
    hipLaunchKernelGGL(grouped_grad_any_kernel, dim3(unsigned(grid)), dim3(256), 0, stream, p);
    return hipGetLastError();
}

}  // namespace fff

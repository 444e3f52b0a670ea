// fff_grouped.hip -- matrix products grouped by expert with ragged sizes
// (fff_grouped_matmul) and their weight gradients (fff_grouped_weight_grad).
//
// Only the device knows how many entries a group has, so a launch covers the
// most row tiles there can be and every workgroup finds its tile from the
// offsets (find_tile).
#include "fff_device.hpp"
#include "fff_internal.hpp"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

namespace fff {

namespace {

enum { ST_OK_ = 0, ST_UNSUPPORTED_ = -2 };

__device__ __forceinline__ float load_elem(const void* p, bool bf, int64_t i) {
    return bf ? bf16_to_f32(static_cast<const uint16_t*>(p)[i]) : static_cast<const float*>(p)[i];
}
__device__ __forceinline__ void store_elem(void* p, bool bf, int64_t i, float v) {
    if (bf) static_cast<uint16_t*>(p)[i] = f32_to_bf16(v);
    else static_cast<float*>(p)[i] = v;
}

// Entries [lo, hi) of group g: within [0, n_entries], empty where the offsets fall.
__device__ __forceinline__ void group_range(const int32_t* offsets, int64_t n_entries, int g, int64_t* lo, int64_t* hi) {
    const int64_t a = offsets[g], b = offsets[g + 1];
    *lo = a < 0 ? 0 : a > n_entries ? n_entries : a;
    *hi = b < *lo ? *lo : b > n_entries ? n_entries : b;
}

struct Tile {
    int g;           // group, or -1: no tile of this number
    int64_t m0, m1;  // its entries
};

// Row tile number t over all groups (tiles of bm entries, groups in order, each group's last tile
// partly filled): every thread sums the tiles of a few consecutive groups, the workgroup scans the
// sums, and the thread whose groups hold tile t finds it.
template <int THREADS>
__device__ __forceinline__ Tile find_tile(const int32_t* offsets, int n_groups, int64_t n_entries, int bm, int64_t t) {
    __shared__ int64_t wave_sum[THREADS / 64];
    __shared__ Tile found;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int per = (n_groups + THREADS - 1) / THREADS;
    const int g0 = std::min(n_groups, tid * per), g1 = std::min(n_groups, g0 + per);
    int64_t mine = 0, lo, hi;
    for (int g = g0; g < g1; ++g) {
        group_range(offsets, n_entries, g, &lo, &hi);
        mine += (hi - lo + bm - 1) / bm;
    }
    int64_t run = mine;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int64_t v = __shfl_up(run, d);
        if (lane >= d) run += v;
    }
    if (lane == 63) wave_sum[wave] = run;
    if (tid == 0) found.g = -1;
    __syncthreads();
    for (int w = 0; w < wave; ++w) run += wave_sum[w];
    int64_t at = run - mine;
    if (at <= t && t < run) {
        for (int g = g0; g < g1; ++g) {
            group_range(offsets, n_entries, g, &lo, &hi);
            const int64_t tiles = (hi - lo + bm - 1) / bm;
            if (t < at + tiles) {
                found.g = g;
                found.m0 = lo + (t - at) * bm;
                found.m1 = hi;
                break;
            }
            at += tiles;
        }
    }
    __syncthreads();
    return found;
}

// Most row tiles of bm entries that n_entries in n_groups groups can make.
int64_t most_tiles(int64_t n_entries, int32_t n_groups, int bm) {
    return n_entries / bm + std::min<int64_t>(n_groups, n_entries);
}

// Row of x that entry i reads, or -1 where there is none.
__device__ __forceinline__ int64_t source_row(const int32_t* index, int x_div, int64_t rows, int64_t i) {
    const int64_t v = index ? index[i] : i;
    if (v < 0) return -1;
    const int64_t r = x_div == 1 ? v : v / x_div;
    return r < rows ? r : -1;
}

// z of entry i, column n: the epilogue and the store.
__device__ __forceinline__ void grouped_store(const GroupedParams& p, int64_t i, int64_t dst, int n, float z) {
    if (p.z_in) z *= activation_grad(load_elem(p.z_in, p.z_bf16, i * p.n + n), p.act);
    else {
        if (p.z_out) store_elem(p.z_out, p.z_bf16, i * p.n + n, z);
        z = activation(z, p.act);
    }
    if (dst >= 0) store_elem(p.y, p.y_bf16, dst * p.n + n, z);
}

// Any sizes and types: 64 x 64 tiles, fp32 FMAs on tiles widened into LDS.
__global__ __launch_bounds__(256) void grouped_any_kernel(GroupedParams p) {
    __shared__ float sa[16][65], sb[16][65];
    const int tn = (p.n + 63) / 64;
    const Tile t = find_tile<256>(p.offsets, p.n_groups, p.n_entries, 64, blockIdx.x / tn);
    if (t.g < 0) return;
    const int n0 = int(blockIdx.x % tn) * 64, tid = threadIdx.x;
    const int64_t wg = int64_t(t.g) * p.n * p.k;
    float acc[4][4] = {};
    const int tm = tid / 16, tc = tid % 16;
    for (int k0 = 0; k0 < p.k; k0 += 16) {
        for (int v = tid; v < 1024; v += 256) {
            const int kk = v % 16, r = v / 16;
            const int64_t i = t.m0 + r;
            const int64_t src = i < t.m1 ? source_row(p.x_index, p.x_div, p.x_rows, i) : -1;
            sa[kk][r] = src >= 0 && k0 + kk < p.k ? load_elem(p.x, p.bf16, src * p.k + k0 + kk) : 0.0f;
        }
        for (int v = tid; v < 1024; v += 256) {
            const int kk = p.w_transposed ? v / 64 : v % 16, c = p.w_transposed ? v % 64 : v / 16;
            const int64_t n = n0 + c, k = k0 + kk;
            sb[kk][c] = n < p.n && k < p.k
                            ? load_elem(p.w, p.bf16, wg + (p.w_transposed ? k * p.n + n : n * p.k + k)) : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int kk = 0; kk < 16; ++kk)
#pragma unroll
            for (int a = 0; a < 4; ++a)
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    acc[a][b] = __builtin_fmaf(sa[kk][tm * 4 + a], sb[kk][tc * 4 + b], acc[a][b]);
        __syncthreads();
    }
#pragma unroll
    for (int a = 0; a < 4; ++a) {
        const int64_t i = t.m0 + tm * 4 + a;
        if (i >= t.m1) continue;
        const int64_t dst = source_row(p.y_index, 1, p.y_rows, i);
#pragma unroll
        for (int b = 0; b < 4; ++b)
            if (n0 + tc * 4 + b < p.n) grouped_store(p, i, dst, n0 + tc * 4 + b, acc[a][b]);
    }
}

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
            const int64_t d = i < hi ? source_row(p.dy_index, 1, p.dy_rows, i) : -1;
            const int64_t s = i < hi ? source_row(p.x_index, p.x_div, p.x_rows, i) : -1;
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

hipError_t run_grouped_matmul(const GroupedParams& p, const DeviceInfo&, hipStream_t stream, int* status) {
    const int64_t grid = most_tiles(p.n_entries, p.n_groups, 64) * ((int64_t(p.n) + 63) / 64);
    *status = grid > INT32_MAX ? ST_UNSUPPORTED_ : ST_OK_;
    if (*status != ST_OK_) return hipSuccess;
    hipLaunchKernelGGL(grouped_any_kernel, dim3(unsigned(grid)), dim3(256), 0, stream, p);
    return hipGetLastError();
}

size_t grouped_grad_workspace_bytes(int64_t, int32_t, int32_t, int32_t) { return 0; }

hipError_t run_grouped_weight_grad(const GroupedGradParams& p, const DeviceInfo&, hipStream_t stream, int* status) {
    const int64_t grid = int64_t(p.n_groups) * ((int64_t(p.n) + 63) / 64) * ((int64_t(p.k) + 63) / 64);
    *status = grid > INT32_MAX ? ST_UNSUPPORTED_ : ST_OK_;
    if (*status != ST_OK_) return hipSuccess;
    hipLaunchKernelGGL(grouped_grad_any_kernel, dim3(unsigned(grid)), dim3(256), 0, stream, p);
    return hipGetLastError();
}

}  // namespace fff

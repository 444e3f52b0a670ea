// fff_norm.hip -- LayerNorm with its residual, dropout and gradients, and
// dropout alone (fff_layer_norm, fff_layer_norm_backward, fff_dropout).
//
//   s = residual + drop(x);  y = (s - mean) rstd gamma + beta
//   ds = rstd (g - mean(g) - xh mean(g xh)) + ds_in,  xh = (s - mean) rstd,
//   g = dy gamma;  dx = drop(ds);  dgamma = sum dy xh;  dbeta = sum dy
//
// All of it is bound by the bytes of the rows.  Statistics, sums and gradients
// are held in fp32; the variance is taken of the centred values (a sum of
// squares less the squared mean would cancel for rows with a large mean).
#include "fff_device.hpp"
#include "fff_internal.hpp"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

namespace fff {

namespace {

// The generator's words of columns 4 blk .. 4 blk + 3 of a row: Philox4x32-10 from its paper
// (Salmon, Moraes, Dror and Shaw, 2011): ten rounds of two 32 x 32 -> 64 bit products.
__device__ __forceinline__ uint4 philox(uint32_t blk, uint32_t row, uint64_t offset, uint32_t k0, uint32_t k1) {
    uint32_t c0 = blk, c1 = row, c2 = uint32_t(offset), c3 = uint32_t(offset >> 32);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const uint64_t p0 = uint64_t(c0) * 0xD2511F53u, p1 = uint64_t(c2) * 0xCD9E8D57u;
        c0 = uint32_t(p1 >> 32) ^ c1 ^ k0;
        c1 = uint32_t(p1);
        c2 = uint32_t(p0 >> 32) ^ c3 ^ k1;
        c3 = uint32_t(p0);
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
}

__device__ __forceinline__ uint64_t rng_offset(const DropRng& d) {
    return d.offset + (d.offset_dev ? uint64_t(*d.offset_dev) : 0);
}

// Dropout of the four values of a generator block; a dropped value is 0 whatever it was.
__device__ __forceinline__ void drop4(float* f, const DropRng& d, uint64_t offset, uint32_t blk, uint32_t row) {
    const uint4 r = philox(blk, row, offset, d.k0, d.k1);
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = word(r, j) >= d.threshold ? f[j] * d.scale : 0.0f;
}

__device__ __forceinline__ float load_elem(const void* p, bool bf, int64_t i) {
    return bf ? bf16_to_f32(static_cast<const uint16_t*>(p)[i]) : static_cast<const float*>(p)[i];
}
__device__ __forceinline__ void store_elem(void* p, bool bf, int64_t i, float v) {
    if (bf) static_cast<uint16_t*>(p)[i] = f32_to_bf16(v);
    else static_cast<float*>(p)[i] = v;
}

// Sum over the workgroup of 256; every thread gets the same bits.
__device__ __forceinline__ float block_sum(float v, float* red) {
    v = group_sum<64>(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

// Rows of any length: a workgroup per row, the row read again in every pass.
__global__ __launch_bounds__(256) void norm_any_kernel(NormParams p) {
    __shared__ float red[4];
    const uint64_t off = p.drop.on ? rng_offset(p.drop) : 0;
    const int H = p.hidden, blocks = (H + 3) / 4;
    for (int64_t row = blockIdx.x; row < p.n_tokens; row += gridDim.x) {
        const int64_t r0 = row * H;
        auto sum4 = [&](int b, float* f) {
#pragma unroll
            for (int j = 0; j < 4; ++j) f[j] = 4 * b + j < H ? load_elem(p.x, p.x_bf16, r0 + 4 * b + j) : 0.0f;
            if (p.drop.on) drop4(f, p.drop, off, uint32_t(b), uint32_t(row));
            if (p.residual) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (4 * b + j < H) f[j] += load_elem(p.residual, p.s_bf16, r0 + 4 * b + j);
            }
        };
        float f[4], acc = 0.0f;
        for (int b = threadIdx.x; b < blocks; b += 256) {
            sum4(b, f);
            acc += (f[0] + f[1]) + (f[2] + f[3]);
        }
        const float mean = block_sum(acc, red) / float(H);
        acc = 0.0f;
        for (int b = threadIdx.x; b < blocks; b += 256) {
            sum4(b, f);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (4 * b + j < H) acc = __builtin_fmaf(f[j] - mean, f[j] - mean, acc);
        }
        const float rstd = 1.0f / sqrtf(block_sum(acc, red) / float(H) + p.eps);
        for (int b = threadIdx.x; b < blocks; b += 256) {
            sum4(b, f);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int c = 4 * b + j;
                if (c >= H) continue;
                if (p.s) store_elem(p.s, p.s_bf16, r0 + c, f[j]);
                const float g = p.gamma ? p.gamma[c] : 1.0f, h = p.beta ? p.beta[c] : 0.0f;
                store_elem(p.y, p.y_bf16, r0 + c, __builtin_fmaf((f[j] - mean) * rstd, g, h));
            }
        }
        if (threadIdx.x == 0) {
            if (p.mean) p.mean[row] = mean;
            if (p.rstd) p.rstd[row] = rstd;
        }
    }
}

// ds and dx of rows of any length: a workgroup per row.
__global__ __launch_bounds__(256) void norm_bwd_any_kernel(NormBwdParams p) {
    __shared__ float red[4];
    const uint64_t off = p.drop.on ? rng_offset(p.drop) : 0;
    const int H = p.hidden, blocks = (H + 3) / 4;
    for (int64_t row = blockIdx.x; row < p.n_tokens; row += gridDim.x) {
        const int64_t r0 = row * H;
        const float mean = p.mean[row], rstd = p.rstd[row];
        auto gh = [&](int c, float* g, float* xh) {
            *xh = (load_elem(p.s, p.s_bf16, r0 + c) - mean) * rstd;
            *g = load_elem(p.dy, p.y_bf16, r0 + c) * (p.gamma ? p.gamma[c] : 1.0f);
        };
        float a = 0.0f, b = 0.0f, g, xh;
        for (int c = threadIdx.x; c < H; c += 256) {
            gh(c, &g, &xh);
            a += g;
            b = __builtin_fmaf(g, xh, b);
        }
        const float c1 = block_sum(a, red) / float(H), c2 = block_sum(b, red) / float(H);
        for (int blk = threadIdx.x; blk < blocks; blk += 256) {
            float f[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int c = 4 * blk + j;
                f[j] = 0.0f;
                if (c >= H) continue;
                gh(c, &g, &xh);
                f[j] = rstd * (g - c1 - xh * c2);
                if (p.ds_in) f[j] += load_elem(p.ds_in, p.s_bf16, r0 + c);
                if (p.ds) store_elem(p.ds, p.s_bf16, r0 + c, f[j]);
            }
            if (!p.dx) continue;
            if (p.drop.on) drop4(f, p.drop, off, uint32_t(blk), uint32_t(row));
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (4 * blk + j < H) store_elem(p.dx, p.x_bf16, r0 + 4 * blk + j, f[j]);
        }
    }
}

// Partial sums of dgamma and dbeta: thread = column, workgroup = 256 columns of one piece of rows.
__global__ __launch_bounds__(256) void norm_bwd_cols_kernel(NormBwdParams p, int parts, int64_t rows_per) {
    const int64_t c = int64_t(blockIdx.x) * 256 + threadIdx.x;
    const int H = p.hidden;
    if (c >= H) return;
    for (int q = blockIdx.y; q < parts; q += gridDim.y) {
        const int64_t r1 = std::min<int64_t>(p.n_tokens, (q + 1) * rows_per);
        float dg = 0.0f, db = 0.0f;
        for (int64_t r = q * rows_per; r < r1; ++r) {
            const float d = load_elem(p.dy, p.y_bf16, r * H + c);
            db += d;
            dg = __builtin_fmaf(d, (load_elem(p.s, p.s_bf16, r * H + c) - p.mean[r]) * p.rstd[r], dg);
        }
        p.part[(int64_t(q) * 2) * H + c] = dg;
        p.part[(int64_t(q) * 2 + 1) * H + c] = db;
    }
}

// dgamma and dbeta: the partial sums in order of the pieces.
__global__ __launch_bounds__(256) void norm_bwd_sum_kernel(NormBwdParams p, int parts) {
    const int64_t c = int64_t(blockIdx.x) * 256 + threadIdx.x;
    const int H = p.hidden;
    if (c >= H) return;
    float dg = 0.0f, db = 0.0f;
    for (int q = 0; q < parts; ++q) {
        dg += p.part[(int64_t(q) * 2) * H + c];
        db += p.part[(int64_t(q) * 2 + 1) * H + c];
    }
    if (p.dgamma) p.dgamma[c] = p.accumulate ? p.dgamma[c] + dg : dg;
    if (p.dbeta) p.dbeta[c] = p.accumulate ? p.dbeta[c] + db : db;
}

// Pieces of rows whose dgamma and dbeta are summed apart.
int norm_parts(int64_t n_tokens) { return int(std::min<int64_t>(512, (n_tokens + 7) / 8)); }

// A thread per generator block of four columns.
__global__ __launch_bounds__(256) void dropout_any_kernel(DropoutParams p) {
    const uint64_t off = p.drop.on ? rng_offset(p.drop) : 0;
    const int64_t H = p.hidden, blocks = (H + 3) / 4, all = p.n_tokens * blocks;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < all; i += int64_t(gridDim.x) * 256) {
        const int64_t row = i / blocks, b = i - row * blocks, e = row * H + 4 * b;
        float f[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] = 4 * b + j < H ? load_elem(p.x, p.x_bf16, e + j) : 0.0f;
        if (p.drop.on) drop4(f, p.drop, off, uint32_t(b), uint32_t(row));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (4 * b + j >= H) continue;
            if (p.residual) f[j] += load_elem(p.residual, p.r_bf16, e + j);
            store_elem(p.y, p.y_bf16, e + j, f[j]);
        }
    }
}

}  // namespace

hipError_t run_layer_norm(const NormParams& p, const DeviceInfo& dev, hipStream_t stream) {
    const unsigned grid = unsigned(std::min<int64_t>(p.n_tokens, 8 * std::max(dev.cu_count, 1)));
    hipLaunchKernelGGL(norm_any_kernel, dim3(grid), dim3(256), 0, stream, p);
    return hipGetLastError();
}

size_t norm_bwd_workspace_bytes(int64_t n_tokens, int32_t hidden) {
    return size_t(norm_parts(n_tokens)) * 2 * size_t(hidden) * sizeof(float);
}

hipError_t run_layer_norm_backward(const NormBwdParams& p, const DeviceInfo& dev, hipStream_t stream) {
    const unsigned cols = unsigned((p.hidden + 255) / 256);
    if ((p.ds || p.dx) && p.n_tokens > 0) {
        const unsigned grid = unsigned(std::min<int64_t>(p.n_tokens, 8 * std::max(dev.cu_count, 1)));
        hipLaunchKernelGGL(norm_bwd_any_kernel, dim3(grid), dim3(256), 0, stream, p);
    }
    if (p.dgamma || p.dbeta) {
        const int parts = norm_parts(p.n_tokens);
        if (parts > 0)
            hipLaunchKernelGGL(norm_bwd_cols_kernel, dim3(cols, unsigned(parts)), dim3(256), 0, stream, p, parts,
                               (p.n_tokens + parts - 1) / parts);
        hipLaunchKernelGGL(norm_bwd_sum_kernel, dim3(cols), dim3(256), 0, stream, p, parts);
    }
    return hipGetLastError();
}

hipError_t run_dropout(const DropoutParams& p, const DeviceInfo& dev, hipStream_t stream) {
    const int64_t blocks = p.n_tokens * ((int64_t(p.hidden) + 3) / 4);
    const unsigned grid = unsigned(std::min<int64_t>((blocks + 255) / 256, 16 * std::max(dev.cu_count, 1)));
    hipLaunchKernelGGL(dropout_any_kernel, dim3(grid), dim3(256), 0, stream, p);
    return hipGetLastError();
}

}  // namespace fff

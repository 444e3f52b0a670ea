// fff_pack.hip -- rows kept in 8 bits for the backward pass (fff_pack_rows), and what
// the backward pass takes from them (fff_unpack_rows): act(z) and dy act'(z).
//
// Bound by the rows' bytes; the format is fff_pack.hpp's.  Four lanes hold the 32 columns of a
// block, eight each, so a block's largest value is two DPP steps away.
#include "fff_activations.hpp"
#include "fff_device.hpp"
#include "fff_operators.hpp"
#include "fff_pack.hpp"
#include "fff_rows.hpp"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

namespace fff {

namespace {

typedef uint32_t u32x2_a1 __attribute__((ext_vector_type(2), aligned(1)));

// Place of unit i: eight columns; a row is `upr` units long, four a block.
struct Unit {
    int64_t row;
    int col;
};
__device__ __forceinline__ Unit unit_of(int64_t i, int upr) {
    const int64_t row = i / upr;
    return {row, int(i - row * upr) * 8};
}

__global__ __launch_bounds__(256) void pack_kernel(PackParams p, int upr, int64_t all) {
    const int H = p.hidden, blocks = upr / 4;
    const int64_t total = p.n_rows * H;
    // whole waves take part, so that a block's four lanes do
    for (int64_t i0 = int64_t(blockIdx.x) * 256; i0 < all; i0 += int64_t(gridDim.x) * 256) {
        const int64_t i = i0 + threadIdx.x;
        const Unit at = unit_of(std::min<int64_t>(i, all - 1), upr);
        const int left = i < all ? H - at.col : 0;
        float f[8];
        uint32_t most = 0;
        if (left > 0) unpack8(f, load8(p.x, p.x_bf16, at.row * H + at.col, total), p.x_bf16);
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            if (c >= left) f[c] = 0.0f;
            most = max(most, finite_bits(f[c]));
        }
        const uint32_t code = scale_code(max_quad(most));
        const float inverse = scale_inverse(code);
#pragma unroll
        for (int c = 0; c < 8; ++c) f[c] = scaled(f[c], code, inverse);
        if (left <= 0) continue;
        uint8_t* q = p.q + at.row * H + at.col;
        const uint32_t lo = pack_e4m3(f[0], f[1], f[2], f[3]), hi = pack_e4m3(f[4], f[5], f[6], f[7]);
        if (left >= 8) {
            *reinterpret_cast<u32x2_a1*>(q) = u32x2_a1{lo, hi};
        } else {
            for (int c = 0; c < left; ++c) q[c] = uint8_t((c < 4 ? lo : hi) >> (c % 4 * 8));
        }
        if (at.col % PACK_BLOCK == 0) p.q_scale[at.row * blocks + at.col / PACK_BLOCK] = uint8_t(code);
    }
}

template <int ACT>
__global__ __launch_bounds__(256) void unpack_kernel(UnpackParams p, int upr, int64_t all) {
    const int H = p.hidden, blocks = upr / 4;
    const int64_t total = p.n_rows * H;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < all; i += int64_t(gridDim.x) * 256) {
        const Unit at = unit_of(i, upr);
        const int left = H - at.col;
        if (left <= 0) continue;
        const int64_t e = at.row * H + at.col;
        uint32_t w[2] = {0, 0};
        if (e + 8 <= total) {
            const u32x2_a1 v = *reinterpret_cast<const u32x2_a1*>(p.q + e);
            w[0] = v.x;
            w[1] = v.y;
        } else {
            for (int c = 0; c < 8 && e + c < total; ++c) w[c / 4] |= uint32_t(p.q[e + c]) << (c % 4 * 8);
        }
        const float scale = scale_value(p.q_scale[at.row * blocks + at.col / PACK_BLOCK]);
        float z[8], f[8];
        unpack_e4m3(z, w[0]);
        unpack_e4m3(z + 4, w[1]);
#pragma unroll
        for (int c = 0; c < 8; ++c) z[c] *= scale;
        if (p.dx) {
            unpack8(f, load8(p.dy, p.dy_bf16, e, total), p.dy_bf16);
#pragma unroll
            for (int c = 0; c < 8; ++c) f[c] *= act_slope<ACT, true>(z[c]);
            store8(p.dx, p.dx_bf16, e, left, f);
        }
        if (p.y) {
#pragma unroll
            for (int c = 0; c < 8; ++c) f[c] = act_value<ACT, true>(z[c]);
            store8(p.y, p.y_bf16, e, left, f);
        }
    }
}

int units_of(int32_t hidden) { return int(pack_blocks(hidden)) * 4; }

}  // namespace

hipError_t run_pack_rows(const PackParams& p, const DeviceInfo& dev, hipStream_t stream) {
    const int upr = units_of(p.hidden);
    const int64_t all = p.n_rows * upr;
    const unsigned grid = unsigned(std::min<int64_t>((all + 255) / 256, 64 * std::max(dev.cu_count, 1)));
    hipLaunchKernelGGL(pack_kernel, dim3(grid), dim3(256), 0, stream, p, upr, all);
    return hipGetLastError();
}

hipError_t run_unpack_rows(const UnpackParams& p, const DeviceInfo& dev, hipStream_t stream) {
    const int upr = units_of(p.hidden);
    const int64_t all = p.n_rows * upr;
    const unsigned grid = unsigned(std::min<int64_t>((all + 255) / 256, 64 * std::max(dev.cu_count, 1)));
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, stream, p, upr, all); };
    if (p.act == ACT_GELU_ERF) launch(unpack_kernel<ACT_GELU_ERF>);
    else if (p.act == ACT_GELU_TANH) launch(unpack_kernel<ACT_GELU_TANH>);
    else launch(unpack_kernel<ACT_IDENTITY>);
    return hipGetLastError();
}

}  // namespace fff

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
#include <type_traits>

namespace fff {

namespace {

typedef uint32_t u32x2_a1 __attribute__((ext_vector_type(2), aligned(1)));

// Where a thread's units of eight columns lie: a workgroup takes U x 256 that follow each other, a thread those 256
// apart, four a block.  FLAT: rows are whole blocks, so places need no division.  Units behind the last one, and those
// behind a row's end, have none of their columns (left <= 0).
template <bool FLAT, int U>
struct Units {
    int64_t e[U], scale[U];
    int left[U];
    __device__ __forceinline__ Units(int64_t i0, int64_t all, int hidden, int upr) {
        if constexpr (FLAT) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t i = i0 + u * 256 + threadIdx.x;
                left[u] = i < all ? 8 : 0;
                e[u] = i < all ? i * 8 : 0;
                scale[u] = i / 4;
            }
        } else {
            const int64_t row0 = i0 / upr;
            const uint32_t rest = uint32_t(i0 - row0 * upr);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t at = rest + u * 256 + threadIdx.x, q = at / uint32_t(upr), v = at - q * uint32_t(upr);
                const bool in = i0 + u * 256 + threadIdx.x < all;
                left[u] = in ? hidden - int(v * 8) : 0;
                e[u] = left[u] > 0 ? (row0 + q) * hidden + int64_t(v) * 8 : 0;
                scale[u] = (row0 + q) * (upr / 4) + v / 4;
            }
        }
    }
};

constexpr int PACK_U = 2, UNPACK_U = 4;

// 65536 x 4096 bf16: 144 us for 814 MB, 5.7 TB/s, past a copy's rate, with two units in flight a thread.  Rows of whole blocks need
// neither the division nor the checks behind a row's end.
template <bool FLAT>
__global__ __launch_bounds__(256) void pack_kernel(PackParams p, int upr, int64_t all) {
    constexpr int U = PACK_U;
    const int64_t total = p.n_rows * p.hidden;
    // whole waves take part, so that a block's four lanes do
    for (int64_t i0 = int64_t(blockIdx.x) * (256 * U); i0 < all; i0 += int64_t(gridDim.x) * (256 * U)) {
        const Units<FLAT, U> at(i0, all, p.hidden, upr);
        Raw8 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = load8<FLAT>(p.x, p.x_bf16, at.e[u], total);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int left = at.left[u];
            float f[8];
            uint32_t most = 0;
            unpack8(f, raw[u], p.x_bf16);
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                if (!FLAT && c >= left) f[c] = 0.0f;
                most = max(most, finite_bits(f[c]));
            }
            const uint32_t code = scale_code(max_quad(most));
            const float inverse = scale_inverse(code);
#pragma unroll
            for (int c = 0; c < 8; ++c) f[c] = scaled(f[c], code, inverse);
            if (left <= 0) continue;
            uint8_t* q = p.q + at.e[u];
            const uint32_t lo = pack_e4m3(f[0], f[1], f[2], f[3]), hi = pack_e4m3(f[4], f[5], f[6], f[7]);
            if (FLAT || left >= 8) {
                *reinterpret_cast<u32x2_a1*>(q) = u32x2_a1{lo, hi};
            } else {
                for (int c = 0; c < left; ++c) q[c] = uint8_t((c < 4 ? lo : hi) >> (c % 4 * 8));
            }
            if (threadIdx.x % 4 == 0) p.q_scale[at.scale[u]] = uint8_t(code);
        }
    }
}

// act(z).  GELU to be stored in bf16: z Phi(z) as max(z, 0) - |z| Phi(-|z|), two instructions less than the choice between
// Phi(-|z|) and 1 - Phi(-|z|), at a rounding less.  FAR: z may be +inf, which stays finite beside Phi(-inf) = 0; the same bits
// for every other z.
template <int ACT, bool FINE, bool FAR>
__device__ __forceinline__ float packed_act(float z) {
    if constexpr (ACT == ACT_GELU_ERF && !FINE) {
        float e;
        const float m = __builtin_fabsf(FAR ? __builtin_fminf(z, 3.4028234663852886e38f) : z);
        return __builtin_fmaf(-m, normal_tail(z, e), __builtin_fmaxf(z, 0.0f));
    } else {
        return act_value<ACT, FINE>(z);
    }
}

// FINE: an output is stored in fp32, and the activation as exact as that shows.
//
// 65536 x 4096 bf16: the identity 133 us for 814 MB, 6.1 TB/s, GELU's output 160, 5.1 (its instructions, 21 a value, not all
// of them behind the loads), and its gradient and output in one pass 334 for 1.89 GB, 5.7.  Four units in flight: with two
// 10 us more for GELU, with eight 5.
template <int ACT, bool FLAT, bool FINE>
__global__ __launch_bounds__(256) void unpack_kernel(UnpackParams p, int upr, int64_t all) {
    constexpr int U = UNPACK_U;
    const int64_t total = p.n_rows * p.hidden;
    for (int64_t i0 = int64_t(blockIdx.x) * (256 * U); i0 < all; i0 += int64_t(gridDim.x) * (256 * U)) {
        const Units<FLAT, U> at(i0, all, p.hidden, upr);
        uint32_t w[U][2], code[U];
        Raw8 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t e = at.e[u];
            w[u][0] = w[u][1] = 0;
            if (FLAT || e + 8 <= total) {
                const u32x2_a1 v = *reinterpret_cast<const u32x2_a1*>(p.q + e);
                w[u][0] = v.x;
                w[u][1] = v.y;
            } else {
                for (int c = 0; c < 8 && e + c < total; ++c) w[u][c / 4] |= uint32_t(p.q[e + c]) << (c % 4 * 8);
            }
            code[u] = p.q_scale[at.left[u] > 0 ? at.scale[u] : 0];
        }
        if (p.dx) {
#pragma unroll
            for (int u = 0; u < U; ++u) raw[u] = load8<FLAT>(p.dy, p.dy_bf16, at.e[u], total);
        }
        auto units = [&](auto far) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int left = at.left[u];
                if (left <= 0) continue;
                const float scale = scale_value(code[u]);
                float z[8], f[8];
                unpack_e4m3(z, w[u][0], scale);
                unpack_e4m3(z + 4, w[u][1], scale);
                if (p.dx) {
                    unpack8(f, raw[u], p.dy_bf16);
#pragma unroll
                    for (int c = 0; c < 8; ++c) f[c] *= act_slope<ACT, FINE>(z[c]);
                    store8(p.dx, p.dx_bf16, at.e[u], FLAT ? 8 : left, f);
                }
                if (p.y) {
#pragma unroll
                    for (int c = 0; c < 8; ++c) f[c] = packed_act<ACT, FINE, far.value>(z[c]);
                    store8(p.y, p.y_bf16, at.e[u], FLAT ? 8 : left, f);
                }
            }
        };
        if constexpr (ACT == ACT_GELU_ERF && !FINE) {
            // a wave's own form where a scale of its units reaches past fp32: 65536 x 4096, GELU's output 160 us, its gradient
            // and output 334, and 159 and 339 without it (a minimum for each value: 169 and 356)
            if (__any(max(max(code[0], code[1]), max(code[2], code[3])) >= INFINITE_CODE)) units(std::true_type{});
            else units(std::false_type{});
        } else {
            units(std::true_type{});
        }
    }
}

int units_of(int32_t hidden) { return int(pack_blocks(hidden)) * 4; }

// A turn a workgroup: with loops over a capped grid packing 65536 x 4096 bf16 took 155 us, 144 so (a launch holds less than
// 2^32 threads).
unsigned grid_of(int64_t all, int per) {
    return unsigned(std::min<int64_t>((all + per - 1) / per, int64_t(1) << 23));
}

}  // namespace

hipError_t run_pack_rows(const PackParams& p, const DeviceInfo& dev, hipStream_t stream) {
    const int upr = units_of(p.hidden);
    const int64_t all = p.n_rows * upr;
    const unsigned grid = grid_of(all, 256 * PACK_U);
    if (p.hidden % PACK_BLOCK == 0) hipLaunchKernelGGL(pack_kernel<true>, dim3(grid), dim3(256), 0, stream, p, upr, all);
    else hipLaunchKernelGGL(pack_kernel<false>, dim3(grid), dim3(256), 0, stream, p, upr, all);
    return hipGetLastError();
}

hipError_t run_unpack_rows(const UnpackParams& p, const DeviceInfo& dev, hipStream_t stream) {
    const int upr = units_of(p.hidden);
    const int64_t all = p.n_rows * upr;
    const unsigned grid = grid_of(all, 256 * UNPACK_U);
    const bool flat = p.hidden % PACK_BLOCK == 0, fine = (p.dx && !p.dx_bf16) || (p.y && !p.y_bf16);
    auto launch = [&](auto act) {
        constexpr int ACT = act.value;
        auto of = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, stream, p, upr, all); };
        if (flat) fine ? of(unpack_kernel<ACT, true, true>) : of(unpack_kernel<ACT, true, false>);
        else fine ? of(unpack_kernel<ACT, false, true>) : of(unpack_kernel<ACT, false, false>);
    };
    if (p.act == ACT_GELU_ERF) launch(std::integral_constant<int, ACT_GELU_ERF>{});
    else if (p.act == ACT_GELU_TANH) launch(std::integral_constant<int, ACT_GELU_TANH>{});
    else launch(std::integral_constant<int, ACT_IDENTITY>{});
    return hipGetLastError();
}

}  // namespace fff

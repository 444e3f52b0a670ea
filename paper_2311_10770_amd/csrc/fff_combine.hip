// fff_combine.hip -- the rows of a token's experts added up, and the gradients
// (fff_combine, fff_combine_backward).
//
//   y_t = residual_t + sum_j w_tj row_tj;  drow_tj = w_tj dy_t;  dw_tj = <dy_t, row_tj>
//
// Bound by the rows' bytes: every row is read or written once, eight columns a lane.
#include "fff_device.hpp"
#include "fff_operators.hpp"
#include "fff_rows.hpp"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

namespace fff {

namespace {

// A thread takes eight columns of a token; U rows are in flight at a time.  16384 x 8 rows of 1024 bf16, few of them without
// an expert, onto an fp32 stream: 71 us for 386 MB, 5.4 TB/s, past a copy's rate.  8 tokens x 8 rows of 4096: 4.4 us, which
// the launch is most of.
constexpr int U = 4;
__global__ __launch_bounds__(256) void combine_kernel(CombineParams p, int vecs, int64_t all) {
    const int64_t entries = p.n_tokens * p.top_k, total = entries * p.hidden, ytotal = p.n_tokens * p.hidden;
    for (int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x; i < all; i += int64_t(gridDim.x) * 256) {
        const int64_t t = i / vecs;
        const int col = int(i - t * vecs) * 8;
        const int64_t e0 = t * p.top_k;
        float acc[8] = {};
        for (int j0 = 0; j0 < p.top_k; j0 += U) {
            Raw8 r[U];
            float w[U];
            bool live[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int j = j0 + u;
                live[u] = j < p.top_k && (!p.ids || p.ids[e0 + j] >= 0);
                w[u] = live[u] && p.weights ? p.weights[e0 + j] : 1.0f;
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (live[u]) r[u] = load8(p.rows, p.rows_bf16, (e0 + j0 + u) * p.hidden + col, total);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (!live[u]) continue;
                float f[8];
                unpack8(f, r[u], p.rows_bf16);
#pragma unroll
                for (int c = 0; c < 8; ++c) acc[c] = __builtin_fmaf(w[u], f[c], acc[c]);
            }
        }
        if (p.residual) {
            float f[8];
            unpack8(f, load8(p.residual, p.y_bf16, t * p.hidden + col, ytotal), p.y_bf16);
#pragma unroll
            for (int c = 0; c < 8; ++c) acc[c] += f[c];
        }
        store8(p.y, p.y_bf16, t * p.hidden + col, p.hidden - col, acc);
    }
}

// Eight columns from element e on, with OWN those alone that lie behind the first `skip`.
template <bool OWN>
__device__ __forceinline__ void store_own(void* base, int bf, int64_t e, int skip, const float* f) {
    if (OWN && skip) {
#pragma unroll
        for (int c = 1; c < 8; ++c)
            if (c >= skip) store_elem(base, bf, e + c, f[c]);
    } else {
        store8(base, bf, e, 8, f);
    }
}

// LPE lanes an entry, two vectors of eight columns a lane in flight.  A vector that would end behind its row starts
// earlier instead, so that all of it lies in the row: its first columns are another lane's, and left out of the sum
// (16384 x 4 rows of 1001 bf16 with both gradients: 72 -> 68 us, of 1024: 62, 4.8 TB/s; 22085 x 5 rows of 133
// without the weights': 25.5 -> 18.5).  SHORT: rows of less than eight columns, a column at a time.
//
// drows may be the buffer rows: a wave reads a row's columns before it writes their gradient there, and what two of its
// lanes write is the same from both.  Where a row is shared by several waves (LPE 256), whose order is
// open, a lane writes its own columns alone.  A token's entries are neighbours: its dy comes from the caches but once.
template <int LPE, bool SHORT>
__global__ __launch_bounds__(256) void combine_bwd_kernel(CombineBwdParams p) {
    constexpr int EPB = 256 / LPE, STEP = LPE * 8;
    __shared__ float red[LPE == 256 ? 4 : 1];
    const int sl = threadIdx.x % LPE;
    const uint32_t H = p.hidden;
    const int64_t entries = p.n_tokens * p.top_k;
    for (int64_t e0 = int64_t(blockIdx.x) * EPB; e0 < entries; e0 += int64_t(gridDim.x) * EPB) {
        const int64_t e = e0 + threadIdx.x / LPE;
        if (e >= entries) break;
        const int64_t t = uint32_t(e) / uint32_t(p.top_k);
        const bool live = !p.ids || p.ids[e] >= 0;
        const float w = live && p.weights ? p.weights[e] : 1.0f;
        const bool dot = live && p.dweights;
        float acc = 0.0f;
        if constexpr (SHORT) {
            if (uint32_t(sl) < H) {
                const float dy = live ? load_elem(p.dy, p.y_bf16, t * H + sl) : 0.0f;
                if (dot) acc = dy * load_elem(p.rows, p.rows_bf16, e * H + sl);
                if (p.drows) store_elem(p.drows, p.drows_bf16, e * H + sl, live ? w * dy : 0.0f);
            }
        } else {
            for (uint32_t c0 = sl * 8; c0 < H; c0 += 2 * STEP) {
                Raw8 dy[2], row[2];
                uint32_t col[2];
                int skip[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const uint32_t c = c0 + u * STEP;
                    col[u] = c + 8 <= H ? c : H - 8;
                    skip[u] = c < H ? int(c - col[u]) : 8;
                    if (live && skip[u] < 8) dy[u] = load8<true>(p.dy, p.y_bf16, t * H + col[u], 0);
                }
                if (dot) {
#pragma unroll
                    for (int u = 0; u < 2; ++u)
                        if (skip[u] < 8) row[u] = load8<true>(p.rows, p.rows_bf16, e * H + col[u], 0);
                }
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    if (skip[u] == 8) continue;
                    float f[8] = {}, g[8];
                    if (live) unpack8(f, dy[u], p.y_bf16);
                    if (dot) {
                        unpack8(g, row[u], p.rows_bf16);
#pragma unroll
                        for (int c = 0; c < 8; ++c) acc = c >= skip[u] ? __builtin_fmaf(f[c], g[c], acc) : acc;
                    }
                    if (!p.drows) continue;
                    if (live) {
#pragma unroll
                        for (int c = 0; c < 8; ++c) f[c] *= w;
                    }
                    store_own<(LPE > 64)>(p.drows, p.drows_bf16, e * H + col[u], skip[u], f);
                }
            }
        }
        if (p.dweights) {
            acc = group_sum<LPE < 64 ? LPE : 64>(acc);
            if constexpr (LPE == 256) {
                __syncthreads();  // a turn's sums are read before the next one's are written
                if (sl % 64 == 0) red[sl / 64] = acc;
                __syncthreads();
                acc = (red[0] + red[1]) + (red[2] + red[3]);
            }
            if (sl == 0) p.dweights[e] = acc;
        }
    }
}

// The gradients of many tokens' rows: LPT lanes a token, U of its rows in flight, for which its dy is read once (by the next U
// again, out of the caches).  Vectors as above.  us, into buffers in turn, beside the kernel above: 16384 x 4 rows of 1001 bf16, both gradients 64 (4.5 TB/s; of
// 1024 columns, whole lines of memory, 56, 5.3) and 72; 65536 x 4 of 768 with weights 163 and 214; 16384 x 8 of 4096 430
// and 451; 65536 x 8 of 64, into one buffer, 29 and 54; but 9000 x 5 of 1024 fp32 87 and 82 (bf16 42 and 45).  A row takes one or two turns of its
// lanes (16384 x 8 of 2048: four of a wave 238, one of 256 lanes 205).  Fewer tokens than fill the chip leave it to the
// kernel above (256 x 8 rows of 4096 with a wave a token: 26 and 12).
template <int LPT>
__global__ __launch_bounds__(256) void combine_bwd_token_kernel(CombineBwdParams p) {
    __shared__ float red[2][U][4];
    const int sl = threadIdx.x % LPT;
    const uint32_t H = p.hidden;
    const int in_group = threadIdx.x / LPT;
    int turn = 0;
    for (int64_t t0 = int64_t(blockIdx.x) * (256 / LPT); t0 < p.n_tokens; t0 += int64_t(gridDim.x) * (256 / LPT)) {
        const int64_t t = t0 + (LPT >= 64 ? __builtin_amdgcn_readfirstlane(in_group) : in_group);
        if (t >= p.n_tokens) break;
        const int64_t e0 = t * p.top_k;
        for (int j0 = 0; j0 < p.top_k; j0 += U) {
            float w[U], acc[U] = {};
            bool in[U], live[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                in[u] = j0 + u < p.top_k;
                live[u] = in[u] && (!p.ids || p.ids[e0 + j0 + u] >= 0);
                w[u] = live[u] && p.weights ? p.weights[e0 + j0 + u] : 1.0f;
            }
            for (uint32_t c = sl * 8; c < H; c += LPT * 8) {
                const uint32_t col = c + 8 <= H ? c : H - 8;
                const int skip = int(c - col);
                Raw8 row[U];
                float dy[8];
                const Raw8 d = load8<true>(p.dy, p.y_bf16, t * H + col, 0);
                if (p.dweights) {
#pragma unroll
                    for (int u = 0; u < U; ++u)
                        if (live[u]) row[u] = load8<true>(p.rows, p.rows_bf16, (e0 + j0 + u) * H + col, 0);
                }
                unpack8(dy, d, p.y_bf16);
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (!in[u]) continue;
                    float f[8];
                    if (live[u] && p.dweights) {
                        unpack8(f, row[u], p.rows_bf16);
#pragma unroll
                        for (int i = 0; i < 8; ++i) acc[u] = i >= skip ? __builtin_fmaf(dy[i], f[i], acc[u]) : acc[u];
                    }
                    if (!p.drows) continue;
#pragma unroll
                    for (int i = 0; i < 8; ++i) f[i] = live[u] ? w[u] * dy[i] : 0.0f;
                    store_own<(LPT > 64)>(p.drows, p.drows_bf16, (e0 + j0 + u) * H + col, skip, f);
                }
            }
            if (p.dweights) {
#pragma unroll
                for (int u = 0; u < U; ++u) acc[u] = group_sum<LPT < 64 ? LPT : 64>(acc[u]);
                if constexpr (LPT == 256) {
                    if (sl % 64 == 0) {
#pragma unroll
                        for (int u = 0; u < U; ++u) red[turn][u][sl / 64] = acc[u];
                    }
                    __syncthreads();
#pragma unroll
                    for (int u = 0; u < U; ++u) acc[u] = (red[turn][u][0] + red[turn][u][1]) + (red[turn][u][2] + red[turn][u][3]);
                    turn ^= 1;
                }
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (sl == 0 && in[u]) p.dweights[e0 + j0 + u] = acc[u];
            }
        }
    }
}

constexpr int64_t MOST = int64_t(1) << 23;  // workgroups: a launch holds less than 2^32 threads

}  // namespace

hipError_t run_combine(const CombineParams& p, const DeviceInfo& dev, hipStream_t stream) {
    const int vecs = int((int64_t(p.hidden) + 7) / 8);
    const int64_t all = p.n_tokens * vecs;
    const unsigned grid = unsigned(std::min<int64_t>((all + 255) / 256, MOST));
    hipLaunchKernelGGL(combine_kernel, dim3(grid), dim3(256), 0, stream, p, vecs, all);
    return hipGetLastError();
}

hipError_t run_combine_backward(const CombineBwdParams& p, const DeviceInfo& dev, hipStream_t stream) {
    const int64_t entries = p.n_tokens * p.top_k;
    auto launch = [&](auto kernel, int lanes) {
        const int per = 256 / lanes;
        const unsigned grid = unsigned(std::min<int64_t>((entries + per - 1) / per, 64 * std::max(dev.cu_count, 1)));
        hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, stream, p);
    };
    auto tokens = [&](auto kernel, int lanes) {
        const int per = 256 / lanes;
        const unsigned grid = unsigned(std::min<int64_t>((p.n_tokens + per - 1) / per, MOST));
        hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, stream, p);
    };
    if (p.hidden < 8) launch(combine_bwd_kernel<16, true>, 16);
    // two thousand waves: eight a CU.  us, lanes a token and lanes an entry, at half of a bound, at it and at twice as many
    // tokens, 8 bf16 rows each, both gradients: 64 columns 5.6 and 4.6, 7.1 8.2, 9.6 12.5; 128 6.9 6.1, 9.1 8.9, 13.9 14.0; 256
    // 7.0 5.6, 9.4 9.6, 13.8 14.7; 1024 10.6 10.0, 13.9 15.2, 29.0 33.7; 4096 11.7 11.8, 15.0 14.7, 29.1 42.2.  Of two rows
    // a token the same within 0.2 at the bounds (4096 columns 6.9 10.9).  fp32 rows of up to 1024 columns gain nothing, which
    // the rule leaves out: 8 of 128 18.4 14.4, at four times the bound 67 58; 8 of 1024 35.6 35.6 and 119 112
    else if (p.n_tokens >= 8192 && p.hidden <= 128) tokens(combine_bwd_token_kernel<16>, 16);
    else if (p.n_tokens >= 4096 && p.hidden <= 256) tokens(combine_bwd_token_kernel<32>, 32);
    else if (p.n_tokens >= 2048 && p.hidden <= 1024) tokens(combine_bwd_token_kernel<64>, 64);
    else if (p.n_tokens >= 512 && p.hidden > 1024) tokens(combine_bwd_token_kernel<256>, 256);
    else if (p.hidden <= 256) launch(combine_bwd_kernel<16, false>, 16);
    else if (p.hidden <= 512) launch(combine_bwd_kernel<32, false>, 32);
    // few entries of long rows: a workgroup each (one row of 16384: 18 us with a wave, 10.6 so, which is the host's)
    else if (p.hidden > 2048 && entries <= 2 * std::max(dev.cu_count, 1)) launch(combine_bwd_kernel<256, false>, 256);
    else launch(combine_bwd_kernel<64, false>, 64);
    return hipGetLastError();
}

}  // namespace fff

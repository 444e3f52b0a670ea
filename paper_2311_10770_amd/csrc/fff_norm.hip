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
#include "fff_operators.hpp"
#include "fff_rows.hpp"

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

// Gains or shifts of columns col .. col + 3 (16-byte aligned: col is a multiple of 4).
template <bool FULL>
__device__ __forceinline__ void gain4(float* f, const float* g, int col, int left, float absent) {
    Raw4 r;
    if (g) {
        r = load4<FULL>(g, 0, col, left);
        unpack4(f, r, 0);
    } else {
        f[0] = f[1] = f[2] = f[3] = absent;
    }
}

// Threads of a row kernel's workgroup for LPR lanes a row.
constexpr int row_threads(int lpr) { return lpr > 256 ? lpr : 256; }

// Sums of a and b over the LPR lanes of a row; every lane gets the same bits.  Rows of several
// waves add over LDS: red is [2][waves], and calls alternate between two such, so one barrier a call
// is enough (a wave writes a buffer again only behind the barrier of the call between).
template <int LPR>
__device__ __forceinline__ void row_sums(float& a, float& b, float* red) {
    if constexpr (LPR <= 64) {
        a = group_sum<LPR>(a);
        b = group_sum<LPR>(b);
    } else {
        constexpr int W = LPR / 64;
        a = group_sum<64>(a);
        b = group_sum<64>(b);
        if ((threadIdx.x & 63) == 0) {
            red[threadIdx.x >> 6] = a;
            red[W + (threadIdx.x >> 6)] = b;
        }
        __syncthreads();
        a = b = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w) {
            a += red[w];
            b += red[W + w];
        }
    }
}

// Rows held in registers: LPR lanes a row, lane sl holding the NV generator blocks of four columns
// c LPR + sl.  One read and one write of every byte; the variance is of the centred values.
// FULL: the row is exactly LPR NV blocks long (no checks).
template <int LPR, int NV, bool DROP, bool FULL>
__global__ __launch_bounds__(row_threads(LPR)) void norm_kernel(NormParams p) {
    constexpr int NT = row_threads(LPR), RPB = NT / LPR;
    __shared__ float red[2][2 * (LPR / 64 + 1)];
    const int sl = threadIdx.x % LPR, H = p.hidden;
    const float width = float(H);  // divided by: its inverse would be another rounding of every mean
    const uint64_t off = DROP ? rng_offset(p.drop) : 0;
    for (int64_t r0 = int64_t(blockIdx.x) * RPB; r0 < p.n_tokens; r0 += int64_t(gridDim.x) * RPB) {
        const int64_t row = r0 + threadIdx.x / LPR;
        if (RPB > 1 && row >= p.n_tokens) break;
        Raw4 rx[NV], rr[NV];
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int col = (c * LPR + sl) * 4;
            rx[c] = load4<FULL>(p.x, p.x_bf16, row * H + col, H - col);
        }
        if (p.residual) {
#pragma unroll
            for (int c = 0; c < NV; ++c) {
                const int col = (c * LPR + sl) * 4;
                rr[c] = load4<FULL>(p.residual, p.s_bf16, row * H + col, H - col);
            }
        }
        float f[NV][4], sum = 0.0f, none = 0.0f;
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            unpack4(f[c], rx[c], p.x_bf16);
            if (DROP) drop4(f[c], p.drop, off, uint32_t(c * LPR + sl), uint32_t(row));
        }
        if (p.residual) {
#pragma unroll
            for (int c = 0; c < NV; ++c) {
                float g[4];
                unpack4(g, rr[c], p.s_bf16);
#pragma unroll
                for (int j = 0; j < 4; ++j) f[c][j] += g[j];
            }
        }
        if (p.s) {
#pragma unroll
            for (int c = 0; c < NV; ++c) {
                const int col = (c * LPR + sl) * 4;
                store4<FULL>(p.s, p.s_bf16, row * H + col, H - col, f[c]);
            }
        }
#pragma unroll
        for (int c = 0; c < NV; ++c) sum += (f[c][0] + f[c][1]) + (f[c][2] + f[c][3]);
        row_sums<LPR>(sum, none, red[0]);
        const float mean = sum / width;
        float sq = 0.0f;
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int left = H - (c * LPR + sl) * 4;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                f[c][j] -= mean;
                if (FULL || j < left) sq = __builtin_fmaf(f[c][j], f[c][j], sq);
            }
        }
        row_sums<LPR>(sq, none, red[1]);
        const float rstd = 1.0f / sqrtf(sq / width + p.eps);
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int col = (c * LPR + sl) * 4;
            float g[4], b[4];
            gain4<FULL>(g, p.gamma, col, H - col, 1.0f);
            gain4<FULL>(b, p.beta, col, H - col, 0.0f);
#pragma unroll
            for (int j = 0; j < 4; ++j) g[j] = __builtin_fmaf(f[c][j] * rstd, g[j], b[j]);
            store4<FULL>(p.y, p.y_bf16, row * H + col, H - col, g);
        }
        if (sl == 0) {
            if (p.mean) p.mean[row] = mean;
            if (p.rstd) p.rstd[row] = rstd;
        }
    }
}

// The gradients of rows held in registers, as norm_kernel holds them.  Every workgroup sums dgamma
// and dbeta over its rows in registers and leaves one pair of partial rows.
template <int LPR, int NV, bool DROP, bool FULL>
__global__ __launch_bounds__(row_threads(LPR)) void norm_bwd_kernel(NormBwdParams p) {
    constexpr int NT = row_threads(LPR), RPB = NT / LPR, W = LPR * NV * 4;
    __shared__ float red[2][2 * (LPR / 64 + 1)];
    __shared__ float cols[RPB > 1 ? 2 * W : 1];
    const int sl = threadIdx.x % LPR, H = p.hidden;
    const float width = float(H);  // divided by: its inverse would be another rounding of every mean
    const uint64_t off = DROP ? rng_offset(p.drop) : 0;
    const bool sums = p.dgamma || p.dbeta, rows_out = p.ds || p.dx;
    float gain[NV][4], dg[NV][4] = {}, db[NV][4] = {};
#pragma unroll
    for (int c = 0; c < NV; ++c) {
        const int col = (c * LPR + sl) * 4;
        gain4<FULL>(gain[c], p.gamma, col, H - col, 1.0f);
    }
    int turn = 0;
    for (int64_t r0 = int64_t(blockIdx.x) * RPB; r0 < p.n_tokens; r0 += int64_t(gridDim.x) * RPB) {
        const int64_t row = r0 + threadIdx.x / LPR;
        if (RPB > 1 && row >= p.n_tokens) break;
        Raw4 ry[NV], rs[NV], ru[NV];
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int col = (c * LPR + sl) * 4;
            ry[c] = load4<FULL>(p.dy, p.y_bf16, row * H + col, H - col);
        }
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int col = (c * LPR + sl) * 4;
            rs[c] = load4<FULL>(p.s, p.s_bf16, row * H + col, H - col);
        }
        if (p.ds_in && rows_out) {
#pragma unroll
            for (int c = 0; c < NV; ++c) {
                const int col = (c * LPR + sl) * 4;
                ru[c] = load4<FULL>(p.ds_in, p.s_bf16, row * H + col, H - col);
            }
        }
        const float mean = p.mean[row], rstd = p.rstd[row];
        float g[NV][4], xh[NV][4], a = 0.0f, b = 0.0f;
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            unpack4(g[c], ry[c], p.y_bf16);
            unpack4(xh[c], rs[c], p.s_bf16);
            const int left = H - (c * LPR + sl) * 4;  // columns behind the row hold zeros (-mean rstd may overflow)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                xh[c][j] = FULL || j < left ? (xh[c][j] - mean) * rstd : 0.0f;
                dg[c][j] = __builtin_fmaf(g[c][j], xh[c][j], dg[c][j]);
                db[c][j] += g[c][j];
                g[c][j] *= gain[c][j];
                a += g[c][j];
                b = __builtin_fmaf(g[c][j], xh[c][j], b);
            }
        }
        if (!rows_out) continue;
        row_sums<LPR>(a, b, red[turn]);
        turn ^= 1;
        const float c1 = a / width, c2 = b / width;
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) g[c][j] = rstd * (g[c][j] - c1 - xh[c][j] * c2);
        if (p.ds_in) {
#pragma unroll
            for (int c = 0; c < NV; ++c) {
                float u[4];
                unpack4(u, ru[c], p.s_bf16);
#pragma unroll
                for (int j = 0; j < 4; ++j) g[c][j] += u[j];
            }
        }
        if (p.ds) {
#pragma unroll
            for (int c = 0; c < NV; ++c) {
                const int col = (c * LPR + sl) * 4;
                store4<FULL>(p.ds, p.s_bf16, row * H + col, H - col, g[c]);
            }
        }
        if (p.dx) {
#pragma unroll
            for (int c = 0; c < NV; ++c) {
                const int col = (c * LPR + sl) * 4;
                if (DROP) drop4(g[c], p.drop, off, uint32_t(c * LPR + sl), uint32_t(row));
                store4<FULL>(p.dx, p.x_bf16, row * H + col, H - col, g[c]);
            }
        }
    }
    if (!sums) return;
    // the workgroup's row groups add up in order, then one row each of dgamma and dbeta is stored
    float* part = p.part + int64_t(blockIdx.x) * 2 * H;
    if constexpr (RPB > 1) {
        const int group = threadIdx.x / LPR;
        for (int q = 0; q < RPB; ++q) {
            if (group == q) {
#pragma unroll
                for (int c = 0; c < NV; ++c)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float* d = cols + (c * LPR + sl) * 4 + j;
                        d[0] = q ? d[0] + dg[c][j] : dg[c][j];
                        d[W] = q ? d[W] + db[c][j] : db[c][j];
                    }
            }
            __syncthreads();
        }
        for (int i = threadIdx.x; i < H; i += NT) {
            part[i] = cols[i];
            part[H + i] = cols[W + i];
        }
    } else {
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int col = (c * LPR + sl) * 4;
            store4<FULL>(part, 0, col, H - col, dg[c]);
            store4<FULL>(part, 0, int64_t(H) + col, H - col, db[c]);
        }
    }
}

// Sum over the workgroup of 256; every thread gets the same bits.
__device__ __forceinline__ float block_sum(float v, float* red) {
    v = group_sum<64>(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

// Rows of any length: a workgroup per row, the row read again in every pass, an element a load (4096 rows of 20000
// bf16 with residual: 821 us, 0.8 TB/s of what has to move; 16384 columns in registers: 126 us, 4.3 TB/s).
__global__ __launch_bounds__(256) void norm_any_kernel(NormParams p) {
    __shared__ float red[4];
    const uint64_t off = p.drop.on ? rng_offset(p.drop) : 0;
    const uint32_t H = p.hidden, blocks = (H + 3) / 4;  // unsigned: 4 blocks may pass 31 bits
    for (int64_t row = blockIdx.x; row < p.n_tokens; row += gridDim.x) {
        const int64_t r0 = row * H;
        auto sum4 = [&](uint32_t b, float* f) {
#pragma unroll
            for (int j = 0; j < 4; ++j) f[j] = 4 * b + j < H ? load_elem(p.x, p.x_bf16, r0 + 4 * b + j) : 0.0f;
            if (p.drop.on) drop4(f, p.drop, off, b, uint32_t(row));
            if (p.residual) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (4 * b + j < H) f[j] += load_elem(p.residual, p.s_bf16, r0 + 4 * b + j);
            }
        };
        float f[4], acc = 0.0f;
        for (uint32_t b = threadIdx.x; b < blocks; b += 256) {
            sum4(b, f);
            acc += (f[0] + f[1]) + (f[2] + f[3]);
        }
        const float mean = block_sum(acc, red) / float(H);
        acc = 0.0f;
        for (uint32_t b = threadIdx.x; b < blocks; b += 256) {
            sum4(b, f);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (4 * b + j < H) acc = __builtin_fmaf(f[j] - mean, f[j] - mean, acc);
        }
        const float rstd = 1.0f / sqrtf(block_sum(acc, red) / float(H) + p.eps);
        for (uint32_t b = threadIdx.x; b < blocks; b += 256) {
            sum4(b, f);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t c = 4 * b + j;
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
    const uint32_t H = p.hidden, blocks = (H + 3) / 4;
    for (int64_t row = blockIdx.x; row < p.n_tokens; row += gridDim.x) {
        const int64_t r0 = row * H;
        const float mean = p.mean[row], rstd = p.rstd[row];
        auto gh = [&](uint32_t c, float* g, float* xh) {
            *xh = (load_elem(p.s, p.s_bf16, r0 + c) - mean) * rstd;
            *g = load_elem(p.dy, p.y_bf16, r0 + c) * (p.gamma ? p.gamma[c] : 1.0f);
        };
        float a = 0.0f, b = 0.0f, g, xh;
        for (uint32_t c = threadIdx.x; c < H; c += 256) {
            gh(c, &g, &xh);
            a += g;
            b = __builtin_fmaf(g, xh, b);
        }
        const float c1 = block_sum(a, red) / float(H), c2 = block_sum(b, red) / float(H);
        for (uint32_t blk = threadIdx.x; blk < blocks; blk += 256) {
            float f[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t c = 4 * blk + j;
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

// dgamma and dbeta: the partial sums of 32 columns of a workgroup, 32 pieces apart, then over those.
// A launch holds less than 2^32 threads: columns past its workgroups' are taken in further turns.
constexpr int64_t SUM_GROUPS = int64_t(1) << 20;
__global__ __launch_bounds__(1024) void norm_bwd_sum_kernel(NormBwdParams p, int parts) {
    __shared__ float sum[32][33];
    const int H = p.hidden, col = threadIdx.x % 32, lane = threadIdx.x / 32;
    const int64_t all = 2 * int64_t(H);  // dgamma's columns, then dbeta's
    for (int64_t c0 = int64_t(blockIdx.x) * 32; c0 < all; c0 += int64_t(gridDim.x) * 32) {
        const int64_t c = c0 + col;
        float v = 0.0f;
        if (c < all)
            for (int q = lane; q < parts; q += 32) v += p.part[int64_t(q) * 2 * H + c];
        sum[lane][col] = v;
        __syncthreads();
        if (lane == 0 && c < all) {
            v = 0.0f;
#pragma unroll
            for (int l = 0; l < 32; ++l) v += sum[l][col];
            float* out = c < H ? p.dgamma : p.dbeta;
            if (out) {
                out += c < H ? c : c - H;
                *out = p.accumulate ? *out + v : v;
            }
        }
        __syncthreads();
    }
}

// A thread takes DU generator blocks, 256 apart; a workgroup's blocks are consecutive, rows being
// `vecs` blocks long (step_q and step_v: 256 / vecs and 256 % vecs, so only the first place of a
// thread is divided for).  Threads behind the last block load it again and store nothing: loads
// without a branch stay in flight together.
constexpr int DU = 4;
template <bool DROP, bool FULL>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutParams p, int vecs, int64_t all, uint32_t step_q,
                                                      uint32_t step_v) {
    const uint64_t off = DROP ? rng_offset(p.drop) : 0;
    const int H = p.hidden;
    for (int64_t i0 = int64_t(blockIdx.x) * (256 * DU); i0 < all; i0 += int64_t(gridDim.x) * (256 * DU)) {
        const int64_t row0 = i0 / vecs;
        const uint32_t at = uint32_t(i0 - row0 * vecs) + threadIdx.x;
        const int count = int(all - i0 < 256 * DU ? all - i0 : 256 * DU);
        uint32_t q = at / uint32_t(vecs), v = at - q * uint32_t(vecs);
        int64_t e[DU];
        uint32_t qs[DU], vs[DU];
        Raw4 rx[DU], rr[DU];
#pragma unroll
        for (int u = 0; u < DU; ++u) {
            const bool in = u * 256 + int(threadIdx.x) < count;
            qs[u] = in ? q : 0;
            vs[u] = in ? v : uint32_t(vecs - 1);
            e[u] = in ? (row0 + q) * H + 4 * int64_t(v) : (p.n_tokens - 1) * H + 4 * int64_t(vecs - 1);
            rx[u] = load4<FULL>(p.x, p.x_bf16, e[u], H - 4 * int(vs[u]));
            q += step_q;
            v += step_v;
            if (v >= uint32_t(vecs)) {
                v -= uint32_t(vecs);
                ++q;
            }
        }
        if (p.residual) {
#pragma unroll
            for (int u = 0; u < DU; ++u) rr[u] = load4<FULL>(p.residual, p.r_bf16, e[u], H - 4 * int(vs[u]));
        }
#pragma unroll
        for (int u = 0; u < DU; ++u) {
            float f[4], g[4];
            unpack4(f, rx[u], p.x_bf16);
            if (DROP) drop4(f, p.drop, off, vs[u], uint32_t(row0 + qs[u]));
            if (p.residual) {
                unpack4(g, rr[u], p.r_bf16);
#pragma unroll
                for (int j = 0; j < 4; ++j) f[j] += g[j];
            }
            if (u * 256 + int(threadIdx.x) < count) store4<FULL>(p.y, p.y_bf16, e[u], H - 4 * int(vs[u]), f);
        }
    }
}

// Lanes a row and generator blocks a lane of the register kernels: the first that holds the row.
struct RowShape {
    int lanes, nv;
};
constexpr RowShape ROW_SHAPES[] = {{16, 1},  {32, 1},  {64, 1},  {64, 2},   {64, 3},  {64, 4},
                                    {256, 2}, {256, 3}, {256, 4}, {1024, 2}, {1024, 4}};
constexpr int N_ROW_SHAPES = sizeof ROW_SHAPES / sizeof ROW_SHAPES[0];
int row_shape(int32_t hidden) {
    for (int i = 0; i < N_ROW_SHAPES; ++i)
        if (int64_t(ROW_SHAPES[i].lanes) * ROW_SHAPES[i].nv * 4 >= hidden) return i;
    return -1;  // longer: a workgroup per row that reads it again for every pass
}
int rows_per_group(int32_t hidden) {
    const int i = row_shape(hidden);
    return i < 0 ? 8 : row_threads(ROW_SHAPES[i].lanes) / ROW_SHAPES[i].lanes;
}

template <int I, bool DROP, bool FULL>
void launch_norm(const NormParams& p, unsigned grid, hipStream_t stream) {
    hipLaunchKernelGGL((norm_kernel<ROW_SHAPES[I].lanes, ROW_SHAPES[I].nv, DROP, FULL>), dim3(grid),
                       dim3(row_threads(ROW_SHAPES[I].lanes)), 0, stream, p);
}
template <int I, bool DROP, bool FULL>
void launch_norm(const NormBwdParams& p, unsigned grid, hipStream_t stream) {
    hipLaunchKernelGGL((norm_bwd_kernel<ROW_SHAPES[I].lanes, ROW_SHAPES[I].nv, DROP, FULL>), dim3(grid),
                       dim3(row_threads(ROW_SHAPES[I].lanes)), 0, stream, p);
}
template <int I, class P>
void launch_rows(int shape, const P& p, unsigned grid, hipStream_t stream) {
    if constexpr (I < N_ROW_SHAPES) {
        if (shape != I) return launch_rows<I + 1>(shape, p, grid, stream);
        const bool full = p.hidden == ROW_SHAPES[I].lanes * ROW_SHAPES[I].nv * 4;
        if (p.drop.on) full ? launch_norm<I, true, true>(p, grid, stream) : launch_norm<I, true, false>(p, grid, stream);
        else full ? launch_norm<I, false, true>(p, grid, stream) : launch_norm<I, false, false>(p, grid, stream);
    }
}

// Workgroups of the backward, each leaving one pair of partial rows: two a CU at most.
int norm_parts(int64_t n_tokens, int32_t hidden) {
    const int per = rows_per_group(hidden);
    return int(std::min<int64_t>(512, (n_tokens + per - 1) / per));
}

}  // namespace

hipError_t run_layer_norm(const NormParams& p, const DeviceInfo& dev, hipStream_t stream) {
    const int shape = row_shape(p.hidden), cus = std::max(dev.cu_count, 1);
    if (shape < 0) {
        const unsigned grid = unsigned(std::min<int64_t>(p.n_tokens, 8 * cus));
        hipLaunchKernelGGL(norm_any_kernel, dim3(grid), dim3(256), 0, stream, p);
        return hipGetLastError();
    }
    const int per = rows_per_group(p.hidden);
    launch_rows<0>(shape, p, unsigned(std::min<int64_t>((p.n_tokens + per - 1) / per, 16 * cus)), stream);
    return hipGetLastError();
}

size_t norm_bwd_workspace_bytes(int64_t n_tokens, int32_t hidden) {
    return size_t(norm_parts(n_tokens, hidden)) * 2 * size_t(hidden) * sizeof(float);
}

hipError_t run_layer_norm_backward(const NormBwdParams& p, const DeviceInfo& dev, hipStream_t stream) {
    const int shape = row_shape(p.hidden), parts = norm_parts(p.n_tokens, p.hidden);
    const bool sums = p.dgamma || p.dbeta;
    if (p.n_tokens > 0 && shape >= 0) {
        launch_rows<0>(shape, p, unsigned(parts), stream);
    } else if (p.n_tokens > 0) {
        if (p.ds || p.dx) {
            const unsigned grid = unsigned(std::min<int64_t>(p.n_tokens, 8 * std::max(dev.cu_count, 1)));
            hipLaunchKernelGGL(norm_bwd_any_kernel, dim3(grid), dim3(256), 0, stream, p);
        }
        if (sums)
            hipLaunchKernelGGL(norm_bwd_cols_kernel, dim3(unsigned((int64_t(p.hidden) + 255) / 256), unsigned(parts)),
                               dim3(256), 0, stream, p, parts, (p.n_tokens + parts - 1) / parts);
    }
    if (sums)
        hipLaunchKernelGGL(norm_bwd_sum_kernel, dim3(unsigned(std::min<int64_t>(SUM_GROUPS, (2 * int64_t(p.hidden) + 31) / 32))),
                           dim3(1024), 0, stream, p, parts);
    return hipGetLastError();
}

hipError_t run_dropout(const DropoutParams& p, const DeviceInfo& dev, hipStream_t stream) {
    const int vecs = int((int64_t(p.hidden) + 3) / 4);
    const int64_t all = p.n_tokens * vecs;
    const unsigned grid = unsigned(std::min<int64_t>((all + 256 * DU - 1) / (256 * DU), 64 * std::max(dev.cu_count, 1)));
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, stream, p, vecs, all, 256u / unsigned(vecs), 256u % unsigned(vecs)); };
    const bool full = p.hidden % 4 == 0;
    if (p.drop.on) full ? launch(dropout_kernel<true, true>) : launch(dropout_kernel<true, false>);
    else full ? launch(dropout_kernel<false, true>) : launch(dropout_kernel<false, false>);
    return hipGetLastError();
}

}  // namespace fff

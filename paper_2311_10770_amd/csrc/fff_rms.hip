// fff_rms.hip -- RMS norm with the residual's addition, an 8-bit copy of its rows, and
// its gradients (fff_rms_norm, fff_rms_norm_backward).
//
//   s = residual + x;  y = s rstd gamma,  rstd = 1 / sqrt(mean(s^2) + eps)
//   ds = rstd (g - xh mean(g xh)) + ds_in,  xh = s rstd,  g = dy gamma;  dgamma = sum dy xh
//
// All of it is bound by the bytes of the rows; statistics, sums and gradients are held in fp32, and so is the stream s
// until everything that depends on it is formed.
#include "fff_device.hpp"
#include "fff_operators.hpp"
#include "fff_pack.hpp"
#include "fff_rows.hpp"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

namespace fff {

namespace {

// Threads of a row kernel's workgroup for LPR lanes a row.
constexpr int row_threads(int lpr) { return lpr > 256 ? lpr : 256; }

// Sum over the LPR lanes of a row; every lane gets the same bits.  Rows of several waves add over LDS;
// calls alternate between two buffers, so one barrier a call is enough.
template <int LPR>
__device__ __forceinline__ float row_sum(float v, float* red) {
    if constexpr (LPR <= 64) {
        return group_sum<LPR>(v);
    } else {
        v = group_sum<64>(v);
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int w = 0; w < LPR / 64; ++w) v += red[w];
        return v;
    }
}

// Four columns (col .. col + 3, `left` of them in the row) of a row in 8 bits; eight neighbouring lanes hold a
// block of 32 and all take part.  q and scale: the row's.
typedef uint32_t u32_a1 __attribute__((aligned(1)));
__device__ __forceinline__ void put_packed(uint8_t* q, uint8_t* scale, int col, int left, const float* f) {
    uint32_t most = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) most = max(most, j < left ? finite_bits(f[j]) : 0);
    const uint32_t code = scale_code(max_eight(most));
    const float inverse = scale_inverse(code);
    const uint32_t w = pack_e4m3(scaled(f[0], code, inverse), scaled(f[1], code, inverse), scaled(f[2], code, inverse),
                                 scaled(f[3], code, inverse));
    if (left >= 4) {
        *reinterpret_cast<u32_a1*>(q + col) = w;
    } else {
        for (int j = 0; j < left; ++j) q[col + j] = uint8_t(w >> (8 * j));
    }
    if (left > 0 && col % PACK_BLOCK == 0) scale[col / PACK_BLOCK] = uint8_t(code);
}

// How a row fits its lanes' vectors of four: exactly, in whole vectors, or with a part of one at its end.
enum { ROW_FULL = 0, ROW_WHOLE = 1, ROW_RAGGED = 2 };

// Four values of a row from element e on, `left` of them in the row, of a matrix of `all` elements; zeros behind the
// row, but that a ragged row's last vector may run on into the next one, and clear4 takes those values out (element by
// element such ends cost a row more than all its vectors: 65536 rows of 250 bf16, backward: 69 us, 33 so).  Only
// the matrix's last ones are read one by one.
template <int FIT>
__device__ __forceinline__ Raw4 row4(const void* base, int bf, int64_t e, int left, int64_t all) {
    if (FIT == ROW_FULL) return load4<true>(base, bf, e, 4);
    if (FIT == ROW_RAGGED && left > 0 && e + 4 > all) return load4<false>(base, bf, e, left);
    Raw4 r = {0, 0, 0, 0};
    if (left > 0) r = load4<true>(base, bf, e, 4);
    return r;
}
template <int FIT>
__device__ __forceinline__ void clear4(float* f, int left) {
    if (FIT != ROW_RAGGED) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = j < left ? f[j] : 0.0f;
}
template <int FIT>
__device__ __forceinline__ void put4(void* base, int bf, int64_t e, int left, const float* f) {
    if (FIT == ROW_FULL || (FIT == ROW_WHOLE && left > 0)) store4<true>(base, bf, e, 4, f);
    else if (FIT == ROW_RAGGED) store4<false>(base, bf, e, left, f);
}

template <int FIT>
__device__ __forceinline__ void gain4(float* f, const float* g, int col, int left) {
    if (g) {
        unpack4(f, load4<FIT == ROW_FULL>(g, 0, col, left), 0);
    } else {
        f[0] = f[1] = f[2] = f[3] = 1.0f;
    }
}

// Rows held in registers: LPR lanes a row, lane sl holding the NV vectors of four columns
// c LPR + sl.  One read and one write of every byte.  Rows of up to 1024 columns take a wave or less, whose sum needs no LDS;
// longer ones a workgroup.  65536 x 1024, bf16 x on an fp32 stream, with bf16 and 8-bit y: 158 us for 873 MB,
// 5.5 TB/s; one row of 4096: 2.8 us, and the host 11.
template <int LPR, int NV, int FIT>
__global__ __launch_bounds__(row_threads(LPR)) void rms_kernel(RmsParams p) {
    constexpr int NT = row_threads(LPR), RPB = NT / LPR;
    __shared__ float red[2][LPR / 64 + 1];
    const int sl = threadIdx.x % LPR, H = p.hidden;
    const int64_t blocks = pack_blocks(H), total = p.n_tokens * H;
    const float width = float(H);
    float gain[NV][4];
#pragma unroll
    for (int c = 0; c < NV; ++c) {
        const int col = (c * LPR + sl) * 4;
        gain4<FIT>(gain[c], p.gamma, col, H - col);
    }
    int turn = 0;
    for (int64_t r0 = int64_t(blockIdx.x) * RPB; r0 < p.n_tokens; r0 += int64_t(gridDim.x) * RPB) {
        const int64_t row = r0 + threadIdx.x / LPR;
        if (RPB > 1 && row >= p.n_tokens) break;
        Raw4 rx[NV], rr[NV];
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int col = (c * LPR + sl) * 4;
            rx[c] = row4<FIT>(p.x, p.x_bf16, row * H + col, H - col, total);
        }
        if (p.residual) {
#pragma unroll
            for (int c = 0; c < NV; ++c) {
                const int col = (c * LPR + sl) * 4;
                rr[c] = row4<FIT>(p.residual, p.s_bf16, row * H + col, H - col, total);
            }
        }
        float f[NV][4], sq = 0.0f;
#pragma unroll
        for (int c = 0; c < NV; ++c) unpack4(f[c], rx[c], p.x_bf16);
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
                put4<FIT>(p.s, p.s_bf16, row * H + col, H - col, f[c]);
            }
        }
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            clear4<FIT>(f[c], H - (c * LPR + sl) * 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) sq = __builtin_fmaf(f[c][j], f[c][j], sq);
        }
        sq = row_sum<LPR>(sq, red[turn]);
        turn ^= 1;
        const float rstd = 1.0f / sqrtf(sq / width + p.eps);
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int col = (c * LPR + sl) * 4;
#pragma unroll
            for (int j = 0; j < 4; ++j) f[c][j] = f[c][j] * rstd * gain[c][j];
            if (p.y) put4<FIT>(p.y, p.y_bf16, row * H + col, H - col, f[c]);
            if (p.q) put_packed(p.q + row * H, p.q_scale + row * blocks, col, H - col, f[c]);
        }
        if (sl == 0 && p.rstd) p.rstd[row] = rstd;
    }
}

// The gradients of rows held in registers, as rms_kernel holds them.  Every workgroup sums dgamma over its
// rows in registers and leaves one partial row, which rms_bwd_sum_kernel adds up in a fixed order: no atomics.
// 65536 x 768 bf16 with ds_in: 71 us and 4 for the sums, for 403 MB, 5.4 TB/s.
template <int LPR, int NV, int FIT>
__global__ __launch_bounds__(row_threads(LPR)) void rms_bwd_kernel(RmsBwdParams p) {
    constexpr int NT = row_threads(LPR), RPB = NT / LPR, W = LPR * NV * 4;
    __shared__ float red[2][LPR / 64 + 1];
    __shared__ float cols[RPB > 1 ? W : 1];
    const int sl = threadIdx.x % LPR, H = p.hidden;
    const float width = float(H);
    const int64_t total = p.n_tokens * H;
    const bool rows_out = p.ds || p.dx;
    float gain[NV][4], dg[NV][4] = {};
#pragma unroll
    for (int c = 0; c < NV; ++c) {
        const int col = (c * LPR + sl) * 4;
        gain4<FIT>(gain[c], p.gamma, col, H - col);
    }
    int turn = 0;
    for (int64_t r0 = int64_t(blockIdx.x) * RPB; r0 < p.n_tokens; r0 += int64_t(gridDim.x) * RPB) {
        const int64_t row = r0 + threadIdx.x / LPR;
        if (RPB > 1 && row >= p.n_tokens) break;
        Raw4 ry[NV], rs[NV], ru[NV];
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int col = (c * LPR + sl) * 4;
            ry[c] = row4<FIT>(p.dy, p.y_bf16, row * H + col, H - col, total);
        }
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int col = (c * LPR + sl) * 4;
            rs[c] = row4<FIT>(p.s, p.s_bf16, row * H + col, H - col, total);
        }
        if (p.ds_in && rows_out) {
#pragma unroll
            for (int c = 0; c < NV; ++c) {
                const int col = (c * LPR + sl) * 4;
                ru[c] = row4<FIT>(p.ds_in, p.s_bf16, row * H + col, H - col, total);
            }
        }
        const float rstd = p.rstd[row];
        float g[NV][4], xh[NV][4], b = 0.0f;
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            unpack4(g[c], ry[c], p.y_bf16);
            unpack4(xh[c], rs[c], p.s_bf16);
#pragma unroll
            for (int j = 0; j < 4; ++j) xh[c][j] *= rstd;
            clear4<FIT>(xh[c], H - (c * LPR + sl) * 4);
            clear4<FIT>(g[c], H - (c * LPR + sl) * 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                dg[c][j] = __builtin_fmaf(g[c][j], xh[c][j], dg[c][j]);
                g[c][j] *= gain[c][j];
                b = __builtin_fmaf(g[c][j], xh[c][j], b);
            }
        }
        if (!rows_out) continue;
        const float c2 = row_sum<LPR>(b, red[turn]) / width;
        turn ^= 1;
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) g[c][j] = rstd * (g[c][j] - xh[c][j] * c2);
        if (p.ds_in) {
#pragma unroll
            for (int c = 0; c < NV; ++c) {
                float u[4];
                unpack4(u, ru[c], p.s_bf16);
#pragma unroll
                for (int j = 0; j < 4; ++j) g[c][j] += u[j];
            }
        }
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int col = (c * LPR + sl) * 4;
            if (p.ds) put4<FIT>(p.ds, p.s_bf16, row * H + col, H - col, g[c]);
            if (p.dx) put4<FIT>(p.dx, p.x_bf16, row * H + col, H - col, g[c]);
        }
    }
    if (!p.dgamma) return;
    // the workgroup's row groups add up in order, then one row of dgamma is stored
    float* part = p.part + int64_t(blockIdx.x) * H;
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
                    }
            }
            __syncthreads();
        }
        for (int i = threadIdx.x; i < H; i += NT) part[i] = cols[i];
    } else {
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int col = (c * LPR + sl) * 4;
            put4<FIT>(part, 0, col, H - col, dg[c]);
        }
    }
}

// Rows past 16384 columns: a workgroup of 1024 a row, which is read again for the second pass.  4096 x 20000 bf16 with a
// residual: 242 us, the floor is 131 (the second pass misses the L2 where a row of each CU does not fit); 8 rows of
// 1048576 leave most of the chip idle (513 us).
constexpr int LONG = 1024;
__global__ __launch_bounds__(LONG) void rms_any_kernel(RmsParams p) {
    __shared__ float red[2][LONG / 64 + 1];
    const int H = p.hidden;
    const int64_t blocks = pack_blocks(H), turns = (int64_t(H) + 4 * LONG - 1) / (4 * LONG);
    int turn = 0;
    for (int64_t row = blockIdx.x; row < p.n_tokens; row += gridDim.x) {
        auto sum4 = [&](int64_t col, float* f) {
            const int left = int(std::min<int64_t>(4, H - col));
            unpack4(f, load4<false>(p.x, p.x_bf16, row * H + col, left), p.x_bf16);
            if (p.residual) {
                float g[4];
                unpack4(g, load4<false>(p.residual, p.s_bf16, row * H + col, left), p.s_bf16);
#pragma unroll
                for (int j = 0; j < 4; ++j) f[j] += g[j];
            }
            return left;
        };
        float f[4], sq = 0.0f;
#pragma unroll 4
        for (int64_t i = 0; i < turns; ++i) {
            sum4((i * LONG + threadIdx.x) * 4, f);
#pragma unroll
            for (int j = 0; j < 4; ++j) sq = __builtin_fmaf(f[j], f[j], sq);
        }
        sq = row_sum<LONG>(sq, red[turn]);
        turn ^= 1;
        const float rstd = 1.0f / sqrtf(sq / float(H) + p.eps);
        for (int64_t i = 0; i < turns; ++i) {
            const int64_t col = (i * LONG + threadIdx.x) * 4;
            const int left = sum4(col, f);  // may be none, but a block's lanes all take part below
            float g[4] = {1.0f, 1.0f, 1.0f, 1.0f};
            if (p.gamma) unpack4(g, load4<false>(p.gamma, 0, col, left), 0);
            if (p.s) store4<false>(p.s, p.s_bf16, row * H + col, left, f);
#pragma unroll
            for (int j = 0; j < 4; ++j) f[j] = f[j] * rstd * g[j];
            if (p.y) store4<false>(p.y, p.y_bf16, row * H + col, left, f);
            if (p.q) put_packed(p.q + row * H, p.q_scale + row * blocks, int(col), left, f);
        }
        if (threadIdx.x == 0 && p.rstd) p.rstd[row] = rstd;
    }
}

// ds and dx of rows of any length.
__global__ __launch_bounds__(LONG) void rms_bwd_any_kernel(RmsBwdParams p) {
    __shared__ float red[2][LONG / 64 + 1];
    const int64_t H = p.hidden;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < p.n_tokens; row += gridDim.x) {
        const float rstd = p.rstd[row];
        auto gh = [&](int64_t col, float* g, float* xh) {
            const int left = int(std::min<int64_t>(4, H - col));
            unpack4(xh, load4<false>(p.s, p.s_bf16, row * H + col, left), p.s_bf16);
            unpack4(g, load4<false>(p.dy, p.y_bf16, row * H + col, left), p.y_bf16);
            float gain[4] = {1.0f, 1.0f, 1.0f, 1.0f};
            if (p.gamma) unpack4(gain, load4<false>(p.gamma, 0, col, left), 0);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                xh[j] = j < left ? xh[j] * rstd : 0.0f;
                g[j] *= gain[j];
            }
            return left;
        };
        float g[4], xh[4], b = 0.0f;
        for (int64_t col = threadIdx.x * 4; col < H; col += LONG * 4) {
            gh(col, g, xh);
#pragma unroll
            for (int j = 0; j < 4; ++j) b = __builtin_fmaf(g[j], xh[j], b);
        }
        const float c2 = row_sum<LONG>(b, red[turn]) / float(H);
        turn ^= 1;
        for (int64_t col = threadIdx.x * 4; col < H; col += LONG * 4) {
            const int left = gh(col, g, xh);
#pragma unroll
            for (int j = 0; j < 4; ++j) g[j] = rstd * (g[j] - xh[j] * c2);
            if (p.ds_in) {
                float u[4];
                unpack4(u, load4<false>(p.ds_in, p.s_bf16, row * H + col, left), p.s_bf16);
#pragma unroll
                for (int j = 0; j < 4; ++j) g[j] += u[j];
            }
            if (p.ds) store4<false>(p.ds, p.s_bf16, row * H + col, left, g);
            if (p.dx) store4<false>(p.dx, p.x_bf16, row * H + col, left, g);
        }
    }
}

// Partial sums of dgamma for rows of any length: a thread takes four columns of one piece of rows.
__global__ __launch_bounds__(256) void rms_bwd_cols_kernel(RmsBwdParams p, int parts, int64_t rows_per) {
    const int64_t H = p.hidden, col = (int64_t(blockIdx.x) * 256 + threadIdx.x) * 4;
    if (col >= H) return;
    const int left = int(std::min<int64_t>(4, H - col));
    for (int q = blockIdx.y; q < parts; q += gridDim.y) {
        const int64_t r1 = std::min<int64_t>(p.n_tokens, (q + 1) * rows_per);
        float dg[4] = {};
        for (int64_t r = q * rows_per; r < r1; ++r) {
            float d[4], s[4];
            unpack4(d, load4<false>(p.dy, p.y_bf16, r * H + col, left), p.y_bf16);
            unpack4(s, load4<false>(p.s, p.s_bf16, r * H + col, left), p.s_bf16);
            const float rstd = p.rstd[r];
#pragma unroll
            for (int j = 0; j < 4; ++j) dg[j] = __builtin_fmaf(d[j], s[j] * rstd, dg[j]);
        }
        store4<false>(p.part, 0, q * H + col, left, dg);
    }
}

// dgamma: the partial sums of 32 columns a workgroup, 32 pieces apart, then over those.
constexpr int64_t SUM_GROUPS = int64_t(1) << 20;  // a launch holds less than 2^32 threads
__global__ __launch_bounds__(1024) void rms_bwd_sum_kernel(RmsBwdParams p, int parts) {
    __shared__ float sum[32][33];
    const int64_t H = p.hidden;
    const int col = threadIdx.x % 32, lane = threadIdx.x / 32;
    for (int64_t c0 = int64_t(blockIdx.x) * 32; c0 < H; c0 += int64_t(gridDim.x) * 32) {
        const int64_t c = c0 + col;
        float v = 0.0f;
        if (c < H) {
#pragma unroll 8
            for (int q = lane; q < parts; q += 32) v += p.part[q * H + c];
        }
        sum[lane][col] = v;
        __syncthreads();
        if (lane == 0 && c < H) {
            v = 0.0f;
#pragma unroll
            for (int l = 0; l < 32; ++l) v += sum[l][col];
            p.dgamma[c] = p.accumulate ? p.dgamma[c] + v : v;
        }
        __syncthreads();
    }
}

// Lanes a row and vectors of four a lane of the register kernels: the first that holds the row.
struct RowShape {
    int lanes, nv;
};
constexpr RowShape ROW_SHAPES[] = {{16, 1},  {32, 1},  {64, 1},  {64, 2},   {64, 3},  {64, 4},
                                    {256, 2}, {256, 3}, {256, 4}, {1024, 2}, {1024, 4}};
constexpr int N_ROW_SHAPES = sizeof ROW_SHAPES / sizeof ROW_SHAPES[0];
int row_shape(int32_t hidden) {
    for (int i = 0; i < N_ROW_SHAPES; ++i)
        if (int64_t(ROW_SHAPES[i].lanes) * ROW_SHAPES[i].nv * 4 >= hidden) return i;
    return -1;
}
int rows_per_group(int32_t hidden) {
    const int i = row_shape(hidden);
    return i < 0 ? 8 : row_threads(ROW_SHAPES[i].lanes) / ROW_SHAPES[i].lanes;
}

template <int I, int FIT>
void launch_rms(const RmsParams& p, unsigned grid, hipStream_t stream) {
    hipLaunchKernelGGL((rms_kernel<ROW_SHAPES[I].lanes, ROW_SHAPES[I].nv, FIT>), dim3(grid),
                       dim3(row_threads(ROW_SHAPES[I].lanes)), 0, stream, p);
}
template <int I, int FIT>
void launch_rms(const RmsBwdParams& p, unsigned grid, hipStream_t stream) {
    hipLaunchKernelGGL((rms_bwd_kernel<ROW_SHAPES[I].lanes, ROW_SHAPES[I].nv, FIT>), dim3(grid),
                       dim3(row_threads(ROW_SHAPES[I].lanes)), 0, stream, p);
}
template <int I, class P>
void launch_rows(int shape, const P& p, unsigned grid, hipStream_t stream) {
    if constexpr (I < N_ROW_SHAPES) {
        if (shape != I) return launch_rows<I + 1>(shape, p, grid, stream);
        if (p.hidden == ROW_SHAPES[I].lanes * ROW_SHAPES[I].nv * 4) launch_rms<I, ROW_FULL>(p, grid, stream);
        else if (p.hidden % 4 == 0) launch_rms<I, ROW_WHOLE>(p, grid, stream);
        else launch_rms<I, ROW_RAGGED>(p, grid, stream);
    }
}

// Workgroups of the backward, each leaving one partial row: more of them for short rows, whose partial rows are short
// too, and where one works on a row at a time with four waves (us: 65536 rows of 100 fp32, 512 and 2048: 37.9, 24.8; 9069 of
// 1522, 512 and 1024: 60, 43).
int rms_parts(int64_t n_tokens, int32_t hidden) {
    const int per = rows_per_group(hidden), shape = row_shape(hidden);
    int64_t most = std::min<int64_t>(2048, std::max<int64_t>(512, (int64_t(1) << 18) / hidden));
    if (shape >= 0 && ROW_SHAPES[shape].lanes == 256) most = 1024;
    return int(std::min<int64_t>(most, (n_tokens + per - 1) / per));
}

}  // namespace

hipError_t run_rms_norm(const RmsParams& p, const DeviceInfo& dev, hipStream_t stream) {
    const int shape = row_shape(p.hidden), cus = std::max(dev.cu_count, 1);
    if (shape < 0) {
        const unsigned grid = unsigned(std::min<int64_t>(p.n_tokens, 8 * cus));
        hipLaunchKernelGGL(rms_any_kernel, dim3(grid), dim3(LONG), 0, stream, p);
        return hipGetLastError();
    }
    // a wave a row of more than 512 columns: a row a wave, else 16 workgroups a CU that keep gamma (bf16 with a residual, us:
    // 65536 x 768 69 and 75, x 320 34 and 30, x 512 the same; 8192 x 8192 107 and 102)
    const bool once = ROW_SHAPES[shape].lanes == 64 && ROW_SHAPES[shape].nv > 2;
    const int64_t most = once ? int64_t(1) << 23 : 16 * cus;
    const int per = rows_per_group(p.hidden);
    launch_rows<0>(shape, p, unsigned(std::min<int64_t>((p.n_tokens + per - 1) / per, most)), stream);
    return hipGetLastError();
}

size_t rms_bwd_workspace_bytes(int64_t n_tokens, int32_t hidden) {
    return size_t(rms_parts(n_tokens, hidden)) * size_t(hidden) * sizeof(float);
}

hipError_t run_rms_norm_backward(const RmsBwdParams& p, const DeviceInfo& dev, hipStream_t stream) {
    const int shape = row_shape(p.hidden), parts = rms_parts(p.n_tokens, p.hidden);
    if (p.n_tokens > 0 && shape >= 0) {
        launch_rows<0>(shape, p, unsigned(parts), stream);
    } else if (p.n_tokens > 0) {
        if (p.ds || p.dx) {
            const unsigned grid = unsigned(std::min<int64_t>(p.n_tokens, 8 * std::max(dev.cu_count, 1)));
            hipLaunchKernelGGL(rms_bwd_any_kernel, dim3(grid), dim3(LONG), 0, stream, p);
        }
        if (p.dgamma)
            hipLaunchKernelGGL(rms_bwd_cols_kernel, dim3(unsigned((int64_t(p.hidden) + 1023) / 1024), unsigned(parts)),
                               dim3(256), 0, stream, p, parts, (p.n_tokens + parts - 1) / parts);
    }
    if (p.dgamma)
        hipLaunchKernelGGL(rms_bwd_sum_kernel, dim3(unsigned(std::min<int64_t>(SUM_GROUPS, (int64_t(p.hidden) + 31) / 32))),
                           dim3(1024), 0, stream, p, parts);
    return hipGetLastError();
}

}  // namespace fff

// fff_grouped.hip -- matrix products grouped by expert with ragged sizes
// (fff_grouped_matmul): y_dst(i) = epilogue(x_src(i) W_g) for the entries i of
// every group g.
//
// Only the device knows how many entries a group has, so a launch covers the
// most row tiles there can be and every workgroup finds its tile from the
// offsets (find_tile).  The product runs on the matrix cores
// (fff_grouped.hpp); its 32 x 32 blocks then pass through LDS, so that the
// epilogue works on four consecutive columns a lane and stores whole lines.
#include "fff_grouped.hpp"

namespace fff {

namespace {

enum { ST_OK_ = 0, ST_UNSUPPORTED_ = -2 };

// Epilogue and store of four columns n .. n + 3 of entry i (left: columns in the row from n on).
__device__ __forceinline__ void grouped_store4(const GroupedParams& p, int64_t i, int32_t dst, int n, float* z) {
    const int left = p.n - n;
    if (p.z_in) {
        float d[4];
        unpack4(d, load4<false>(p.z_in, p.z_bf16, i * p.n + n, left), p.z_bf16);
#pragma unroll
        for (int j = 0; j < 4; ++j) z[j] *= activation_grad(d[j], p.act);
    } else {
        if (p.z_out) store4<false>(p.z_out, p.z_bf16, i * p.n + n, left, z);
        if (p.act != ACT_IDENTITY) {
#pragma unroll
            for (int j = 0; j < 4; ++j) z[j] = activation(z[j], p.act);
        }
    }
    if (dst >= 0) store4<false>(p.y, p.y_bf16, int64_t(dst) * p.n + n, left, z);
}

// A workgroup per tile.  BCOL: W is [k, n].
template <class G, bool DMA, bool BCOL>
__global__ __launch_bounds__(G::THREADS, 2 * G::THREADS / 256) void grouped_kernel(GroupedParams p) {
    extern __shared__ __align__(16) unsigned char glds[];
    __shared__ int32_t s_dst[G::BM];   // row of y, or -1
    __shared__ uint8_t s_src[G::BM];   // whether the entry has a row of x
    const Tile t = find_tile<G::THREADS>(p.offsets, p.n_groups, p.n_entries, G::BM, G::BN, (p.n + G::BN - 1) / G::BN,
                                         blockIdx.x);
    if (t.g < 0) return;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    for (int r = tid; r < G::BM; r += G::THREADS) {
        const int64_t i = t.m0 + r;
        s_dst[r] = i < t.m1 ? int32_t(entry_row(p.y_index, 1, p.y_rows, i)) : -1;
    }

    // this lane's sources: A rows through the index (rows behind the tile and absent ones read row 0),
    // B rows of [n, k] or reduction rows of [k, n] (columns behind n read the last ones or zeros)
    const char* x = static_cast<const char*>(p.x);
    const char* w = static_cast<const char*>(p.w) + int64_t(t.g) * p.n * p.k * G::ESZ;
    constexpr int RPL = 1024 / G::ROWB, VPR = G::ROWB / 16;  // rows and vectors per row of a wave load
    const char* pa[G::LA];
    const char* pb[G::LB];
    int va[G::LA], vb[G::LB];  // first reduction element of the lane's vector (BCOL's B: its row)
#pragma unroll
    for (int i = 0; i < G::LA; ++i) {
        const int r = (wave * G::LA + i) * RPL + lane / VPR, v = (lane % VPR) ^ row_key<G::ROWB>(r);
        const int64_t e = t.m0 + r;
        const int64_t src = e < t.m1 ? entry_row(p.x_index, p.x_div, p.x_rows, e) : -1;
        if (lane % VPR == 0) s_src[r] = src >= 0;
        va[i] = v * G::EV;
        pa[i] = x + (src >= 0 ? src : 0) * p.k * G::ESZ + v * 16;
    }
    constexpr int CPL = G::BN * G::ESZ / 16;  // vectors of a column tile's row
#pragma unroll
    for (int i = 0; i < G::LB; ++i) {
        if constexpr (BCOL) {
            const int at = (wave * G::LB + i) * 64 + lane, r = at / CPL, v = (at % CPL) ^ col_key<G::BF, G::BN>(r);
            vb[i] = r;
            pb[i] = w + (int64_t(r) * p.n + t.n0 + v * G::EV) * G::ESZ;
        } else {
            const int r = (wave * G::LB + i) * RPL + lane / VPR, v = (lane % VPR) ^ row_key<G::ROWB>(r);
            const int n = t.n0 + r < p.n ? t.n0 + r : p.n - 1;
            vb[i] = v * G::EV;
            pb[i] = w + int64_t(n) * p.k * G::ESZ + v * 16;
        }
    }
    const int64_t steps = (p.k + G::KS - 1) / G::KS;
    const int64_t bstep = BCOL ? int64_t(G::KS) * p.n * G::ESZ : G::ROWB;
    uint4 ra[DMA ? 1 : G::LA], rb[DMA ? 1 : G::LB];
    const uint32_t lds0 = uint32_t(uintptr_t((__attribute__((address_space(3))) unsigned char*)glds));
    const char* zero = reinterpret_cast<const char*>(&g_zero16);
    auto issue = [&](int64_t s, int stage) {
        const bool part = s == steps - 1 && p.k % G::KS != 0;
        const int k0 = int(s) * G::KS;
        if constexpr (DMA) {
            const uint32_t st = lds0 + uint32_t(stage) * G::STAGE;
#pragma unroll
            for (int i = 0; i < G::LA; ++i)
                lds_dma16(part && k0 + va[i] >= p.k ? zero : pa[i] + s * G::ROWB, st + (wave * G::LA + i) * 1024);
#pragma unroll
            for (int i = 0; i < G::LB; ++i) {
                const char* q = pb[i] + s * bstep;
                if constexpr (BCOL) {
                    const int at = (wave * G::LB + i) * 64 + lane, r = at / CPL;
                    const int n = t.n0 + ((at % CPL) ^ col_key<G::BF, G::BN>(r)) * G::EV;
                    if (n >= p.n || (part && k0 + vb[i] >= p.k)) q = zero;
                } else {
                    if (part && k0 + vb[i] >= p.k) q = zero;
                }
                lds_dma16(q, st + G::BM * G::ROWB + (wave * G::LB + i) * 1024);
            }
        } else {
#pragma unroll
            for (int i = 0; i < G::LA; ++i) ra[i] = load16<G::BF>(pa[i] + s * G::ROWB, int64_t(p.k) - k0 - va[i]);
#pragma unroll
            for (int i = 0; i < G::LB; ++i) {
                int64_t left = int64_t(p.k) - k0 - vb[i];
                if constexpr (BCOL) {
                    const int at = (wave * G::LB + i) * 64 + lane, r = at / CPL;
                    const int n = t.n0 + ((at % CPL) ^ col_key<G::BF, G::BN>(r)) * G::EV;
                    left = left > 0 ? int64_t(p.n) - n : 0;
                }
                rb[i] = load16<G::BF>(pb[i] + s * bstep, left);
            }
        }
    };
    auto commit = [&](int stage) {
        if constexpr (!DMA) {
            unsigned char* st = glds + stage * G::STAGE;
#pragma unroll
            for (int i = 0; i < G::LA; ++i) *reinterpret_cast<uint4*>(st + (wave * G::LA + i) * 1024 + lane * 16) = ra[i];
#pragma unroll
            for (int i = 0; i < G::LB; ++i)
                *reinterpret_cast<uint4*>(st + G::BM * G::ROWB + (wave * G::LB + i) * 1024 + lane * 16) = rb[i];
        }
    };
    tile_v16f acc[G::TM][G::TN];
#pragma unroll
    for (int i = 0; i < G::TM; ++i)
#pragma unroll
        for (int j = 0; j < G::TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    grouped_loop<G, DMA, false, BCOL>(glds, steps, acc, issue, commit);

    // a 32 x 32 result: lane l, register r holds row 8 (r / 4) + 4 (l / 32) + r % 4, column l % 32;
    // blocks pass through the wave's own LDS (rows of 36 floats: the two half-waves, four rows
    // apart, fall on different banks) and come back four columns a lane, eight lanes a row
    constexpr int PITCH = 36;
    static_assert(size_t(G::WAVES) * 32 * PITCH * 4 <= G::LDS, "epilogue blocks fit the stages");
    __syncthreads();
    float* blk = reinterpret_cast<float*>(glds) + wave * 32 * PITCH;
    const int wm = wave / G::WGN, wn = wave % G::WGN;
#pragma unroll
    for (int i = 0; i < G::TM; ++i)
#pragma unroll
        for (int j = 0; j < G::TN; ++j) {
#pragma unroll
            for (int r = 0; r < 16; ++r)
                blk[(8 * (r / 4) + 4 * (lane >> 5) + r % 4) * PITCH + (lane & 31)] = acc[i][j][r];
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            const int n = t.n0 + (wn * G::TN + j) * 32 + (lane & 7) * 4;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int rr = q * 8 + (lane >> 3), m = (wm * G::TM + i) * 32 + rr;
                const float4 v = *reinterpret_cast<const float4*>(blk + rr * PITCH + (lane & 7) * 4);
                float z[4] = {v.x, v.y, v.z, v.w};
                if (!s_src[m]) z[0] = z[1] = z[2] = z[3] = 0.0f;
                if (n < p.n && t.m0 + m < t.m1) grouped_store4(p, t.m0 + m, s_dst[m], n, z);
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
}

template <class G>
hipError_t launch_grouped(const GroupedParams& p, hipStream_t stream, int* status) {
    const int64_t grid = most_tiles(p.n_entries, p.n_groups, G::BM) * ((int64_t(p.n) + G::BN - 1) / G::BN);
    *status = grid > INT32_MAX ? ST_UNSUPPORTED_ : ST_OK_;
    if (*status != ST_OK_) return hipSuccess;
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(unsigned(grid)), dim3(G::THREADS), G::LDS, stream, p); };
    // rows of whole 16-byte vectors go straight to LDS
    const bool dma = p.k % G::EV == 0 && (!p.w_transposed || p.n % G::EV == 0);
    if (p.w_transposed) dma ? launch(grouped_kernel<G, true, true>) : launch(grouped_kernel<G, false, true>);
    else dma ? launch(grouped_kernel<G, true, false>) : launch(grouped_kernel<G, false, false>);
    return hipGetLastError();
}

}  // namespace

hipError_t run_grouped_matmul(const GroupedParams& p, const DeviceInfo&, hipStream_t stream, int* status) {
    const int64_t mean = p.n_entries / p.n_groups;
    if (p.bf16) {
        if (mean >= 128) return launch_grouped<GCfg<true, 4, 2, 2, 2, 3, 64>>(p, stream, status);
        return launch_grouped<GCfg<true, 1, 2, 2, 2, 3, 64>>(p, stream, status);
    }
    if (mean >= 128) return launch_grouped<GCfg<false, 2, 2, 2, 2, 3, 64>>(p, stream, status);
    return launch_grouped<GCfg<false, 1, 2, 2, 2, 3, 64>>(p, stream, status);
}

}  // namespace fff

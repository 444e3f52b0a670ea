// fff_grouped_grad.hip -- weight gradients of the grouped products
// (fff_grouped_weight_grad): dW_g = sum over group g's entries of dy_i^T x_i.
//
// A tile of one group's dW is a product over the group's entries, which both
// operands hold as rows: column tiles of fff_grouped.hpp, read back transposed.
// The entries' rows are looked up some steps ahead, into LDS.  Where there are
// few tiles, a group's entries are cut into pieces (splits) for workgroups of
// their own; their partial sums are added in order.
#include "fff_grouped.hpp"

#include <cstdio>

namespace fff {

namespace {

enum { ST_OK_ = 0, ST_UNSUPPORTED_ = -2 };

using GradBig = GCfg<true, 4, 2, 2, 4, 2, 128>;    // 256 x 256, eight waves
using GradSmall = GCfg<true, 2, 2, 2, 2, 2, 128>;  // 128 x 128, four waves
using GradTiny = GCfg<true, 1, 1, 2, 2, 3, 128>;   // 64 x 64, four waves
using GradSmallF32 = GCfg<false, 2, 2, 2, 2, 2, 128>;
using GradTinyF32 = GCfg<false, 1, 1, 2, 2, 3, 128>;

constexpr size_t GRAD_PART_BYTES = size_t(128) << 20;  // partial sums, at most

struct GradPlan {
    int bm, splits;
    int64_t tiles;
};

// 256 x 256 tiles where rows are whole 16-byte vectors and there are 64 of them; else 128 x 128, unless
// they and their splits leave a fifth of the CUs' 512 places empty in their only or second round, where
// 64 x 64 does better (us, 128 and 64: 5003 fp32 entries, 64 groups of 203 x 300: 39, 30; 8000 x 16 of
// 768 x 768: 169, 140; where 128 fills them, 16384 x 8 of 1024 x 1024: 444, 511; bf16, 65536 x 1 of
// 768 x 768: 172, 276).  64 tiles of 256 x 256 are a coarse bound: what they gain goes by the entries a tile
// sums, too (us, 256 and the smaller: below it 65536 entries in 9 tiles of 768 x 768: 160, 119, in 16 of
// 1024 x 1024: 164, 192; 16384 in 60 of 1280 x 1024: 65, 72; above it 65536 in 64 of 1024 x 1024: 168, 197, in 72 of
// 768 x 768: 109, 213; 16384 in 64: 58, 60, in 128: 62, 54; 8192 in 128: 50, 34; 65536 in 64 of one group each,
// 256 x 256: 37, 31).  Splits: up to two workgroups a CU, eight steps of the mean group each at least,
// within GRAD_PART_BYTES.  By the sizes alone, so the workspace's size and the result's bits are too.
GradPlan grad_plan(int64_t n_entries, int32_t n_groups, int32_t k, int32_t n, bool bf16) {
    auto cdiv = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
    const int64_t step = bf16 ? 64 : 32;
    const int64_t most = int64_t(GRAD_PART_BYTES / (size_t(n_groups) * size_t(n) * size_t(k) * 4 + 1));
    auto plan = [&](int bm) {
        const int64_t tiles = n_groups * cdiv(n, bm) * cdiv(k, bm), slots = bm == 256 ? 256 : 512;
        const int64_t splits = tiles >= slots ? 1 : std::min({slots / tiles, n_entries / n_groups / (8 * step), most});
        return GradPlan{bm, int(std::max<int64_t>(1, splits)), tiles};
    };
    if (bf16 && k > 128 && n > 128 && k % 8 == 0 && n % 8 == 0 && plan(256).tiles >= 64) return plan(256);
    const GradPlan p = plan(128);
    const int64_t groups = p.tiles * p.splits, places = cdiv(groups, 512) * 512;
    return groups < 1024 && 5 * groups < 4 * places ? plan(64) : p;
}

// Tiles that one XCD takes in a row (four at least: 32 groups of 16 tiles took 242 us two at a time, 230 four).
__host__ __device__ __forceinline__ int64_t grad_run(int per, int splits) {
    const int64_t run = int64_t(per) * splits / XCDS;
    return run > 4 ? run : 4;
}

// A workgroup per tile and split.
template <class G, bool DMA>
__global__ __launch_bounds__(G::THREADS, 2) void grouped_grad_kernel(GroupedGradParams p, int tk, int tiles, int splits) {
    constexpr int CH = 8 * G::KS;  // entries whose rows are looked up together
    extern __shared__ __align__(16) unsigned char glds[];
    __shared__ int32_t s_row[2][2][CH];  // [buffer][dy, x]: source rows, -1 where there is none
    // Workgroup h runs on XCD h % 8.  Runs of an eighth of a group's tiles go round the XCDs: neighbours
    // share rows in their L2, and every XCD has a part of every group, large or small (whole groups an
    // XCD: 32 uneven groups of 65536 entries, 4096 x 1024: 750 us, 670 so).
    const int per = tiles / p.n_groups;  // tiles of a group
    const int64_t run = grad_run(per, splits);
    const int64_t at = blockIdx.x / XCDS;
    const int64_t tile = (at / run * XCDS + blockIdx.x % XCDS) * run + at % run;
    if (tile >= int64_t(tiles) * splits) return;
    const int g = int(tile / (int64_t(per) * splits)), in = int(tile - int64_t(g) * per * splits);
    const int sp = in / per, n0 = in % per / tk * G::BM, k0 = in % per % tk * G::BN;
    int64_t lo = 0, hi = 0;
    if (p.n_entries > 0) group_range(p.offsets, p.n_entries, g, &lo, &hi);
    const int64_t all = (hi - lo + G::KS - 1) / G::KS;  // steps of the group, and this split's
    const int64_t s0 = all * sp / splits, steps = all * (sp + 1) / splits - s0;
    lo += s0 * G::KS;
    const int64_t count = std::min<int64_t>(hi - lo, steps * G::KS);  // entries

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t lds0 = uint32_t(uintptr_t((__attribute__((address_space(3))) unsigned char*)glds));
    const char* zero = reinterpret_cast<const char*>(&g_zero16);
    const uint32_t dypitch = uint32_t(p.n) * G::ESZ, xpitch = uint32_t(p.k) * G::ESZ;

    // rows of entries [c CH, (c + 1) CH): read, and some steps later stored
    constexpr int PT = (CH + G::THREADS - 1) / G::THREADS;
    int32_t row_dy[PT], row_x[PT];
    auto look = [&](int64_t c) {
#pragma unroll
        for (int u = 0; u < PT; ++u) {
            const int e = u * G::THREADS + tid;
            const int64_t i = c * CH + e;
            row_dy[u] = row_x[u] = -1;
            if (e < CH && i < count) {
                const int32_t dy = int32_t(entry_row(p.dy_index, 1, p.dy_rows, lo + i));
                const int32_t x = int32_t(entry_row(p.x_index, p.x_div, p.x_rows, lo + i));
                if (dy >= 0 && x >= 0) {  // else neither is read: the other's infinities times zero are NaN
                    row_dy[u] = dy;
                    row_x[u] = x;
                }
            }
        }
    };
    auto note = [&](int64_t c) {
#pragma unroll
        for (int u = 0; u < PT; ++u) {
            const int e = u * G::THREADS + tid;
            if (e >= CH) continue;
            s_row[c & 1][0][e] = row_dy[u];
            s_row[c & 1][1][e] = row_x[u];
        }
    };

    constexpr int CPA = G::BM * G::ESZ / 16, CPB = G::BN * G::ESZ / 16;  // vectors of a reduction row
    auto row_of = [&](int at, int cp) { return (at * 64 + lane) / cp; };
    auto acol = [&](int at) { return ((at * 64 + lane) % CPA ^ col_key<G::BF, G::BM>(row_of(at, CPA))) * G::EV; };
    auto bcol = [&](int at) { return ((at * 64 + lane) % CPB ^ col_key<G::BF, G::BN>(row_of(at, CPB))) * G::EV; };
    uint4 ra[DMA ? 1 : G::LA], rb[DMA ? 1 : G::LB];
    [[maybe_unused]] uint64_t offs = 0;  // four bits a load: elements it was read early by
    [[maybe_unused]] int off;
    [[maybe_unused]] auto early = [&](int l, const uint4&, int by) {
        offs = (l == 0 ? 0 : offs) | uint64_t(by) << (4 * l);
    };
    // a step's rows, read from LDS ahead of its loads; the next chunk's rows: looked up at a chunk's second
    // step, stored at its fifth, used from the eighth on (a barrier between any two steps' loads)
    int32_t da[G::LA], xb[G::LB];
    auto prepare = [&](int64_t s) {
        const int64_t c = s / 8;
        const int e0 = int(s % 8) * G::KS;
#pragma unroll
        for (int i = 0; i < G::LA; ++i) da[i] = s_row[c & 1][0][e0 + row_of(wave * G::LA + i, CPA)];
#pragma unroll
        for (int i = 0; i < G::LB; ++i) xb[i] = s_row[c & 1][1][e0 + row_of(wave * G::LB + i, CPB)];
        if (s % 8 == 1) look(c + 1);
        if (s % 8 == 4) note(c + 1);
    };
    auto issue = [&](int64_t, int stage, int l) {
        const uint32_t st = lds0 + uint32_t(stage) * G::STAGE;
        if (l < G::LA) {
            const int i = l, at = wave * G::LA + i, n = n0 + acol(at);
            const char* q = static_cast<const char*>(p.dy) + uint64_t(uint32_t(da[i])) * dypitch + n * G::ESZ;
            if constexpr (DMA) lds_dma16(da[i] < 0 || n >= p.n ? zero : q, st + at * 1024);
            else early(l, ra[i] = load16<G::BF>(q, da[i] < 0 ? 0 : p.n - n, p.n, off), off);
        } else {
            const int i = l - G::LA, at = wave * G::LB + i, k = k0 + bcol(at);
            const char* q = static_cast<const char*>(p.x) + uint64_t(uint32_t(xb[i])) * xpitch + k * G::ESZ;
            if constexpr (DMA) lds_dma16(xb[i] < 0 || k >= p.k ? zero : q, st + G::BM * G::ROWB + at * 1024);
            else early(l, rb[i] = load16<G::BF>(q, xb[i] < 0 ? 0 : p.k - k, p.k, off), off);
        }
    };
    auto commit = [&](int stage) {
        if constexpr (!DMA) {
            unsigned char* st = glds + stage * G::STAGE;
            if (offs) {
#pragma unroll
                for (int i = 0; i < G::LA; ++i) ra[i] = shift16<G::BF>(ra[i], int(offs >> (4 * i)) & 15);
#pragma unroll
                for (int i = 0; i < G::LB; ++i) rb[i] = shift16<G::BF>(rb[i], int(offs >> (4 * (G::LA + i))) & 15);
            }
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
    if (steps > 0) {
        look(0);
        note(0);
        __syncthreads();
        prepare(0);
#pragma unroll
        for (int l = 0; l < G::LPS; ++l) issue(0, 0, l);
        grouped_loop<G, DMA, true, true>(glds, steps, acc, prepare, issue, commit);
    }
    // a result's columns are consecutive over 32 lanes: whole 128-byte lines without another pass
    const bool add = splits == 1 && p.accumulate;
    if (add && hi == lo) return;
    float* dw = (splits > 1 ? p.part + int64_t(sp) * p.n_groups * p.n * p.k : p.dw) + int64_t(g) * p.n * p.k;
    const int wm = wave / G::WGN, wn = wave % G::WGN;
#pragma unroll
    for (int i = 0; i < G::TM; ++i)
#pragma unroll
        for (int j = 0; j < G::TN; ++j) {
            const int k = k0 + (wn * G::TN + j) * 32 + (lane & 31), n = n0 + (wm * G::TM + i) * 32 + 4 * (lane >> 5);
            if (k >= p.k) continue;
            float* d = dw + int64_t(n) * p.k + k;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int dn = 8 * (r / 4) + r % 4;
                if (n + dn >= p.n) continue;
                float* q = d + int64_t(dn) * p.k;
                *q = add ? *q + acc[i][j][r] : acc[i][j][r];
            }
        }
}

// dW: the splits' partial sums in order.
__global__ __launch_bounds__(256) void grouped_grad_sum_kernel(GroupedGradParams p, int splits, int64_t all) {
    for (int64_t i = (int64_t(blockIdx.x) * 256 + threadIdx.x) * 4; i < all; i += int64_t(gridDim.x) * 1024) {
        if (i + 4 <= all && all % 4 == 0) {
            float4 v = *reinterpret_cast<const float4*>(p.part + i);
            for (int s = 1; s < splits; ++s) {
                const float4 w = *reinterpret_cast<const float4*>(p.part + int64_t(s) * all + i);
                v.x += w.x;
                v.y += w.y;
                v.z += w.z;
                v.w += w.w;
            }
            float4* d = reinterpret_cast<float4*>(p.dw + i);
            if (p.accumulate) {
                const float4 o = *d;
                v = make_float4(o.x + v.x, o.y + v.y, o.z + v.z, o.w + v.w);
            }
            *d = v;
        } else {
            for (int64_t e = i; e < std::min<int64_t>(all, i + 4); ++e) {
                float v = p.part[e];
                for (int s = 1; s < splits; ++s) v += p.part[int64_t(s) * all + e];
                p.dw[e] = p.accumulate ? p.dw[e] + v : v;
            }
        }
    }
}

// A launch holds less than 2^32 threads.
template <class G>
hipError_t launch_grad(const GroupedGradParams& p, const GradPlan& plan, hipStream_t stream, int* status, char* buf,
                       size_t len) {
    const int tk = int((int64_t(p.k) + G::BN - 1) / G::BN);
    const int64_t round = XCDS * grad_run(int(plan.tiles / p.n_groups), plan.splits);
    const int64_t grid = (plan.tiles * plan.splits + round - 1) / round * round;
    *status = grid > UINT32_MAX / G::THREADS ? ST_UNSUPPORTED_ : ST_OK_;
    if (*status != ST_OK_) return hipSuccess;
    const bool dma = p.n % G::EV == 0 && p.k % G::EV == 0;
    const size_t lds = dma ? G::LDS : 2 * G::STAGE;  // two stages of registers' loads
    if (buf) {
        std::snprintf(buf, len, "tiles<%s,%dx%d,%s> splits=%d grid=%lld block=%d lds_bytes=%zu", G::BF ? "bf16" : "f32",
                      G::BM, G::BN, dma ? "direct" : "registers", plan.splits, (long long)grid, G::THREADS, lds);
        return hipSuccess;
    }
    auto launch = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3(unsigned(grid)), dim3(G::THREADS), lds, stream, p, tk, int(plan.tiles), plan.splits);
    };
    if (dma) launch(grouped_grad_kernel<G, true>);
    else if constexpr (G::BM < 256) launch(grouped_grad_kernel<G, false>);
    if (plan.splits > 1) {
        const int64_t all = int64_t(p.n_groups) * p.n * p.k;
        const unsigned blocks = unsigned(std::min<int64_t>((all + 1023) / 1024, 2048));
        hipLaunchKernelGGL(grouped_grad_sum_kernel, dim3(blocks), dim3(256), 0, stream, p, plan.splits, all);
    }
    return hipGetLastError();
}

}  // namespace

size_t grouped_grad_workspace_bytes(int64_t n_entries, int32_t n_groups, int32_t k, int32_t n) {
    // either type's plan: the caller's call names the sizes alone
    const size_t one = size_t(n_groups) * size_t(n) * size_t(k) * sizeof(float);
    size_t most = 0;
    for (bool bf16 : {false, true}) {
        const int s = grad_plan(n_entries, n_groups, k, n, bf16).splits;
        most = std::max(most, s > 1 ? s * one : 0);
    }
    return most;
}

hipError_t run_grouped_weight_grad(const GroupedGradParams& p, hipStream_t stream, int* status, char* buf, size_t len) {
    const GradPlan plan = grad_plan(p.n_entries, p.n_groups, p.k, p.n, p.bf16);
    if (plan.bm == 256) return launch_grad<GradBig>(p, plan, stream, status, buf, len);
    if (plan.bm == 128)
        return p.bf16 ? launch_grad<GradSmall>(p, plan, stream, status, buf, len)
                      : launch_grad<GradSmallF32>(p, plan, stream, status, buf, len);
    return p.bf16 ? launch_grad<GradTiny>(p, plan, stream, status, buf, len)
                  : launch_grad<GradTinyF32>(p, plan, stream, status, buf, len);
}

}  // namespace fff

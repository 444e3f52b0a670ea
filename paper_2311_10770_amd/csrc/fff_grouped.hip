// fff_grouped.hip -- matrix products grouped by expert with ragged sizes
// (fff_grouped_matmul): y_dst(i) = epilogue(x_src(i) W_g) for the entries i of
// every group g.
//
// Only the device knows how many entries a group has, so a launch covers the
// most row tiles there can be and every workgroup finds its tile from the
// offsets (TileMap).  The product runs on the matrix cores
// (fff_grouped.hpp); its 32 x 32 blocks then pass through LDS, so that the
// epilogue works on eight consecutive columns a lane and stores whole lines.
#include "fff_grouped.hpp"

#include <cmath>
#include <cstdio>
#include <type_traits>

namespace fff {

namespace {

enum { ST_OK_ = 0, ST_UNSUPPORTED_ = -2 };

// What becomes of z (grouped_rows).
enum { EPI_STORE = 0, EPI_GELU = 1, EPI_TANH = 2, EPI_GELU_GRAD = 3, EPI_TANH_GRAD = 4 };

// Eight consecutive values of a row; `left` of them in it where not FULL.
template <bool FULL>
__device__ __forceinline__ void put8(char* row, int bf, int col, int left, const float* v) {
    if (bf) {
        if (FULL || left >= 8) {
            typedef uint32_t u4_a2 __attribute__((ext_vector_type(4), aligned(2)));
            *reinterpret_cast<u4_a2*>(row + col * 2) = u4_a2{pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]),
                                                             pack2(v[6], v[7])};
            return;
        }
    } else if (FULL || left >= 8) {
        typedef float f4_a4 __attribute__((ext_vector_type(4), aligned(4)));
        reinterpret_cast<f4_a4*>(row + col * 4)[0] = f4_a4{v[0], v[1], v[2], v[3]};
        reinterpret_cast<f4_a4*>(row + col * 4)[1] = f4_a4{v[4], v[5], v[6], v[7]};
        return;
    }
    if constexpr (!FULL) {
        store4<false>(row, bf, col, left, v);
        store4<false>(row, bf, col + 4, left - 4, v + 4);
    }
}

// Epilogue and store of sixteen rows of a tile from row m0 on, COLS columns from n0 on, out of the
// wave's LDS: eight columns a lane.  FULL: all these columns are in the matrix.  The instructions of
// this loop are what the epilogue costs: offsets are one 32 x 32 + 64 bit product, and rows without
// a row of x are looked for in tiles that have some (bad).  FINE: y is fp32.
template <int KIND, bool FINE, bool FULL, int COLS, int PITCH>
__device__ __forceinline__ void grouped_rows(const GroupedParams& p, const float* blk, int m0, int rows, int64_t e0, int n0,
                                             const int32_t* s_dst, const uint8_t* s_src, bool bad) {
    constexpr int LPR = COLS / 8, RPI = 64 / LPR, U = 16 / RPI;
    const int lane = threadIdx.x & 63, c = lane % LPR * 8, n = n0 + c, left = p.n - n;
    if (!FULL && left <= 0) return;
    const uint32_t ypitch = uint32_t(p.n) << (p.y_bf16 ? 1 : 2), zpitch = uint32_t(p.n) << (p.z_bf16 ? 1 : 2);
    const uint32_t ze = uint32_t(e0);  // entries are below 2^31
    Raw4 d[U][2];
    if constexpr (KIND >= EPI_GELU_GRAD) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int m = m0 + u * RPI + lane / LPR;
            if (m >= rows) continue;
            const char* row = static_cast<const char*>(p.z_in) + uint64_t(ze + m) * zpitch;
            d[u][0] = load4<FULL>(row, p.z_bf16, n, left);
            d[u][1] = load4<FULL>(row, p.z_bf16, n + 4, left - 4);
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int rr = u * RPI + lane / LPR, m = m0 + rr;
        const float4 a = *reinterpret_cast<const float4*>(blk + rr * PITCH + c);
        const float4 b = *reinterpret_cast<const float4*>(blk + rr * PITCH + c + 4);
        float z[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        const int32_t dst = s_dst[m];
        if (bad && !s_src[m]) {
#pragma unroll
            for (int j = 0; j < 8; ++j) z[j] = 0.0f;
        }
        if (m >= rows) continue;
        if constexpr (KIND >= EPI_GELU_GRAD) {
            float g[8];
            unpack4(g, d[u][0], p.z_bf16);
            unpack4(g + 4, d[u][1], p.z_bf16);
#pragma unroll
            for (int j = 0; j < 8; ++j) z[j] *= act_slope<KIND == EPI_GELU_GRAD ? ACT_GELU_ERF : ACT_GELU_TANH, FINE>(g[j]);
        } else {
            if (p.z_out) put8<FULL>(static_cast<char*>(p.z_out) + uint64_t(ze + m) * zpitch, p.z_bf16, n, left, z);
            constexpr int ACT = KIND == EPI_GELU ? ACT_GELU_ERF : KIND == EPI_TANH ? ACT_GELU_TANH : ACT_IDENTITY;
#pragma unroll
            for (int j = 0; j < 8; ++j) z[j] = act_value<ACT, FINE>(z[j]);
        }
        if (dst >= 0) put8<FULL>(static_cast<char*>(p.y) + uint64_t(uint32_t(dst)) * ypitch, p.y_bf16, n, left, z);
    }
}
template <int COLS, int PITCH, bool FULL, bool FINE>
__device__ __forceinline__ void grouped_epilogue(int kind, const GroupedParams& p, const float* blk, int m0, int rows,
                                                 int64_t e0, int n0, const int32_t* dst, const uint8_t* src, bool bad) {
    switch (kind) {
        case EPI_GELU: return grouped_rows<EPI_GELU, FINE, FULL, COLS, PITCH>(p, blk, m0, rows, e0, n0, dst, src, bad);
        case EPI_TANH: return grouped_rows<EPI_TANH, FINE, FULL, COLS, PITCH>(p, blk, m0, rows, e0, n0, dst, src, bad);
        case EPI_GELU_GRAD:
            return grouped_rows<EPI_GELU_GRAD, FINE, FULL, COLS, PITCH>(p, blk, m0, rows, e0, n0, dst, src, bad);
        case EPI_TANH_GRAD:
            return grouped_rows<EPI_TANH_GRAD, FINE, FULL, COLS, PITCH>(p, blk, m0, rows, e0, n0, dst, src, bad);
        default: return grouped_rows<EPI_STORE, false, FULL, COLS, PITCH>(p, blk, m0, rows, e0, n0, dst, src, bad);
    }
}

// Workgroups take tiles gridDim.x apart.  BCOL: W is [k, n].  The next tile is looked up while this one
// is multiplied, and its first step is on its way to LDS (DMA) while this one's results are stored.  Y: the
// type of y, bf16 (1) or fp32 (0), where the tile has a kernel for each, else -1: with either's activations beside
// the other's in one kernel the 256 x 256 tiles' registers spilled further (65536 x 32, 1024 -> 4096 with
// GELU 815 -> 823 us).
template <class G, bool DMA, bool BCOL, int Y = -1>
__global__ __launch_bounds__(G::THREADS, 2) void grouped_kernel(GroupedParams p) {
    extern __shared__ __align__(16) unsigned char glds[];
    __shared__ int32_t s_dst[2][G::BM];   // row of y, or -1
    __shared__ uint8_t s_src[2][G::BM];   // whether the entry has a row of x
    __shared__ Tile s_tile[2];
    __shared__ int64_t s_sum[G::WAVES];
    __shared__ int s_bad[2];
    TileMap<G::THREADS> map{p.offsets, p.n_entries, p.n_groups, G::BM, G::BN, (p.n + G::BN - 1) / G::BN};
    map.init(s_sum);
    int64_t h = blockIdx.x;
    map.find(h, &s_tile[0]);
    if (threadIdx.x == 0) s_bad[0] = 0;
    __syncthreads();

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const char* x = static_cast<const char*>(p.x);
    constexpr int RPL = 1024 / G::ROWB, VPR = G::ROWB / 16;  // rows and vectors per row of a wave load
    constexpr int CPL = G::BN * G::ESZ / 16;                 // vectors of a column tile's row
    const int64_t steps = (p.k + G::KS - 1) / G::KS;
    const int64_t bstep = BCOL ? int64_t(G::KS) * p.n * G::ESZ : G::ROWB;
    const uint32_t lds0 = uint32_t(uintptr_t((__attribute__((address_space(3))) unsigned char*)glds));
    const char* zero = reinterpret_cast<const char*>(&g_zero16);

    // this lane's sources: A rows through the index (rows behind the tile and absent ones read row 0),
    // B rows of [n, k] (rows behind n read the last one) or reduction rows of [k, n]
    const char* pa[G::LA];
    const char* pb[G::LB];
    int n0 = 0;
    // reduction element of a row vector's first element; row and column of a column tile's vector
    auto row_at = [&](int i) { return (lane % VPR ^ row_key<G::ROWB>(i * RPL + lane / VPR)) * G::EV; };
    auto col_row = [&](int i) { return (i * 64 + lane) / CPL; };
    auto col_at = [&](int i) {
        const int at = i * 64 + lane;
        return (at % CPL ^ col_key<G::BF, G::BN>(at / CPL)) * G::EV;
    };
    uint4 ra[DMA ? 1 : G::LA], rb[DMA ? 1 : G::LB];
    [[maybe_unused]] uint64_t offs = 0;  // four bits a load: elements it was read early by
    [[maybe_unused]] int off;
    [[maybe_unused]] auto note = [&](int l, const uint4&, int early) {
        offs = (l == 0 ? 0 : offs) | uint64_t(early) << (4 * l);
    };
    auto issue = [&](int64_t s, int stage, int l) {
        const bool part = s == steps - 1 && p.k % G::KS != 0;
        const int k0 = int(s) * G::KS;
        const uint32_t st = lds0 + uint32_t(stage) * G::STAGE;
        if (l < G::LA) {
            const int i = l, at = wave * G::LA + i;
            if constexpr (DMA) lds_dma16(part && k0 + row_at(at) >= p.k ? zero : pa[i] + s * G::ROWB, st + at * 1024);
            else note(l, ra[i] = load16<G::BF>(pa[i] + s * G::ROWB, int64_t(p.k) - k0 - row_at(at), p.k, off), off);
        } else {
            const int i = l - G::LA, at = wave * G::LB + i;
            const char* q = pb[i] + s * bstep;
            if constexpr (DMA) {
                if constexpr (BCOL) {
                    if (n0 + col_at(at) >= p.n || (part && k0 + col_row(at) >= p.k)) q = zero;
                } else {
                    if (part && k0 + row_at(at) >= p.k) q = zero;
                }
                lds_dma16(q, st + G::BM * G::ROWB + at * 1024);
            } else {
                int64_t left = int64_t(p.k) - k0 - (BCOL ? col_row(at) : row_at(at));
                if constexpr (BCOL) left = left > 0 ? int64_t(p.n) - n0 - col_at(at) : 0;
                note(l, rb[i] = load16<G::BF>(q, left, BCOL ? p.n : p.k, off), off);
            }
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
    // a tile's sources, its rows' records in buffer `buf`, and the loads of its first step
    auto begin = [&](const Tile& t, int buf) {
        n0 = t.n0;
        const char* w = static_cast<const char*>(p.w) + int64_t(t.g) * p.n * p.k * G::ESZ;
#pragma unroll
        for (int i = 0; i < G::LA; ++i) {
            const int r = (wave * G::LA + i) * RPL + lane / VPR;
            const int64_t e = t.m0 + r;
            const int64_t src = e < t.m1 ? entry_row(p.x_index, p.x_div, p.x_rows, e) : -1;
            if (lane % VPR == 0) s_src[buf][r] = src >= 0;
            if (e < t.m1 && src < 0) s_bad[buf] = 1;
            pa[i] = x + ((src >= 0 ? src : 0) * p.k + row_at(wave * G::LA + i)) * G::ESZ;
        }
#pragma unroll
        for (int i = 0; i < G::LB; ++i) {
            const int at = wave * G::LB + i;
            if constexpr (BCOL) {
                pb[i] = w + (int64_t(col_row(at)) * p.n + n0 + col_at(at)) * G::ESZ;
            } else {
                const int r = n0 + at * RPL + lane / VPR, n = r < p.n ? r : p.n - 1;
                pb[i] = w + (int64_t(n) * p.k + row_at(at)) * G::ESZ;
            }
        }
#pragma unroll
        for (int l = 0; l < G::LPS; ++l) issue(0, 0, l);
        for (int r = tid; r < G::BM; r += G::THREADS) {
            const int64_t i = t.m0 + r;
            s_dst[buf][r] = i < t.m1 ? int32_t(entry_row(p.y_index, 1, p.y_rows, i)) : -1;
        }
    };

    // Epilogue: a 32 x 32 result holds row 8 (r / 4) + 4 (l / 32) + r % 4, column l % 32 in lane l,
    // register r.  Half a row of blocks at a time (sixteen rows) passes through the wave's own LDS, behind
    // the first stage, where the next tile's first step arrives (row pitch 8 floats past the blocks: the
    // two half-waves, four rows apart, fall on different banks), and comes back eight columns a lane.  Its
    // code stands once, in a rolled loop: unrolled over the blocks it was 45000 instructions, which
    // every workgroup fetched anew (65536 entries, 1024 -> 4096, then a workgroup per tile: 888 against 762 us).
    constexpr int COLS = 32 * G::TN, PITCH = COLS + 8;
    static_assert(size_t(G::WAVES) * 16 * PITCH * 4 <= G::STAGE, "half rows of blocks fit behind the first stage");
    float* blk = reinterpret_cast<float*>(glds + G::STAGE) + wave * 16 * PITCH;
    const int wm = wave / G::WGN, wn = wave % G::WGN;
    const int kind = p.act == ACT_IDENTITY ? EPI_STORE : (p.z_in ? EPI_GELU_GRAD : EPI_GELU) + (p.act == ACT_GELU_TANH);

    Tile t = s_tile[0];
    if (t.g < 0) return;
    begin(t, 0);
    for (int turn = 0;; turn ^= 1) {
        h += gridDim.x;
        map.find(h, &s_tile[turn ^ 1]);  // seen behind the loop's barriers
        if (threadIdx.x == 0) s_bad[turn ^ 1] = 0;
        tile_v16f acc[G::TM][G::TN];
#pragma unroll
        for (int i = 0; i < G::TM; ++i)
#pragma unroll
            for (int j = 0; j < G::TN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
        grouped_loop<G, DMA, false, BCOL>(glds, steps, acc, [](int64_t) {}, issue, commit);
        __syncthreads();  // every wave is done with the stages
        const Tile next = s_tile[turn ^ 1];
        if (DMA && next.g >= 0) begin(next, turn ^ 1);
        const int rows = int(t.m1 - t.m0 < G::BM ? t.m1 - t.m0 : G::BM), c0 = t.n0 + wn * COLS;
        const bool full = c0 + COLS <= p.n, bad = s_bad[turn];
#pragma unroll 1
        for (int i = 0; i < 2 * G::TM; ++i) {
#pragma unroll
            for (int u = 0; u < 2 * G::TM; ++u) {
                if (i != u) continue;
#pragma unroll
                for (int j = 0; j < G::TN; ++j)
#pragma unroll
                    for (int r = 0; r < 8; ++r)
                        blk[(8 * (r / 4) + 4 * (lane >> 5) + r % 4) * PITCH + j * 32 + (lane & 31)] =
                            acc[u / 2][j][u % 2 * 8 + r];
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            const int m0 = wm * G::TM * 32 + i * 16;
            auto rows_out = [&](auto fine) {
                if (full) grouped_epilogue<COLS, PITCH, true, fine.value>(kind, p, blk, m0, rows, t.m0, c0, s_dst[turn], s_src[turn], bad);
                else grouped_epilogue<COLS, PITCH, false, fine.value>(kind, p, blk, m0, rows, t.m0, c0, s_dst[turn], s_src[turn], bad);
            };
            if constexpr (Y >= 0) rows_out(std::bool_constant<Y == 0>{});
            else if (p.y_bf16) rows_out(std::false_type{});
            else rows_out(std::true_type{});
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
        if (next.g < 0) return;
        t = next;
        __syncthreads();  // the blocks' LDS is free, the next tile's records are written
        if constexpr (!DMA) begin(t, turn ^ 1);
    }
}

// Whether the operands' rows are whole 16-byte vectors.
bool whole_vectors(const GroupedParams& p) {
    const int ev = p.bf16 ? 8 : 4;
    return p.k % ev == 0 && (!p.w_transposed || p.n % ev == 0);
}

template <class G>
hipError_t launch_grouped(const GroupedParams& p, int cus, hipStream_t stream, int* status, char* buf, size_t len) {
    const int64_t tiles = most_tiles(p.n_entries, p.n_groups, G::BM) * ((int64_t(p.n) + G::BN - 1) / G::BN);
    *status = tiles > INT32_MAX ? ST_UNSUPPORTED_ : ST_OK_;
    if (*status != ST_OK_) return hipSuccess;
    // rows of whole 16-byte vectors go straight to LDS; two stages of those loaded through registers
    const bool dma = whole_vectors(p);
    const int grid = int(std::min<int64_t>(tiles, int64_t(cus) * (dma ? G::PER_CU : 8 / G::WAVES)));
    const size_t lds = dma ? G::LDS : 2 * G::STAGE;
    if (buf) {
        std::snprintf(buf, len, "tiles<%s,%dx%d,%s,%s> grid=%d block=%d lds_bytes=%zu", p.bf16 ? "bf16" : "f32", G::BM,
                      G::BN, dma ? "direct" : "registers", p.w_transposed ? "w_kn" : "w_nk", grid, G::THREADS, lds);
        return hipSuccess;
    }
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(unsigned(grid)), dim3(G::THREADS), lds, stream, p); };
    if constexpr (G::BM == 256) {  // not built through registers
        if (p.w_transposed) p.y_bf16 ? launch(grouped_kernel<G, true, true, 1>) : launch(grouped_kernel<G, true, true, 0>);
        else p.y_bf16 ? launch(grouped_kernel<G, true, false, 1>) : launch(grouped_kernel<G, true, false, 0>);
    } else if (dma) {
        p.w_transposed ? launch(grouped_kernel<G, true, true>) : launch(grouped_kernel<G, true, false>);
    } else {
        p.w_transposed ? launch(grouped_kernel<G, false, true>) : launch(grouped_kernel<G, false, false>);
    }
    return hipGetLastError();
}

// Few entries a group (decoding): the weights of the groups in use are read once, and that is the time.
// A workgroup takes sixteen columns of a group's matrix and up to sixteen of its entries; its waves
// split the reduction axis, whole 128-byte lines of a row at a time, with FEW_U steps (2 FEW_U KB a wave)
// in flight.  Weights are the MFMA's first operand (sixteen rows of W), the entries its second, straight
// from global memory in the operands' layout (lane l: row l % 16, the 16 bytes l / 16 of every 64); the
// waves' sums meet in LDS.
constexpr int FEW_WAVES = 8, FEW_U = 4;
constexpr int64_t FEW_ENTRIES = int64_t(1) << 28;  // below: 64 groups' tiles are counted in 32 bits

// Row tile mt (of sixteen entries) over all groups, found by every wave for itself, 64 groups at a time.
__device__ __forceinline__ Tile few_tile(const GroupedParams& p, int mt) {
    const int lane = threadIdx.x & 63;
    int64_t at = 0;
    for (int64_t g0 = 0; g0 < p.n_groups; g0 += 64) {
        int64_t lo = 0, hi = 0;
        if (g0 + lane < p.n_groups) group_range(p.offsets, p.n_entries, int(g0) + lane, &lo, &hi);
        const int mine = int((hi - lo + 15) / 16);
        int run = mine;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int v = __shfl_up(run, d);
            if (lane >= d) run += v;
        }
        const uint64_t has = __ballot(at + run > mt);
        if (has) {
            const int l = __builtin_ctzll(has);
            const int64_t before = at + __builtin_amdgcn_readlane(run - mine, l);
            const int first = __builtin_amdgcn_readlane(int(lo), l), end = __builtin_amdgcn_readlane(int(hi), l);
            return Tile{int(g0) + l, 0, first + (mt - before) * 16, end};
        }
        at += __builtin_amdgcn_readlane(run, 63);
    }
    return Tile{-1, 0, 0, 0};
}

template <bool BF, bool ALIGNED>
__global__ __launch_bounds__(64 * FEW_WAVES) void grouped_few_kernel(GroupedParams p) {
    constexpr int ESZ = BF ? 2 : 4, EV = 16 / ESZ, STEP = 128 / ESZ;  // elements of a step
    __shared__ float s_sum[FEW_WAVES][256];
    const int tn = (p.n + 15) / 16;
    const Tile t = few_tile(p, int(blockIdx.x / tn));
    if (t.g < 0) return;
    const int n0 = int(blockIdx.x % tn) * 16, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int r16 = lane & 15, q = lane >> 4;
    const int64_t e = t.m0 + r16;
    const int64_t src = e < t.m1 ? entry_row(p.x_index, p.x_div, p.x_rows, e) : -1;
    const int n = n0 + r16 < p.n ? n0 + r16 : p.n - 1;
    const char* w = static_cast<const char*>(p.w) + (int64_t(t.g) * p.n + n) * p.k * ESZ;
    const char* x = static_cast<const char*>(p.x) + (src >= 0 ? src : 0) * p.k * ESZ;
    auto load = [&](const char* row, int64_t k, bool in) {  // sixteen bytes from element k on
        const int64_t left = in ? int64_t(p.k) - k : 0;
        if constexpr (ALIGNED) return left > 0 ? *reinterpret_cast<const uint4*>(row + k * ESZ) : make_uint4(0, 0, 0, 0);
        else {
            int off;
            const uint4 v = load16<BF>(row + k * ESZ, left, p.k, off);
            return off ? shift16<BF>(v, off) : v;
        }
    };
    tile_v4f acc = {0.0f, 0.0f, 0.0f, 0.0f};
    const int steps = (p.k + STEP - 1) / STEP;
    for (int s = wave; s < steps; s += FEW_WAVES * FEW_U) {
        uint4 fw[FEW_U][2], fx[FEW_U][2];
#pragma unroll
        for (int u = 0; u < FEW_U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t k = int64_t(s + u * FEW_WAVES) * STEP + (h * 4 + q) * EV;
                fw[u][h] = load(w, k, true);
                fx[u][h] = load(x, k, src >= 0);
            }
#pragma unroll
        for (int u = 0; u < FEW_U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if constexpr (BF) {
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, fw[u][h]),
                                                                  __builtin_bit_cast(bf16x8_t, fx[u][h]), acc, 0, 0, 0);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        acc = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(word(fw[u][h], j)),
                                                                   __uint_as_float(word(fx[u][h], j)), acc, 0, 0, 0);
                }
            }
    }
    // lane l, register r: column (entry) l % 16, row (of W) 4 (l / 16) + r
#pragma unroll
    for (int r = 0; r < 4; ++r) s_sum[wave][r16 * 16 + 4 * q + r] = acc[r];
    __syncthreads();
    if (tid >= 256) return;
    float z = 0.0f;
#pragma unroll
    for (int v = 0; v < FEW_WAVES; ++v) z += s_sum[v][tid];
    const int64_t i = t.m0 + tid / 16;
    const int c = n0 + tid % 16;
    if (i >= t.m1 || c >= p.n) return;
    if (entry_row(p.x_index, p.x_div, p.x_rows, i) < 0) z = 0.0f;  // (zeros times infinite weights are NaN)
    if (p.z_in) {
        const float d = load_elem(p.z_in, p.z_bf16, i * p.n + c);
        z *= p.act == ACT_GELU_ERF    ? act_slope<ACT_GELU_ERF, true>(d)
             : p.act == ACT_GELU_TANH ? act_slope<ACT_GELU_TANH, true>(d)
                                      : 1.0f;
    } else {
        if (p.z_out) store_elem(p.z_out, p.z_bf16, i * p.n + c, z);
        z = p.act == ACT_GELU_ERF    ? act_value<ACT_GELU_ERF, true>(z)
            : p.act == ACT_GELU_TANH ? act_value<ACT_GELU_TANH, true>(z)
                                     : z;
    }
    const int64_t dst = entry_row(p.y_index, 1, p.y_rows, i);
    if (dst >= 0) store_elem(p.y, p.y_bf16, dst * p.n + c, z);
}

// Workgroups of the few-entries kernel, and whether a launch holds their threads.
int64_t few_tiles(const GroupedParams& p) { return most_tiles(p.n_entries, p.n_groups, 16) * ((int64_t(p.n) + 15) / 16); }
bool few_fits(const GroupedParams& p) {
    return p.n_entries < FEW_ENTRIES && few_tiles(p) <= UINT32_MAX / (64 * FEW_WAVES);
}

hipError_t launch_few(const GroupedParams& p, hipStream_t stream, char* buf, size_t len) {
    const int64_t tiles = few_tiles(p);
    if (buf) {
        std::snprintf(buf, len, "few<%s,%s> grid=%lld block=%d", p.bf16 ? "bf16" : "f32",
                      whole_vectors(p) ? "aligned" : "unaligned", (long long)tiles, 64 * FEW_WAVES);
        return hipSuccess;
    }
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(unsigned(tiles)), dim3(64 * FEW_WAVES), 0, stream, p); };
    if (p.bf16) whole_vectors(p) ? launch(grouped_few_kernel<true, true>) : launch(grouped_few_kernel<true, false>);
    else whole_vectors(p) ? launch(grouped_few_kernel<false, true>) : launch(grouped_few_kernel<false, false>);
    return hipGetLastError();
}

// Which kernel: the one of the least time by what each took (us, measured with 1 to 64 groups, 64 to 16384
// entries, k and n 128 to 4096): a tile costs `start` and `alone` a 128-byte step of the reduction axis,
// or `pair` where two workgroups share its CU.  Small tiles lose rate (32 x 128: 0.4 of 256 x 256's, whose
// two workgroups' worth of tile has a CU to itself) and win where large ones leave CUs idle or rows of
// the tile empty; sixteen-entry tiles read the weights again for every sixteen entries of a group; 64 x 64 are
// for fp32, whose matrix cores are the bound, where columns of wider tiles are empty.  Some
// of both sides, bf16 (few, 32, 64, 128, 256 rows): 64 entries x 1 group, 4096 -> 1024: 11, 27, 33, 39, 99;
// 1000 x 16 groups, 768 -> 768: 26, 10, 12, 15, 28; 4000 x 64, 1024 -> 1024: 139, 44, 30, 39, 40;
// 9025 x 23, 3224 -> 448 transposed: -, 82, 71, 63, -; fp32 (32, 64, 64 x 64): 8757 x 1, 640 -> 64 transposed: 33, 32,
// 21; 1334 x 18, 2816 -> 448 transposed: 79, 121, 73; 9001 x 16, 768 -> 1000: 144, 142, 158.
struct TileCost {
    int bm, bn;
    double start, alone, pair;
};
constexpr TileCost COST_BF16[] = {{32, 128, 2, 0.34, 0.52}, {64, 128, 2.5, 0.43, 0.58}, {128, 128, 4, 0.50, 0.95},
                                  {256, 256, 6, 1.85, 3.70}};
constexpr TileCost COST_F32[] = {{32, 128, 2, 0.80, 1.25}, {64, 128, 2.5, 1.18, 2.20}, {128, 128, 4, 2.00, 3.60},
                                 {64, 64, 2, 0.77, 1.22}};

// 0: few entries a group; 1 ..: the tiles of the tables.
int grouped_variant(const GroupedParams& p, int cus) {
    const double E = double(p.n_entries), used = double(std::min<int64_t>(p.n_groups, p.n_entries));
    const int esz = p.bf16 ? 2 : 4;
    const double steps = (double(p.k) * esz + 127) / 128;
    auto row_tiles = [&](int bm) { return std::max(used, E / bm + 0.5 * used); };
    int best = 0;
    double least = 1e300;
    if (!p.w_transposed && few_fits(p)) {
        // 768 workgroups at once; rows off 16-byte addresses take 2.4 times as long
        const double rounds = row_tiles(16) * ((p.n + 15) / 16) / (3.0 * cus);
        const double kb = double(p.k) * esz / 64, slow = p.k % (16 / esz) ? 2.4 : 1.0;
        least = rounds < 1 ? 2.5 + 0.115 * kb * std::max(rounds, 0.35) * slow : rounds * (2.5 + 0.115 * kb) * slow;
    }
    const TileCost* cost = p.bf16 ? COST_BF16 : COST_F32;
    // (256 x 256 tiles are not built through registers: they spill, and took as long as 128 x 128: 65536
    // entries, 1023 -> 4095, 1042 and 1046 us)
    for (int v = 0; v < (!p.bf16 || whole_vectors(p) ? 4 : 3); ++v) {
        // (the half tile a group is an estimate: a tenth of a round does not make one)
        const double per_cu =
            std::max(1.0, std::ceil(row_tiles(cost[v].bm) * ((p.n + cost[v].bn - 1) / cost[v].bn) / cus - 0.1));
        const double pairs = std::floor(per_cu / 2), odd = per_cu - 2 * pairs;
        const double t = pairs * (cost[v].start * (cost[v].bm == 256 ? 2 : 1) + steps * cost[v].pair) +
                         odd * (cost[v].start + steps * cost[v].alone);
        if (t < least) {
            least = t;
            best = v + 1;
        }
    }
    return best;
}

}  // namespace

hipError_t run_grouped_matmul(const GroupedParams& p, const DeviceInfo& dev, hipStream_t stream, int* status, char* buf,
                              size_t len) {
    const int cus = dev.cu_count > 0 ? dev.cu_count : 256;
    switch (grouped_variant(p, cus)) {
        case 0: *status = ST_OK_; return launch_few(p, stream, buf, len);
        case 1: return p.bf16 ? launch_grouped<GCfg<true, 1, 1, 1, 4, 3, 128>>(p, cus, stream, status, buf, len)
                              : launch_grouped<GCfg<false, 1, 1, 1, 4, 3, 128>>(p, cus, stream, status, buf, len);
        case 2: return p.bf16 ? launch_grouped<GCfg<true, 1, 2, 2, 2, 3, 128>>(p, cus, stream, status, buf, len)
                              : launch_grouped<GCfg<false, 1, 2, 2, 2, 3, 128>>(p, cus, stream, status, buf, len);
        case 3: return p.bf16 ? launch_grouped<GCfg<true, 2, 2, 2, 2, 2, 128>>(p, cus, stream, status, buf, len)
                              : launch_grouped<GCfg<false, 2, 2, 2, 2, 2, 128>>(p, cus, stream, status, buf, len);
        default: return p.bf16 ? launch_grouped<GCfg<true, 4, 2, 2, 4, 2, 128>>(p, cus, stream, status, buf, len)
                               : launch_grouped<GCfg<false, 1, 1, 2, 2, 3, 128>>(p, cus, stream, status, buf, len);
    }
}

}  // namespace fff

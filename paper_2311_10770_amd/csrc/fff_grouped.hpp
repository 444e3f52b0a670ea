// fff_grouped.hpp -- what the grouped products' kernels share: the tile lookup
// over ragged groups, operand tiles in LDS and the matrix-core loop.
//
// Every product is C[BM, BN] += A[BM, red] B[BN, red]^T over a reduction axis,
// one step of ROWB bytes of it per row at a time.  An operand whose rows run
// along the reduction axis ("row" tiles: x, and W as [n, k]) lies in LDS as BM
// or BN rows of ROWB bytes; one whose rows run across it ("column" tiles: W as
// [k, n], and both operands of a weight gradient) as steps of reduction rows,
// read back transposed.  Tiles are staged 16 bytes a lane, straight from
// global memory (global_load_lds, S - 1 steps ahead) where rows are 16-byte
// aligned, else through registers, which takes rows at any element.
#pragma once

#include "fff_device.hpp"
#include "fff_gemm.hpp"
#include "fff_operators.hpp"
#include "fff_rows.hpp"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

namespace fff {

// Entries [lo, hi) of group g: within [0, n_entries], empty where the offsets fall.
__device__ __forceinline__ void group_range(const int32_t* offsets, int64_t n_entries, int g, int64_t* lo, int64_t* hi) {
    const int64_t a = offsets[g], b = offsets[g + 1];
    *lo = a < 0 ? 0 : a > n_entries ? n_entries : a;
    *hi = b < *lo ? *lo : b > n_entries ? n_entries : b;
}

struct Tile {
    int g;           // group, or -1: no tile of this number
    int n0;          // first column
    int64_t m0, m1;  // its entries
};

// The row tiles of bm entries of all groups (groups in order, each group's last one partly filled)
// times tn column tiles of bn.  Every thread keeps the sum over a few consecutive groups and all
// before them; the thread whose groups hold a tile finds it (find) for the workgroup.  Number h runs
// on XCD h % 8: each XCD takes a contiguous range of the tiles, MB row tiles deep before the next
// column tile, so that neighbours share rows and columns in their L2: about a square of its 32 CUs'
// tiles (65536 entries, 1024 -> 4096, 4, 6, 8 and 16 deep: 648, 647, 651, 668 us; 16384 x 1, 4096 -> 4096: 500, 485,
// 490, 496; 16384 x 8, 1024 -> 4096 -> 1024: 6 deep 349, 8 deep 375).  A thread's groups are walked one by one,
// at the start and for its tiles: little to some thousand groups (64 -> 64 bf16, 8 entries each: 1024 groups 11 us,
// 4096: 45, of 9 for the bytes), the time of 32768 (1142 us, of 69).
template <int THREADS>
struct TileMap {
    static constexpr int MB = 6;
    const int32_t* offsets;
    int64_t n_entries;
    int n_groups, bm, bn, tn;
    int64_t before, mine;  // row tiles before this thread's groups, and in them
    int total;             // of all groups (offsets that name entries twice can make more than a launch holds: those
                           // past 2^31 / tn are left out)

    // wave_sum: LDS of THREADS / 64 words.  Every thread of the workgroup calls this (a barrier).
    __device__ __forceinline__ void init(int64_t* wave_sum) {
        const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
        int64_t lo, hi;
        mine = 0;
        for (int g = first(tid); g < first(tid + 1); ++g) {
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
        __syncthreads();
        before = run - mine;
        int64_t all = 0;
        for (int w = 0; w < THREADS / 64; ++w) {
            if (w < wave) before += wave_sum[w];
            all += wave_sum[w];
        }
        total = int(std::min<int64_t>(all, INT32_MAX / tn));
    }
    __device__ __forceinline__ int first(int tid) const {
        const int64_t per = (int64_t(n_groups) + THREADS - 1) / THREADS;
        return int(std::min<int64_t>(n_groups, tid * per));
    }
    // Writes tile h to *out: the owner thread alone, or thread 0 where there is no such tile.
    __device__ __forceinline__ void find(int64_t number, Tile* out) const {
        // 32-bit arithmetic: the host launches at most 2^31 - 1 tiles
        const uint32_t all = uint32_t(total) * uint32_t(tn);
        if (number >= int64_t(all)) {
            if (threadIdx.x == 0) out->g = -1;
            return;
        }
        const uint32_t h = uint32_t(number), x = h % XCDS, rem = all % XCDS;
        const uint32_t t = x * (all / XCDS) + (x < rem ? x : rem) + h / XCDS;
        const uint32_t wide = uint32_t(MB) * uint32_t(tn);
        const int block = int(t / wide), in = int(t % wide);
        const int deep = std::min(MB, total - block * MB), mt = block * MB + in % deep;
        int64_t at = before;
        if (mt < at || mt >= at + mine) return;
        for (int g = first(threadIdx.x);; ++g) {
            int64_t lo, hi;
            group_range(offsets, n_entries, g, &lo, &hi);
            const int64_t tiles = (hi - lo + bm - 1) / bm;
            if (mt < at + tiles) {
                *out = Tile{g, in / deep * bn, lo + (mt - at) * bm, hi};
                return;
            }
            at += tiles;
        }
    }
};

// Most row tiles of bm entries that n_entries in n_groups groups can make.
inline int64_t most_tiles(int64_t n_entries, int32_t n_groups, int bm) {
    return n_entries / bm + std::min<int64_t>(n_groups, n_entries);
}

// Row that entry i reads or writes, or -1 where there is none.
__device__ __forceinline__ int64_t entry_row(const int32_t* index, int div, int64_t rows, int64_t i) {
    const int64_t v = index ? index[i] : i;
    if (v < 0) return -1;
    const int64_t r = div == 1 ? v : uint32_t(v) / uint32_t(div);
    return r < rows ? r : -1;
}

// Phi(-a) for a = |z|, Phi the standard normal distribution, and e = exp(-a^2 / 2): e t Q(t) with
// t = 1 / (1 + 0.3 a), Q the polynomial of degree 7 nearest to Phi(-a) / (e t) over a = 0 .. 14 in relative
// error (1.5e-7, fitted for this kernel; 15 roundings of fp32 to a = 4, 130 at 13, where e carries
// that of its argument).  Twenty instructions; erfcf's are several times as many, and at 268 M values
// they took as long as the product.
__device__ __forceinline__ float normal_tail(float z, float& e) {
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3f, __builtin_fabsf(z), 1.0f));
    e = __builtin_amdgcn_exp2f(z * z * -0.72134752044448170368f);
    float q = 0.03567512333393097f;
    q = __builtin_fmaf(q, t, -0.15720446407794952f);
    q = __builtin_fmaf(q, t, 0.2063557654619217f);
    q = __builtin_fmaf(q, t, -0.05368557944893837f);
    q = __builtin_fmaf(q, t, 0.1285625696182251f);
    q = __builtin_fmaf(q, t, 0.09991323202848434f);
    q = __builtin_fmaf(q, t, 0.12075399607419968f);
    q = __builtin_fmaf(q, t, 0.11962929368019104f);
    return e * t * q;
}

// Phi(z) where its result is stored in fp32 (FINE below): within |z| < 1, where the tail's roundings are largest
// beside the result, 0.5 + z R(z^2), R the polynomial of degree 5 nearest to (Phi(z) - 0.5) / z there
// (7e-10 relative, fitted for this kernel).  For z ~ N(0, 1) the root mean square errors in units of 2^-24,
// by the tail alone, by this and by the layer's own erfcf (fff_device.hpp): GELU 0.475, 0.381, 0.375; its
// derivative 0.826, 0.454, 0.465.  Time (us) in the same order: 9001 x 16 fp32, 768 -> 1000 with the
// derivative 153.7, 156.3, 162.7; 65536 x 32, bf16 1024 -> 4096 to fp32 with GELU 778, 809, 948.  Results
// stored in bf16 lose 16 bits more than either, and take the tail alone.
__device__ __forceinline__ float normal_cdf(float z, float& e) {
    const float s = z * z, p = normal_tail(z, e);
    float q = -7.654209184693173e-06f;
    q = __builtin_fmaf(q, s, 0.00011348637781338766f);
    q = __builtin_fmaf(q, s, -0.0011863299878314137f);
    q = __builtin_fmaf(q, s, 0.009973322972655296f);
    q = __builtin_fmaf(q, s, -0.06649035960435867f);
    q = __builtin_fmaf(q, s, 0.3989422917366028f);
    return s < 1.0f ? __builtin_fmaf(z, q, 0.5f) : z > 0.0f ? 1.0f - p : p;
}

// The activations and their derivatives (fff_device.hpp has their formulas).  FINE: to be stored in fp32.
template <int ACT, bool FINE>
__device__ __forceinline__ float act_value(float z) {
    if constexpr (ACT == ACT_GELU_ERF) {
        float e;
        if constexpr (FINE) return z * normal_cdf(z, e);
        const float p = normal_tail(z, e);
        return z * (z > 0.0f ? 1.0f - p : p);
    } else if constexpr (ACT == ACT_GELU_TANH) {
        const float d = 1.0f + __builtin_amdgcn_exp2f(-2.88539008177792681472f * gelu_tanh_u(z));
        const float t = __builtin_amdgcn_rcpf(d), q = z * t;
        // the quotient's own remainder once more, as a true division leaves it (0.516 -> 0.465 of the units above);
        // where d overflows, t and q are 0 and stay so, and over 1 there is none (nor a NaN of infinities)
        if constexpr (FINE) {
            const float left = __builtin_fmaf(-__builtin_fminf(d, 3.4028234663852886e38f), q, z);
            return d > 1.0f ? __builtin_fmaf(left, t, q) : q;
        }
        return q;
    } else {
        return z;
    }
}
template <int ACT, bool FINE>
__device__ __forceinline__ float act_slope(float z) {
    if constexpr (ACT == ACT_GELU_ERF) {
        float e;
        if constexpr (FINE) {
            const float c = normal_cdf(z, e);
            return __builtin_fmaf(z * 0.39894228040143267794f, e, c);
        }
        const float p = normal_tail(z, e);
        return __builtin_fmaf(z * 0.39894228040143267794f, e, z > 0.0f ? 1.0f - p : p);
    } else if constexpr (ACT == ACT_GELU_TANH) {
        const float u = 2.88539008177792681472f * gelu_tanh_u(z);
        const float up = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-u));
        const float down = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(u));
        // far out up * down is 0, and so are its products with a finite z and a square kept from overflow
        const float du = __builtin_fminf(__builtin_fmaf(0.134145f * z, z, 1.0f), 1e38f);
        return __builtin_fmaf(z * up * down, 1.59576912160573071176f * du, up);
    } else {
        return 1.0f;
    }
}

// Sixteen zero bytes: what a lane stages for places outside its matrix.
static __device__ const uint4 g_zero16 = {0, 0, 0, 0};

// Sixteen bytes of a row, `left` of its elements from p on in it (none where left <= 0: zeros); rows of
// `len` elements at any element.  A vector that ends past the row is read so that it ends with the row,
// `off` elements early, for shift16 to put right when the load has arrived.  (Element by element, as rows
// shorter than a vector still are, edge tiles took several times as long as whole ones.)
template <bool BF>
__device__ __forceinline__ uint4 load16(const char* p, int64_t left, int len, int& off) {
    constexpr int EV = BF ? 8 : 4, ESZ = 16 / EV;
    typedef uint32_t u4_a2 __attribute__((ext_vector_type(4), aligned(2)));
    off = 0;
    if (left <= 0) return make_uint4(0, 0, 0, 0);
    if (len >= EV) {
        off = left >= EV ? 0 : EV - int(left);
        const u4_a2 v = *reinterpret_cast<const u4_a2*>(p - off * ESZ);
        return make_uint4(v.x, v.y, v.z, v.w);
    }
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < EV - 1; ++j) {
        if (j >= left) continue;
        if constexpr (BF) w[j >> 1] |= uint32_t(reinterpret_cast<const uint16_t*>(p)[j]) << (16 * (j & 1));
        else w[j] = reinterpret_cast<const uint32_t*>(p)[j];
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// The vector without its first `off` elements, zeros behind (off < 8 bf16 or 4 fp32 elements).
template <bool BF>
__device__ __forceinline__ uint4 shift16(const uint4& r, int off) {
    const int bits = off * (BF ? 16 : 32);
    const uint64_t lo = uint64_t(r.y) << 32 | r.x, hi = uint64_t(r.w) << 32 | r.z;
    const uint64_t l = bits == 0 ? lo : bits >= 64 ? hi >> (bits - 64) : lo >> bits | hi << (64 - bits);
    const uint64_t h = bits >= 64 ? 0 : hi >> bits;
    return make_uint4(uint32_t(l), uint32_t(l >> 32), uint32_t(h), uint32_t(h >> 32));
}

// Order of the 16-byte vectors in LDS: vector v of row r at v ^ key, so that the lanes of a fragment
// read fall on different banks.
// Row tiles: the lanes of a b128 read are served eight consecutive rows at a time.
template <int ROWB>
__device__ __forceinline__ int row_key(int r) {
    static_assert(ROWB == 64 || ROWB == 128, "four or eight vectors a row");
    return ROWB == 128 ? swz32(r & 15) : (r >> 1) & 3;
}
// Column tiles of C columns, bf16: a transposing read takes four rows and four adjacent vectors, or
// eight rows (0..3, 8..11) and two; fp32: 32 columns of rows r and r + 4.
template <bool BF, int C>
__device__ __forceinline__ int col_key(int r) {
    if constexpr (!BF) return ((r >> 2) & 1) * 8;
    else if constexpr (C >= 128) return (r & 3) * 4 ^ ((r >> 3) & 1) * 2;
    else return ((r >> 1) & 1) * 4 ^ ((r >> 3) & 1) * 2;
}

// Fragments of reduction slice kk (32 bytes' worth: 16 bf16 or 8 fp32) of a 32-row MFMA operand, as the
// sixteen bytes lane l holds: row l % 32, elements 8 (l / 32) on (fp32: 4 (l / 32) on).
template <int ROWB>
__device__ __forceinline__ uint4 row_frag(const unsigned char* tile, int row0, int kk, int lane) {
    const int r = row0 + (lane & 31);
    return *reinterpret_cast<const uint4*>(tile + r * ROWB + (((2 * kk + (lane >> 5)) ^ row_key<ROWB>(r)) * 16));
}
template <bool BF, int C>
__device__ __forceinline__ uint4 col_frag(const unsigned char* tile, int col0, int kk, int lane) {
    if constexpr (BF) {
        // A transposing read hands lane i of sixteen column i of the 4 x 16 block their addresses cover
        // (lane i: row i / 4, columns 4 (i % 4) .. +3); two of them give eight reduction rows.
        typedef short s4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s4* lds_s4;
        const int grp = lane >> 4, i = lane & 15;
        uint2 u[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = 16 * kk + 8 * (grp >> 1) + 4 * h + (i >> 2);
            const int c = col0 / 8 + 2 * (grp & 1) + ((i & 3) >> 1);
            u[h] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                                 (lds_s4)(tile + r * (C * 2) + ((c ^ col_key<true, C>(r)) * 16) + (i & 1) * 8)));
        }
        return make_uint4(u[0].x, u[0].y, u[1].x, u[1].y);
    } else {
        uint32_t w[4];
        const int c = col0 + (lane & 31);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int r = 8 * kk + 4 * (lane >> 5) + t;
            w[t] = *reinterpret_cast<const uint32_t*>(tile + r * (C * 4) + (((c >> 2) ^ col_key<false, C>(r)) * 16) + (c & 3) * 4);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
}

// c += a b over one slice: one 32 x 32 x 16 MFMA in bf16; in fp32 four 32 x 32 x 2, the t-th on
// element t of both operands' vectors (a permutation of the slice's reduction indices).
template <bool BF>
__device__ __forceinline__ void mfma_slice(tile_v16f& c, const uint4& a, const uint4& b) {
    if constexpr (BF) {
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c,
                                                    0, 0, 0);
    } else {
#pragma unroll
        for (int t = 0; t < 4; ++t)
            c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(word(a, t)), __uint_as_float(word(b, t)), c, 0, 0, 0);
    }
}

// Shape of a workgroup's tile: WGM x WGN waves of TM x TN 32 x 32 blocks, S stages of ROWB bytes a row.
template <bool BF_, int TM_, int TN_, int WGM_, int WGN_, int S_, int ROWB_>
struct GCfg {
    static constexpr bool BF = BF_;
    static constexpr int TM = TM_, TN = TN_, WGM = WGM_, WGN = WGN_, S = S_, ROWB = ROWB_;
    static constexpr int BM = 32 * TM * WGM, BN = 32 * TN * WGN;
    static constexpr int WAVES = WGM * WGN, THREADS = 64 * WAVES;
    static constexpr int ESZ = BF ? 2 : 4, EV = 16 / ESZ;
    static constexpr int KS = ROWB / ESZ;      // reduction elements a step
    static constexpr int SLICES = ROWB / 32;
    static constexpr int LA = BM * ROWB / 1024 / WAVES, LB = BN * ROWB / 1024 / WAVES;  // wave loads a step
    static constexpr int LPS = LA + LB;
    static constexpr int STAGE = (BM + BN) * ROWB;
    static constexpr size_t LDS = size_t(S) * STAGE;
    // workgroups a CU holds: 160 KB of LDS (4 KB for the kernels' own arrays), two waves a SIMD
    static constexpr int PER_CU = int(std::min<size_t>((160 * 1024) / (LDS + 4096), 8 / WAVES));
    static_assert(BM * ROWB % (1024 * WAVES) == 0 && BN * ROWB % (1024 * WAVES) == 0, "whole wave loads");
    static_assert(LPS * (S - 1) <= 63, "vmcnt holds 6 bits");
    static_assert(SLICES % 2 == 0, "slice 0 of every step reads the same registers");
};

// The matrix-core loop over `steps` steps.  issue(step, stage, l) starts load l of LPS of a step into its
// stage (DMA) or reads it into registers, which commit(stage) stores; prepare(step) does what the loads
// of a step need earlier.  The caller has prepared and issued step 0.  ACOL, BCOL:
// column tiles.
//
// The fragments of slice kk + 1 are read while slice kk's MFMAs run, across steps too: the barrier that
// ends a step stands before its last slice's MFMAs, when all its fragments are in registers, so the next
// step's first reads, and the loads into the stage just read, run under those MFMAs (with the
// barrier between the steps the matrix cores waited for a whole LDS read each step).  Those loads start at
// once behind the barrier, which is soonest, or (SPREAD: two column tiles, whose reads take twice the
// instructions) between the MFMAs.  At once and spread, us, 65536 entries in 32 groups: weight gradients
// 4096 x 1024: 705, 670; 1024 -> 4096 with GELU 828, 825; its data gradient 695, 713; fp32, 16384 entries
// x 8, 1024 -> 1024: 334, 345.
template <class G, bool DMA, bool ACOL, bool BCOL, class Prepare, class Issue, class Commit>
__device__ __forceinline__ void grouped_loop(unsigned char* lds, int64_t steps, tile_v16f (&acc)[G::TM][G::TN],
                                             Prepare prepare, Issue issue, Commit commit) {
    constexpr int S = DMA ? G::S : 2;
    constexpr bool SPREAD = DMA && ACOL;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / G::WGN, wn = wave % G::WGN;
    uint4 fa[2][G::TM], fb[2][G::TN];
    auto read = [&](const unsigned char* st, int kk) {
#pragma unroll
        for (int j = 0; j < G::TN; ++j) {
            const int c0 = (wn * G::TN + j) * 32;
            if constexpr (BCOL) fb[kk & 1][j] = col_frag<G::BF, G::BN>(st + G::BM * G::ROWB, c0, kk, lane);
            else fb[kk & 1][j] = row_frag<G::ROWB>(st + G::BM * G::ROWB, c0, kk, lane);
        }
#pragma unroll
        for (int i = 0; i < G::TM; ++i) {
            const int r0 = (wm * G::TM + i) * 32;
            if constexpr (ACOL) fa[kk & 1][i] = col_frag<G::BF, G::BM>(st, r0, kk, lane);
            else fa[kk & 1][i] = row_frag<G::ROWB>(st, r0, kk, lane);
        }
    };
    auto issue_all = [&](int64_t s, int stage) {
#pragma unroll
        for (int l = 0; l < G::LPS; ++l) issue(s, stage, l);
    };
    if constexpr (DMA) {
#pragma unroll
        for (int s = 1; s < S; ++s)
            if (s < steps) {
                prepare(s);
                issue_all(s, s);
            }
        wait_steps<S - 1, G::LPS>(int(steps - 1 < S - 1 ? steps - 1 : S - 1));
    } else {
        commit(0);
        if (steps > 1) {
            prepare(1);
            issue_all(1, 0);
        }
    }
    __syncthreads();  // step 0 is in LDS
    read(lds, 0);
    int stage = 0;
    for (int64_t s = 0; s < steps; ++s) {
        const unsigned char* st = lds + stage * G::STAGE;
        const int follow = stage + 1 == S ? 0 : stage + 1;
        const int64_t load = s + S;  // the step whose loads this one starts
        if (load < steps) prepare(load);
#pragma unroll
        for (int kk = 0; kk < G::SLICES; ++kk) {
            if (kk + 1 < G::SLICES) {
                read(st, kk + 1);
            } else if (s + 1 < steps) {
                if constexpr (DMA) {
                    const int64_t left = steps - 2 - s;
                    wait_steps<S - 2, G::LPS>(int(left < S - 2 ? left : S - 2));
                } else {
                    commit(follow);
                }
                __syncthreads();  // step s + 1 is in LDS; every wave has read all of step s
                if (!SPREAD && load < steps) issue_all(load, stage);
                read(lds + follow * G::STAGE, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < G::TM; ++i) {
                if (SPREAD && kk + 1 == G::SLICES && load < steps) {
#pragma unroll
                    for (int l = i * G::LPS / G::TM; l < (i + 1) * G::LPS / G::TM; ++l) issue(load, stage, l);
                }
#pragma unroll
                for (int j = 0; j < G::TN; ++j) mfma_slice<G::BF>(acc[i][j], fa[kk & 1][i], fb[kk & 1][j]);
                if (SPREAD && kk + 1 == G::SLICES) __builtin_amdgcn_sched_barrier(0);
            }
        }
        stage = follow;
    }
}

}  // namespace fff

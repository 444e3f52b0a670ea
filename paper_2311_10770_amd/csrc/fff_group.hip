// fff_group.hip -- fff_group_rows: a stable counting sort of entries by group.
//
// Every wave owns a run of consecutive entries and a row of counters in LDS.
// It counts its entries per group; the counts become running sums over the
// waves (and over the workgroups, through the workspace) and over the groups;
// then the wave goes through its entries again, 64 at a time, and places
// them.  Within 64 entries equal groups are found with one ballot per bit of
// the group number, so no place depends on the order of atomics.
//
// Up to GROUP_ONE entries take one workgroup and one launch; more take three
// (count, scan, place), every workgroup with a chunk of its own.  The work is a
// few bytes per entry: launches and the latency of dependent steps are the time.
// 16384 entries of 64 groups: 12.3 us in one launch, called or in a graph (15.0 with the entries read again
// for placing; three launches took 11.4 in a graph, but 19.1 called).  524288 entries of 4096 groups: 23.4
// us; 100000 of 32768: 52.6, a row of counters there being all that LDS holds, one wave places.
#include "fff_operators.hpp"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

namespace fff {

namespace {

constexpr int GROUP_ONE = 16384;         // entries of the one-launch form, at most
constexpr int GROUP_ONE_GROUPS = 1024;   // its groups: their counters and the staged order fit LDS
constexpr int GROUP_COUNTERS = 32768;    // counters in LDS: waves x groups
constexpr int64_t GROUP_CHUNKS = 256;    // about so many chunks, of at least GROUP_ROUNDS rounds a wave
constexpr int GROUP_ROUNDS = 4;

// Waves of a workgroup: as many as have counters, up to sixteen.
int group_waves(int32_t n_groups) {
    int w = 16;
    while (w > 1 && w * n_groups > GROUP_COUNTERS) w /= 2;
    return w;
}
bool group_one(int64_t n, int32_t n_groups) { return n <= GROUP_ONE && n_groups <= GROUP_ONE_GROUPS; }
// Entries of a chunk: whole rounds of 64 for each of its waves.
int64_t group_chunk(int64_t n, int waves) {
    const int64_t round = 64 * waves, c = (n + GROUP_CHUNKS - 1) / GROUP_CHUNKS;
    return std::max<int64_t>(GROUP_ROUNDS, (c + round - 1) / round) * round;
}
int64_t group_chunks(int64_t n, int32_t n_groups) {
    const int64_t c = group_chunk(n, group_waves(n_groups));
    return std::max<int64_t>(1, (n + c - 1) / c);
}

// The group of entry e, or -1.
__device__ __forceinline__ int group_of(const GroupParams& p, uint32_t e) {
    const int64_t id = int64_t(p.ids[e]) - p.first;
    const int tree = p.n_trees == 1 ? 0 : int(e % uint32_t(p.n_trees));
    return id >= 0 && id < p.n_ids ? tree * p.n_ids + int(id) : -1;
}

// Groups of RB rounds of 64 entries from b + lane on: -1 for an entry without one, -2 behind e1.
template <int RB>
__device__ __forceinline__ void load_groups(const GroupParams& p, int64_t b, int64_t e1, int* g) {
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        const int64_t e = b + 64 * r + (threadIdx.x & 63);
        g[r] = e < e1 ? group_of(p, uint32_t(e)) : -2;
    }
}

// RB rounds counted into the wave's row of counters; returns how many have no group.
template <int RB>
__device__ __forceinline__ int count_groups(const int* g, int32_t* row) {
    int lost = 0;
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        if (g[r] >= 0) atomicAdd(&row[g[r]], 1);
        lost += g[r] == -1;
    }
    return lost;
}

// RB rounds from entry b on placed in order; row[g]: the wave's next place in group g.  Entries go to
// order, or (STAGE) as 16 bits to `staged` in LDS.
template <int RB, bool STAGE>
__device__ __forceinline__ void place_groups(const int* g, int64_t b, int32_t* row, int32_t* order, uint16_t* staged,
                                             int bits) {
    const int lane = threadIdx.x & 63;
    // the lanes of each round with this lane's group; the rounds' chains of ballots run side by side
    uint32_t lo[RB], hi[RB];
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        const uint64_t any = __ballot(g[r] >= 0);
        lo[r] = uint32_t(any);
        hi[r] = uint32_t(any >> 32);
    }
    for (int k = 0; k < bits; ++k) {
#pragma unroll
        for (int r = 0; r < RB; ++r) {
            const int32_t one = __builtin_amdgcn_sbfe(g[r], k, 1);  // bit k in every bit
            const uint64_t set = __ballot(one != 0);
            lo[r] &= ~(uint32_t(set) ^ uint32_t(one));
            hi[r] &= ~(uint32_t(set >> 32) ^ uint32_t(one));
        }
    }
#pragma unroll
    for (int r = 0; r < RB; ++r) {
        if (g[r] >= 0) {
            const uint64_t same = uint64_t(hi[r]) << 32 | lo[r];
            const int before = __popcll(same & ((uint64_t(1) << lane) - 1));
            const int32_t at = row[g[r]];
            // every lane has read its group's counter before the group's first lane moves it on
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (before == 0) row[g[r]] = at + __popcll(same);
            if constexpr (STAGE) staged[at + before] = uint16_t(b + 64 * r + lane);
            else order[at + before] = int32_t(b + 64 * r + lane);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    }
}

// One wave's entries [e0, e1) counted, RB rounds loaded at a time.
template <int RB>
__device__ __forceinline__ void count_run(const GroupParams& p, int64_t e0, int64_t e1, int32_t* row, bool tell) {
    int lost = 0;
    for (int64_t b = e0; b < e1; b += 64 * RB) {
        int g[RB];
        load_groups<RB>(p, b, e1, g);
        lost += count_groups<RB>(g, row);
    }
    if (tell && p.bad && lost) atomicAdd(p.bad, lost);
}

// Counters of group g in W rows of n_groups: exclusive sums from `at` on; returns their end.
template <int W>
__device__ __forceinline__ int32_t rows_scan(int32_t* cnt, int n_groups, int g, int32_t at) {
    int32_t c[W];
#pragma unroll
    for (int w = 0; w < W; ++w) c[w] = cnt[w * n_groups + g];
#pragma unroll
    for (int w = 0; w < W; ++w) {
        cnt[w * n_groups + g] = at;
        at += c[w];
    }
    return at;
}

// Inclusive sums over the 64 lanes.
__device__ __forceinline__ int32_t wave_scan(int32_t v) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int32_t u = __shfl_up(v, d);
        if (lane >= d) v += u;
    }
    return v;
}

// Exclusive sums over a workgroup of `waves` waves.
__device__ __forceinline__ int32_t block_scan(int32_t v, int32_t* sums, int waves) {
    const int32_t in = wave_scan(v);
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 63) sums[wave] = in;
    __syncthreads();
    int32_t before = 0;
    for (int w = 0; w < wave; ++w) before += sums[w];
    return before + in - v;
}

// Everything in one workgroup of sixteen waves.  The order is put together in LDS and stored in whole
// lines.
__global__ __launch_bounds__(1024) void group_one_kernel(GroupParams p, int bits) {
    extern __shared__ int32_t g_cnt[];  // [16][n_groups], then the order as 16-bit entries
    __shared__ int32_t sums[16], listed;
    const int G = p.n_groups, tid = threadIdx.x, wave = tid >> 6;
    uint16_t* staged = reinterpret_cast<uint16_t*>(g_cnt + 16 * G);
    constexpr int ROUNDS = GROUP_ONE / 1024;
    const int64_t run = (p.n_entries + 1023) / 1024 * 64;  // at most ROUNDS rounds: a wave's groups stay in registers
    const int64_t e0 = std::min<int64_t>(p.n_entries, wave * run), e1 = std::min<int64_t>(p.n_entries, e0 + run);
    int mine_of[ROUNDS];
    load_groups<ROUNDS>(p, e0, e1, mine_of);
    for (int i = tid; i < 16 * G; i += 1024) g_cnt[i] = 0;
    __syncthreads();
    const int lost = count_groups<ROUNDS>(mine_of, g_cnt + wave * G);
    if (p.bad && lost) atomicAdd(p.bad, lost);
    __syncthreads();
    // a thread takes a few consecutive groups: their totals, then every wave's first place in them
    const int per = (G + 1023) / 1024, g0 = std::min(G, tid * per), g1 = std::min(G, g0 + per);
    int32_t mine = 0;
    for (int g = g0; g < g1; ++g) {
#pragma unroll
        for (int w = 0; w < 16; ++w) mine += g_cnt[w * G + g];
    }
    int32_t at = block_scan(mine, sums, 16);
    for (int g = g0; g < g1; ++g) {
        p.offsets[g] = at;
        at = rows_scan<16>(g_cnt, G, g, at);
        if (g == G - 1) p.offsets[G] = listed = at;
    }
    __syncthreads();
    place_groups<ROUNDS, true>(mine_of, e0, g_cnt + wave * G, nullptr, staged, bits);
    __syncthreads();
    for (int i = tid; i < listed; i += 1024) p.order[i] = staged[i];
}

// A chunk's entries per group: hist [chunk][group].
__global__ __launch_bounds__(1024) void group_count_kernel(GroupParams p, int64_t chunk, int32_t* hist) {
    extern __shared__ int32_t g_cnt[];  // [n_groups]
    const int G = p.n_groups, tid = threadIdx.x, waves = blockDim.x >> 6, wave = tid >> 6;
    for (int g = tid; g < G; g += blockDim.x) g_cnt[g] = 0;
    __syncthreads();
    const int64_t c0 = int64_t(blockIdx.x) * chunk, run = chunk / waves;
    const int64_t e0 = std::min<int64_t>(p.n_entries, c0 + wave * run), e1 = std::min<int64_t>(p.n_entries, e0 + run);
    count_run<GROUP_ROUNDS>(p, e0, e1, g_cnt, true);
    __syncthreads();
    for (int g = tid; g < G; g += blockDim.x) hist[int64_t(blockIdx.x) * G + g] = g_cnt[g];
}

// Running sums of hist over the chunks, 32 groups a workgroup, a piece of the chunks for each of 32
// threads; the groups' totals behind it.
__global__ __launch_bounds__(1024) void group_scan_kernel(GroupParams p, int chunks, int32_t* hist, int32_t* totals) {
    __shared__ int32_t piece[32][33];
    const int G = p.n_groups, col = threadIdx.x % 32, part = threadIdx.x / 32;
    const int g = blockIdx.x * 32 + col, per = (chunks + 31) / 32;
    const int c0 = std::min(chunks, part * per), c1 = std::min(chunks, c0 + per);
    int32_t sum = 0;
    if (g < G) {
#pragma unroll 8
        for (int c = c0; c < c1; ++c) sum += hist[int64_t(c) * G + g];
    }
    piece[part][col] = sum;
    __syncthreads();
    int32_t run = 0, all = 0;
#pragma unroll
    for (int q = 0; q < 32; ++q) {
        run += q < part ? piece[q][col] : 0;
        all += piece[q][col];
    }
    if (g >= G) return;
    for (int cb = c0; cb < c1; cb += 8) {
        int32_t v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = cb + j < c1 ? hist[int64_t(cb + j) * G + g] : 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (cb + j < c1) hist[int64_t(cb + j) * G + g] = run;
            run += v[j];
        }
    }
    if (part == 0) totals[g] = all;
}

// A chunk's entries to their places: W of the sixteen waves have entries and counters, all of them
// sum the totals to the groups' offsets (every workgroup for itself: a launch for it took 4 us, and as
// the last act of the scan's last workgroup to finish 50, for the device-scope release that it needs of
// every workgroup writes back its XCD's L2).
template <int W>
__global__ __launch_bounds__(1024) void group_place_kernel(GroupParams p, int64_t chunk,
                                                           const int32_t* __restrict__ hist,
                                                           const int32_t* __restrict__ totals, int bits) {
    extern __shared__ int32_t g_cnt[];  // [W][n_groups]
    __shared__ int32_t sums[16];
    const int G = p.n_groups, tid = threadIdx.x, wave = tid >> 6;
    const int64_t c0 = int64_t(blockIdx.x) * chunk, run = chunk / W;
    const int64_t e0 = std::min<int64_t>(p.n_entries, c0 + wave * run);
    const int64_t e1 = wave < W ? std::min<int64_t>(p.n_entries, e0 + run) : e0;
    constexpr int64_t BATCH = 64 * GROUP_ROUNDS;
    int first[GROUP_ROUNDS];  // the first batch's groups stay in registers (up to 2^19 entries, all there are)
    load_groups<GROUP_ROUNDS>(p, e0, e1, first);
    for (int i = tid; i < W * G; i += 1024) g_cnt[i] = 0;
    // a wave takes consecutive groups, 64 at a time (a thread with consecutive groups met its neighbours' LDS
    // banks: 32768 groups 145 us)
    const int lane = tid & 63, part = (G + 1023) / 1024 * 64, g0 = std::min(G, wave * part), g1 = std::min(G, g0 + part);
    int32_t mine = 0;
#pragma unroll 4
    for (int g = g0 + lane; g < g1; g += 64) mine += totals[g];
    block_scan(mine, sums, 16);  // (a barrier: the counters are clear)
    int32_t at = 0;
    for (int w = 0; w < wave; ++w) at += sums[w];
    count_groups<GROUP_ROUNDS>(first, g_cnt + wave * G);
    if (e0 + BATCH < e1) count_run<GROUP_ROUNDS>(p, e0 + BATCH, e1, g_cnt + wave * G, false);
    __syncthreads();
    hist += int64_t(blockIdx.x) * G;
    for (int g = g0 + lane; g - lane < g1; g += 64) {
        const int32_t all = g < g1 ? totals[g] : 0, before = g < g1 ? hist[g] : 0, end = at + wave_scan(all);
        if (g < g1) {
            if (blockIdx.x == 0) p.offsets[g] = end - all;
            rows_scan<W>(g_cnt, G, g, end - all + before);
            if (blockIdx.x == 0 && g == G - 1) p.offsets[G] = end;
        }
        at = __builtin_amdgcn_readlane(end, 63);
    }
    __syncthreads();
    place_groups<GROUP_ROUNDS, false>(first, e0, g_cnt + wave * G, p.order, nullptr, bits);
    for (int64_t b = e0 + BATCH; b < e1; b += BATCH) {
        int g[GROUP_ROUNDS];
        load_groups<GROUP_ROUNDS>(p, b, e1, g);
        place_groups<GROUP_ROUNDS, false>(g, b, g_cnt + wave * G, p.order, nullptr, bits);
    }
}

template <int W>
void launch_place(int waves, const GroupParams& p, int chunks, int64_t chunk, const int32_t* hist, const int32_t* totals,
                  int bits, hipStream_t stream) {
    if constexpr (W > 1) {
        if (waves < W) return launch_place<W / 2>(waves, p, chunks, chunk, hist, totals, bits, stream);
    }
    hipLaunchKernelGGL(group_place_kernel<W>, dim3(chunks), dim3(1024), size_t(W) * p.n_groups * sizeof(int32_t),
                       stream, p, chunk, hist, totals, bits);
}

}  // namespace

size_t group_workspace_bytes(int64_t n_entries, int32_t n_groups) {
    if (group_one(n_entries, n_groups)) return 0;
    return (size_t(group_chunks(n_entries, n_groups)) + 1) * size_t(n_groups) * sizeof(int32_t);
}

hipError_t run_group_rows(const GroupParams& p, hipStream_t stream) {
    const int G = p.n_groups, waves = group_waves(G);
    int bits = 0;
    while ((1 << bits) < G) ++bits;
    if (group_one(p.n_entries, G)) {
        hipLaunchKernelGGL(group_one_kernel, dim3(1), dim3(1024),
                           16 * size_t(G) * sizeof(int32_t) + size_t(p.n_entries) * sizeof(uint16_t), stream, p, bits);
        return hipGetLastError();
    }
    const int64_t chunk = group_chunk(p.n_entries, waves);
    const int chunks = int(group_chunks(p.n_entries, G));
    int32_t* hist = static_cast<int32_t*>(p.workspace);  // [chunks][n_groups], then the totals
    int32_t* totals = hist + size_t(chunks) * G;
    hipLaunchKernelGGL(group_count_kernel, dim3(chunks), dim3(1024), size_t(G) * sizeof(int32_t), stream, p, chunk, hist);
    hipLaunchKernelGGL(group_scan_kernel, dim3((G + 31) / 32), dim3(1024), 0, stream, p, chunks, hist, totals);
    launch_place<16>(waves, p, chunks, chunk, hist, totals, bits, stream);
    return hipGetLastError();
}

}  // namespace fff

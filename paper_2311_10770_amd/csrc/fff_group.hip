// fff_group.hip -- fff_group_rows: a stable counting sort of entries by group.
//
// Entries are cut into chunks; a workgroup counts its chunk's entries per
// group in LDS (hist), every group's counts become running sums over the
// chunks, the totals the groups' offsets, and a wave per chunk places the
// chunk's entries in order.  Within a wave equal groups are found with one
// ballot per bit of the group number, so no order depends on an atomic.
#include "fff_internal.hpp"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

namespace fff {

namespace {

constexpr int GROUP_CHUNKS = 256;  // at most
constexpr int64_t GROUP_MIN_CHUNK = 1024;

int64_t group_chunk(int64_t n) {
    const int64_t c = (n + GROUP_CHUNKS - 1) / GROUP_CHUNKS;
    return std::max(GROUP_MIN_CHUNK, (c + 63) / 64 * 64);
}
int64_t group_chunks(int64_t n) { return (n + group_chunk(n) - 1) / group_chunk(n); }

// The group of entry e, or -1.
__device__ __forceinline__ int group_of(const GroupParams& p, int64_t e) {
    const int64_t id = int64_t(p.ids[e]) - p.first;
    return id >= 0 && id < p.n_ids ? int(e % p.n_trees) * p.n_ids + int(id) : -1;
}

__global__ __launch_bounds__(256) void group_count_kernel(GroupParams p, int64_t chunk) {
    extern __shared__ int32_t g_cnt[];  // [n_groups]
    const int G = p.n_groups;
    for (int g = threadIdx.x; g < G; g += 256) g_cnt[g] = 0;
    __syncthreads();
    const int64_t e1 = std::min<int64_t>(p.n_entries, (int64_t(blockIdx.x) + 1) * chunk);
    for (int64_t e = int64_t(blockIdx.x) * chunk + threadIdx.x; e < e1; e += 256) {
        const int g = group_of(p, e);
        if (g >= 0) atomicAdd(&g_cnt[g], 1);
        else if (p.bad) atomicAdd(p.bad, 1);
    }
    __syncthreads();
    int32_t* hist = static_cast<int32_t*>(p.workspace) + int64_t(blockIdx.x) * G;
    for (int g = threadIdx.x; g < G; g += 256) hist[g] = g_cnt[g];
}

// Counts become running sums over the chunks; the totals go to offsets[1 + g].
__global__ __launch_bounds__(256) void group_scan_kernel(GroupParams p, int chunks) {
    const int64_t g = int64_t(blockIdx.x) * 256 + threadIdx.x;
    const int G = p.n_groups;
    if (g >= G) return;
    int32_t* hist = static_cast<int32_t*>(p.workspace);
    int32_t run = 0;
    for (int c = 0; c < chunks; ++c) {
        const int32_t v = hist[int64_t(c) * G + g];
        hist[int64_t(c) * G + g] = run;
        run += v;
    }
    p.offsets[1 + g] = run;
}

// offsets: totals to inclusive sums, by one workgroup.
__global__ __launch_bounds__(1024) void group_offsets_kernel(GroupParams p) {
    __shared__ int32_t part[1024];
    const int G = p.n_groups, tid = threadIdx.x, per = (G + 1023) / 1024;
    const int g0 = std::min(G, tid * per), g1 = std::min(G, g0 + per);
    int32_t sum = 0;
    for (int g = g0; g < g1; ++g) sum += p.offsets[1 + g];
    part[tid] = sum;
    __syncthreads();
    for (int d = 1; d < 1024; d *= 2) {
        const int32_t v = tid >= d ? part[tid - d] : 0;
        __syncthreads();
        part[tid] += v;
        __syncthreads();
    }
    int32_t run = part[tid] - sum;
    for (int g = g0; g < g1; ++g) {
        run += p.offsets[1 + g];
        p.offsets[1 + g] = run;
    }
    if (tid == 0) p.offsets[0] = 0;
}

__global__ __launch_bounds__(64) void group_place_kernel(GroupParams p, int64_t chunk, int bits) {
    extern __shared__ int32_t g_next[];  // [n_groups] next place of each group
    const int G = p.n_groups, lane = threadIdx.x;
    const int32_t* hist = static_cast<const int32_t*>(p.workspace) + int64_t(blockIdx.x) * G;
    for (int g = lane; g < G; g += 64) g_next[g] = p.offsets[g] + hist[g];
    __syncthreads();
    const int64_t e1 = std::min<int64_t>(p.n_entries, (int64_t(blockIdx.x) + 1) * chunk);
    for (int64_t e0 = int64_t(blockIdx.x) * chunk; e0 < e1; e0 += 64) {
        const int64_t e = e0 + lane;
        const int g = e < e1 ? group_of(p, e) : -1;
        uint64_t same = __ballot(g >= 0);
        for (int b = 0; b < bits; ++b) {
            const uint64_t set = __ballot((g >> b) & 1);
            same &= (g >> b) & 1 ? set : ~set;
        }
        const int before = __popcll(same & ((uint64_t(1) << lane) - 1));
        int32_t place = 0;
        if (g >= 0) place = g_next[g] + before;
        __syncthreads();
        if (g >= 0) {
            if (before == 0) g_next[g] += __popcll(same);
            p.order[place] = int32_t(e);
        }
        __syncthreads();
    }
}

}  // namespace

size_t group_workspace_bytes(int64_t n_entries, int32_t n_groups) {
    return size_t(group_chunks(n_entries)) * size_t(n_groups) * sizeof(int32_t);
}

hipError_t run_group_rows(const GroupParams& p, hipStream_t stream) {
    const int G = p.n_groups;
    const int64_t chunk = group_chunk(p.n_entries);
    const int chunks = int(group_chunks(p.n_entries));
    const size_t lds = size_t(G) * sizeof(int32_t);
    int bits = 0;
    while ((1 << bits) < G) ++bits;
    if (chunks > 0) hipLaunchKernelGGL(group_count_kernel, dim3(chunks), dim3(256), lds, stream, p, chunk);
    hipLaunchKernelGGL(group_scan_kernel, dim3((G + 255) / 256), dim3(256), 0, stream, p, chunks);
    hipLaunchKernelGGL(group_offsets_kernel, dim3(1), dim3(1024), 0, stream, p);
    if (chunks > 0) hipLaunchKernelGGL(group_place_kernel, dim3(chunks), dim3(64), lds, stream, p, chunk, bits);
    return hipGetLastError();
}

}  // namespace fff

// fff_route.hip -- routing of tokens to experts and its gradient (fff_route,
// fff_route_backward).
//
// The choice is an order of sums s_e + b_e whose neighbours may lie closer than fp32's
// roundings; it is taken in fp64 (or, without a bias, by the logits themselves,
// which the scores grow with), so that it depends on the logits alone.
#include "fff_device.hpp"
#include "fff_operators.hpp"
#include "fff_rows.hpp"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

namespace fff {

namespace {

constexpr float NONE = -__builtin_inff();

// A logit: -inf where it is NaN (no expert), the largest fp32 value where it is infinite.
__device__ __forceinline__ float clean_logit(float l) {
    return l > NONE ? __builtin_fminf(l, 3.4028234663852886e38f) : NONE;
}
__device__ __forceinline__ float logit(const RouteParams& p, int64_t row, int e) {
    return clean_logit(load_elem(p.logits, p.bf16, row * p.n_experts + e));
}

// A token's softmax as fp64 exponentials: exp(l - most) / sum.
struct Softmax {
    float most;
    double sum;
};
__device__ __forceinline__ double score(float l, int sigmoid, const Softmax& m) {
    if (l == NONE) return 0.0;
    return sigmoid ? 1.0 / (1.0 + exp(-double(l))) : exp(double(l) - double(m.most)) / m.sum;
}

constexpr int ANY = 256;  // threads of the kernel for any size

// Largest v (lowest i among equals) of the workgroup, for every thread.
__device__ __forceinline__ void block_best(double& v, int& i, double* sv, int* si) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const double w = __shfl_xor(v, d);
        const int j = __shfl_xor(i, d);
        if (w > v || (w == v && j < i)) {
            v = w;
            i = j;
        }
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) {
        sv[threadIdx.x >> 6] = v;
        si[threadIdx.x >> 6] = i;
    }
    __syncthreads();
    v = sv[0];
    i = si[0];
#pragma unroll
    for (int w = 1; w < ANY / 64; ++w)
        if (sv[w] > v || (sv[w] == v && si[w] < i)) {
            v = sv[w];
            i = si[w];
        }
}
__device__ __forceinline__ double block_add(double v, double* sv) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sv[threadIdx.x >> 6] = v;
    __syncthreads();
    return (sv[0] + sv[1]) + (sv[2] + sv[3]);
}

// Any number of experts: a workgroup a token.  Nothing is kept of the row but its groups: each pick is the
// best expert that comes behind the one before it in the order.
__global__ __launch_bounds__(ANY) void route_any_kernel(RouteParams p) {
    __shared__ double sv[ANY / 64], s_group[MAX_ROUTE_GROUPS];
    __shared__ int si[ANY / 64];
    __shared__ uint8_t s_kept[MAX_ROUTE_GROUPS];
    __shared__ float s_logit[MAX_TOP_K];
    const int E = p.n_experts, G = p.n_groups, size = E / G, tid = threadIdx.x;
    for (int64_t row = blockIdx.x; row < p.n_tokens; row += gridDim.x) {
        Softmax m{0.0f, 1.0};
        if (p.score == SCORE_SOFTMAX) {
            double most = -HUGE_VAL;
            int at = 0;
            for (int e = tid; e < E; e += ANY) most = fmax(most, double(logit(p, row, e)));
            block_best(most, at, sv, si);
            m.most = float(most);
            double sum = 0.0;
            for (int e = tid; e < E; e += ANY) {
                const float l = logit(p, row, e);
                if (l > NONE) sum += exp(double(l) - most);
            }
            m.sum = block_add(sum, sv);
        }
        auto choice = [&](int e) {
            const float l = logit(p, row, e);
            if (l == NONE) return -HUGE_VAL;
            const double c = p.bias ? score(l, p.score, m) + double(p.bias[e]) : double(l);
            return c > -HUGE_VAL ? c : -HUGE_VAL;
        };
        if (G > 1) {
            __syncthreads();
            for (int g = tid; g < G; g += ANY) {
                double a = -HUGE_VAL, b = -HUGE_VAL;
                for (int e = g * size; e < (g + 1) * size; ++e) {
                    double c = choice(e);
                    if (!p.bias && p.group_score == GROUP_TOP2 && c > -HUGE_VAL) c = score(logit(p, row, e), p.score, m);
                    b = fmax(b, fmin(a, c));
                    a = fmax(a, c);
                }
                s_group[g] = p.group_score == GROUP_TOP2 && b > -HUGE_VAL ? a + b : a;
            }
            __syncthreads();
            for (int g = tid; g < G; g += ANY) {
                const double v = s_group[g];
                int before = 0;
                for (int h = 0; h < G; ++h) before += s_group[h] > v || (s_group[h] == v && h < g);
                s_kept[g] = v > -HUGE_VAL && before < p.top_groups;
            }
            __syncthreads();
        }
        double last = HUGE_VAL;
        int last_at = -1, got = 0;
        for (; got < p.top_k; ++got) {
            double best = -HUGE_VAL;
            int at = E;
            for (int e = tid; e < E; e += ANY) {
                if (G > 1 && !s_kept[e / size]) continue;
                const double c = choice(e);
                if (c > best && (c < last || (c == last && e > last_at))) {
                    best = c;
                    at = e;
                }
            }
            block_best(best, at, sv, si);
            if (best == -HUGE_VAL) break;
            last = best;
            last_at = at;
            if (tid == 0) {
                p.ids[row * p.top_k + got] = at;
                s_logit[got] = logit(p, row, at);
            }
        }
        __syncthreads();
        if (tid < p.top_k) {
            // renormalised sums start from the largest chosen logit: scores that underflow keep their shares
            float most = NONE;
            for (int j = 0; j < got; ++j) most = __builtin_fmaxf(most, s_logit[j]);
            const bool small = p.renormalise && (p.score == SCORE_SOFTMAX || most < -300.0f);
            auto weight = [&](int j) {
                return small ? exp(double(s_logit[j]) - double(most)) : score(s_logit[j], p.score, m);
            };
            double w = tid < got ? weight(tid) : 0.0;
            if (p.renormalise && tid < got) {
                double sum = 0.0;
                for (int j = 0; j < got; ++j) sum += weight(j);
                w /= sum;
            }
            p.weights[row * p.top_k + tid] = float(double(p.scale) * w);
            if (tid >= got) p.ids[row * p.top_k + tid] = -1;
        }
        __syncthreads();
    }
}

// The gradient: a wave a token.
__global__ __launch_bounds__(256) void route_bwd_any_kernel(RouteBwdParams p) {
    const int lane = threadIdx.x & 63, E = p.n_experts, K = p.top_k;
    const bool sigmoid = p.score != SCORE_SOFTMAX;
    for (int64_t row = int64_t(blockIdx.x) * 4 + (threadIdx.x >> 6); row < p.n_tokens; row += int64_t(gridDim.x) * 4) {
        auto at = [&](int e) { return clean_logit(load_elem(p.logits, p.bf16, row * E + e)); };
        float most = NONE, sum = 1.0f;
        // entry `lane` of the token
        int id = -1;
        float l = NONE, d = 0.0f;
        if (lane < K) {
            id = p.ids[row * K + lane];
            if (id < 0 || id >= E) id = -1;
            else l = at(id);
            if (l == NONE) id = -1;
            d = id >= 0 ? p.scale * p.dweights[row * K + lane] : 0.0f;
        }
        auto wave_max = [](float v) {
            for (int s = 1; s < 64; s *= 2) v = __builtin_fmaxf(v, __shfl_xor(v, s));
            return v;
        };
        if (p.renormalise) most = wave_max(l);
        else if (!sigmoid) {
            for (int e = lane; e < E; e += 64) most = __builtin_fmaxf(most, at(e));
            most = wave_max(most);
            sum = 0.0f;
            for (int e = lane; e < E; e += 64) {
                const float v = at(e);
                if (v > NONE) sum += expf(v - most);
            }
            sum = group_sum<64>(sum);
        }
        const bool shifted = !sigmoid || (p.renormalise && most < -60.0f);
        // this entry's part of d, and what is taken from every expert's
        float s = id < 0 ? 0.0f : shifted ? expf(l - most) : 1.0f / (1.0f + expf(-l)), all = 0.0f;
        if (p.renormalise) {
            const float total = group_sum<64>(s);
            s = id < 0 ? 0.0f : s / total;
            d = s * (d - group_sum<64>(d * s));
        } else if (!sigmoid) {
            all = group_sum<64>(d * (s / sum));
        }
        for (int e = lane; e - lane < E; e += 64) {
            float own = 0.0f;
            for (int j = 0; j < K; ++j) {
                const int i = __shfl(id, j);
                const float v = __shfl(d, j);
                if (i == e) own += v;
            }
            if (e >= E) continue;
            const float v = at(e);
            float g = 0.0f;
            if (v > NONE) {
                if (sigmoid) {
                    const float rest = 1.0f / (1.0f + expf(v));  // 1 - s
                    g = own == 0.0f ? 0.0f : p.renormalise ? own * rest : own * (1.0f / (1.0f + expf(-v))) * rest;
                } else {
                    g = p.renormalise ? own : expf(v - most) / sum * (own - all);
                }
            }
            store_elem(p.dlogits, p.d_bf16, row * E + e, g);
        }
    }
}

}  // namespace

hipError_t run_route(const RouteParams& p, const DeviceInfo& dev, hipStream_t stream) {
    const unsigned grid = unsigned(std::min<int64_t>(p.n_tokens, 8 * std::max(dev.cu_count, 1)));
    hipLaunchKernelGGL(route_any_kernel, dim3(grid), dim3(ANY), 0, stream, p);
    return hipGetLastError();
}

hipError_t run_route_backward(const RouteBwdParams& p, const DeviceInfo& dev, hipStream_t stream) {
    const unsigned grid = unsigned(std::min<int64_t>((p.n_tokens + 3) / 4, 8 * std::max(dev.cu_count, 1)));
    hipLaunchKernelGGL(route_bwd_any_kernel, dim3(grid), dim3(256), 0, stream, p);
    return hipGetLastError();
}

}  // namespace fff

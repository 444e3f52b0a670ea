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
#include <type_traits>

namespace fff {

namespace {

constexpr float NONE = -__builtin_inff();

// A sigmoid times exp(-shift), for shift = 0 or the largest of a token's chosen logits where that is below 0: the common factor
// cancels from their shares, which so keep their bits where the sigmoids themselves leave fp32 (1 / (1 + exp(-l)) is 0 from
// -88.8 on; its share beside one at -19 is 1e-30).  No step overflows: of -l it is 1 - s down to fp32's smallest step.
__device__ __forceinline__ float sigmoid_part(float l, float shift) {
    return expf(__builtin_fminf(l, 0.0f) - shift) / (1.0f + expf(-__builtin_fabsf(l)));
}

// A logit: -inf where it is NaN (no expert), the largest fp32 value where it is infinite.
__device__ __forceinline__ float clean_logit(float l) {
    return __builtin_fminf(__builtin_fmaxf(l, NONE), 3.4028234663852886e38f);  // the larger of NaN and a number is that
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

// What an expert is chosen by.
__device__ __forceinline__ double choice(const RouteParams& p, float l, int e, const Softmax& m) {
    if (l == NONE) return -HUGE_VAL;
    const double c = p.bias ? score(l, p.score, m) + double(p.bias[e]) : double(l);
    return c > -HUGE_VAL ? c : -HUGE_VAL;
}

// ---- up to 1024 experts: LPT lanes a token ---------------------------------

// v of the lane that a DPP control names (one that has a lane for each, as the rotations of a row of 16 do).
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xf, 0xf, true));
}
constexpr int ROR = 0x120;  // row_ror: + 1 .. 15

// Largest v of the LPT lanes of a token, for each of them.
template <int LPT>
__device__ __forceinline__ float group_max(float v) {
    v = __builtin_fmaxf(v, dpp<ROR + 8>(v));
    v = __builtin_fmaxf(v, dpp<ROR + 4>(v));
    v = __builtin_fmaxf(v, dpp<ROR + 2>(v));
    v = __builtin_fmaxf(v, dpp<ROR + 1>(v));
    if constexpr (LPT >= 32) v = __builtin_fmaxf(v, __shfl_xor(v, 16));
    if constexpr (LPT == 64) v = __builtin_fmaxf(v, __shfl_xor(v, 32));
    return v;
}
// bits, one place up, with the sign bit of d below them: of differences, a bit for each that is negative in two
// instructions (a comparison and its count are three).  Of finite values: infinities less themselves are NaN.
__device__ __forceinline__ uint32_t push_sign(uint32_t bits, float d) {
    return __builtin_amdgcn_alignbit(bits, __float_as_uint(d), 31);
}
__device__ __forceinline__ float finite_value(float v) {
    return __builtin_amdgcn_fmed3f(v, -3.4028234663852886e38f, 3.4028234663852886e38f);
}
// A bit for each of the 16 values of w that the lane's row holds that is larger than v.
template <int R = 0>
__device__ __forceinline__ uint32_t row_larger(float v, float w, uint32_t bits = 0) {
    if constexpr (R == 16) {
        return bits;
    } else {
        const float x = R == 0 ? w : dpp<ROR + (R == 0 ? 1 : R)>(w);
        return row_larger<R + 1>(v, w, push_sign(bits, v - x));
    }
}
// How many of the LPT lanes' (finite) values w are larger than v.
template <int LPT>
__device__ __forceinline__ int group_larger(float v, float w) {
    int n = __builtin_popcount(row_larger(v, w));
    if constexpr (LPT >= 32) n += __builtin_popcount(row_larger(v, __shfl_xor(w, 16)));
    if constexpr (LPT == 64)
        n += __builtin_popcount(row_larger(v, __shfl_xor(w, 32))) + __builtin_popcount(row_larger(v, __shfl_xor(w, 48)));
    return n;
}
// The bits of all of the token's lanes.
template <int LPT>
__device__ __forceinline__ uint32_t group_or(uint32_t v) {
    v |= __builtin_amdgcn_mov_dpp(int(v), ROR + 8, 0xf, 0xf, true);
    v |= __builtin_amdgcn_mov_dpp(int(v), ROR + 4, 0xf, 0xf, true);
    v |= __builtin_amdgcn_mov_dpp(int(v), ROR + 2, 0xf, 0xf, true);
    v |= __builtin_amdgcn_mov_dpp(int(v), ROR + 1, 0xf, 0xf, true);
    if constexpr (LPT >= 32) v |= __shfl_xor(v, 16);
    return v;
}
// Sum of v over the token's lanes before this one.
template <int LPT>
__device__ __forceinline__ int group_before(int v, int sl) {
    int sum = v;
#pragma unroll
    for (int d = 1; d < LPT; d *= 2) {
        const int w = __shfl_up(sum, d);
        if (sl >= d) sum += w;
    }
    return sum - v;
}
__device__ __forceinline__ void wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// The larger two of (a, b) and the same pair of the lane that CTRL (a DPP control) names.
template <int CTRL>
__device__ __forceinline__ void top2_step(float& a, float& b) {
    const float x = dpp<CTRL>(a), y = dpp<CTRL>(b);
    b = __builtin_fmaxf(__builtin_fmaxf(b, y), __builtin_fminf(a, x));
    a = __builtin_fmaxf(a, x);
}

// The best (v, then the lowest i) of the wave's lanes, for each of them.
__device__ __forceinline__ void wave_best(double& v, int& i) {
    auto meet = [&](double w, int j) {
        const bool take = w > v || (w == v && j < i);
        v = take ? w : v;
        i = take ? j : i;
    };
    auto step = [&](auto ctrl) {
        const uint64_t u = __builtin_bit_cast(uint64_t, v);
        const uint32_t lo = __builtin_amdgcn_mov_dpp(int(uint32_t(u)), ctrl.value, 0xf, 0xf, true);
        const uint32_t hi = __builtin_amdgcn_mov_dpp(int(uint32_t(u >> 32)), ctrl.value, 0xf, 0xf, true);
        meet(__builtin_bit_cast(double, uint64_t(hi) << 32 | lo), __builtin_amdgcn_mov_dpp(i, ctrl.value, 0xf, 0xf, true));
    };
    step(std::integral_constant<int, ROR + 8>{});
    step(std::integral_constant<int, ROR + 4>{});
    step(std::integral_constant<int, ROR + 2>{});
    step(std::integral_constant<int, ROR + 1>{});
    // rows, then halves: each swap hands a lane both partners' values, of which it holds one
    auto swap = [&](auto step32) {
        auto both = [&](uint32_t u) {
            if constexpr (step32.value) return __builtin_amdgcn_permlane32_swap(u, u, false, false);
            else return __builtin_amdgcn_permlane16_swap(u, u, false, false);
        };
        const uint64_t u = __builtin_bit_cast(uint64_t, v);
        const auto lo = both(uint32_t(u)), hi = both(uint32_t(u >> 32)), at = both(uint32_t(i));
        v = __builtin_bit_cast(double, uint64_t(hi[0]) << 32 | lo[0]);
        i = int(at[0]);
        meet(__builtin_bit_cast(double, uint64_t(hi[1]) << 32 | lo[1]), int(at[1]));
    };
    swap(std::false_type{});
    swap(std::true_type{});
}

constexpr int ANY = 256;  // threads of the kernel for any size

// Largest v (lowest i among equals) of the workgroup, for every thread.  Calls alternate between two of sv and si, so one
// barrier a call is enough.
__device__ __forceinline__ void block_best(double& v, int& i, double* sv, int* si) {
    wave_best(v, i);
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

// ---- any number of experts, groups and picks: a workgroup a token ------------
//
// All of it in fp64.  Nothing is kept of the row but its groups' values and each thread's best expert: a pick is a
// reduction over the workgroup, behind which one wave looks through the winner's experts again.  4096 tokens, top 8 of 2048
// bf16: 71 us, 123 with softmax, bias and groups (a pass over the row for each pick took 143 and 377).
__global__ __launch_bounds__(ANY) void route_any_kernel(RouteParams p) {
    __shared__ double sv[2][ANY / 64], s_add[ANY / 64], s_group[MAX_ROUTE_GROUPS];
    __shared__ int si[2][ANY / 64];
    __shared__ uint8_t s_kept[MAX_ROUTE_GROUPS];
    __shared__ float s_logit[MAX_TOP_K];
    const int E = p.n_experts, G = p.n_groups, size = p.group_size, tid = threadIdx.x;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < p.n_tokens; row += gridDim.x) {
        Softmax m{0.0f, 1.0};
        if (p.score == SCORE_SOFTMAX && (p.bias || !p.renormalise || (G > 1 && p.group_score == GROUP_TOP2))) {
            double most = -HUGE_VAL;
            int at = 0;
            for (int e = tid; e < E; e += ANY) most = fmax(most, double(logit(p, row, e)));
            block_best(most, at, sv[turn], si[turn]);
            turn ^= 1;
            m.most = float(most);
            double sum = 0.0;
            for (int e = tid; e < E; e += ANY) {
                const float l = logit(p, row, e);
                if (l > NONE) sum += exp(double(l) - most);
            }
            m.sum = block_add(sum, s_add);
        }
        if (G > 1) {
            __syncthreads();
            // h threads a group, that many experts apart
            int h = 1;
            while (h < 64 && 2 * h * G <= ANY) h *= 2;
            for (int g0 = 0; g0 < G; g0 += ANY / h) {
                const int g = g0 + tid / h;
                double a = -HUGE_VAL, b = -HUGE_VAL;  // the group's largest, and the second
                auto take = [&](double c) {
                    b = fmax(b, fmin(a, c));
                    a = fmax(a, c);
                };
                for (int e = g * size + tid % h; g < G && e < (g + 1) * size; e += h) {
                    const float l = logit(p, row, e);
                    double c = choice(p, l, e, m);
                    if (!p.bias && p.group_score == GROUP_TOP2 && c > -HUGE_VAL) c = score(l, p.score, m);
                    take(c);
                }
                for (int d = 1; d < h; d *= 2) {
                    const double x = __shfl_xor(a, d), y = __shfl_xor(b, d);
                    take(x);
                    b = fmax(b, y);
                }
                if (g < G && tid % h == 0) s_group[g] = p.group_score == GROUP_TOP2 && b > -HUGE_VAL ? a + b : a;
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
        // a thread has the best of the experts tid, tid + ANY, ...; when it is picked, the lanes of its wave look for the next
        double last = HUGE_VAL, v = -HUGE_VAL;
        int last_at = -1, mine = E, got = 0;
        auto look = [&](int e0, int step, double& best, int& at) {
            for (int e = e0; e < E; e += step) {
                if (G > 1 && !s_kept[e / size]) continue;
                const double c = choice(p, logit(p, row, e), e, m);
                if (c > best && (c < last || (c == last && e > last_at))) {
                    best = c;
                    at = e;
                }
            }
        };
        look(tid, ANY, v, mine);
        for (; got < p.top_k; ++got) {
            double best = v;
            int at = mine;
            block_best(best, at, sv[turn], si[turn]);
            turn ^= 1;
            if (best == -HUGE_VAL) break;
            last = best;
            last_at = at;
            const int owner = at % ANY;
            if (owner >> 6 == tid >> 6) {
                double next = -HUGE_VAL;
                int next_at = E;
                look(owner + ANY * (tid & 63), ANY * 64, next, next_at);
                wave_best(next, next_at);
                if (tid == owner) {
                    v = next;
                    mine = next_at;
                }
            }
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

// What few tokens come to, by a whole wave: the fp64 values that a token's experts are chosen by (groups: that its groups
// are) go to LDS, by_e, and the softmax's largest logit and sum come back.
__device__ __forceinline__ Softmax choices64(const RouteParams& p, int64_t row, bool groups, double* by_e) {
    const int lane = threadIdx.x & 63, E = p.n_experts;
    const bool plain = groups && p.group_score == GROUP_TOP2 && !p.bias;  // by s, where experts go by their logits
    Softmax m{0.0f, 1.0};
    wave_sync();
#pragma unroll 4
    for (int e = lane; e < E; e += 64) by_e[e] = double(logit(p, row, e));
    if (p.score == SCORE_SOFTMAX) {
        float most = NONE;
        for (int e = lane; e < E; e += 64) most = __builtin_fmaxf(most, float(by_e[e]));
        most = group_max<64>(most);
        m.most = most > NONE ? most : 0.0f;
        double sum = 0.0;
        for (int e = lane; e < E; e += 64) sum += by_e[e] > -HUGE_VAL ? exp(by_e[e] - double(m.most)) : 0.0;
#pragma unroll
        for (int x = 1; x < 64; x *= 2) sum += __shfl_xor(sum, x);
        m.sum = sum > 0.0 ? sum : 1.0;
    }
    if (p.bias || plain) {
#pragma unroll 2
        for (int e = lane; e < E; e += 64) {
            const float l = float(by_e[e]);
            by_e[e] = plain ? (l > NONE ? score(l, p.score, m) : -HUGE_VAL) : choice(p, l, e, m);
        }
    }
    wave_sync();
    return m;
}

// A token's groups (at most 64) by their fp64 values: a bit every 1 << shift for each that is kept.
__device__ __forceinline__ uint64_t kept_groups(const RouteParams& p, int64_t row, int shift, double* by_e) {
    const int lane = threadIdx.x & 63, G = p.n_groups, size = p.group_size, g = lane >> shift;
    choices64(p, row, true, by_e);
    double a = -HUGE_VAL, b = -HUGE_VAL;
    if (g < G) {
        int at = g % size;  // groups start at different banks
#pragma unroll 4
        for (int i = 0; i < size; ++i) {
            const double c = by_e[g * size + at];
            at = at + 1 == size ? 0 : at + 1;
            b = fmax(b, fmin(a, c));
            a = fmax(a, c);
        }
    }
    const double value = p.group_score == GROUP_TOP2 && b > -HUGE_VAL ? a + b : a;
    int before = 0;
    for (int h = 0; h < G; ++h) {
        const double v = __shfl(value, h << shift);
        before += v > value || (v == value && h < g);
    }
    wave_sync();
    return __ballot(g < G && value > -HUGE_VAL && before < p.top_groups);
}

// A token with more candidates than route_kernel has room for: each pick is the best that is left of all.
__device__ __forceinline__ void route_token(const RouteParams& p, int64_t row, uint64_t kept, int shift, double* by_e) {
    const int lane = threadIdx.x & 63, E = p.n_experts, size = p.group_size;
    const Softmax m = choices64(p, row, false, by_e);
    if (p.n_groups > 1) {
        for (int e = lane; e < E; e += 64)
            if (!(kept >> (e / size << shift & 63) & 1)) by_e[e] = -HUGE_VAL;
    }
    auto mine_best = [&](double& v, int& i) {
        v = -HUGE_VAL;
        i = E;
#pragma unroll 4
        for (int e = lane; e < E; e += 64) {
            const double c = by_e[e];
            if (c > v) {
                v = c;
                i = e;
            }
        }
    };
    double v;
    int at, picks = 0, mine = -1;
    mine_best(v, at);
    for (; picks < p.top_k; ++picks) {
        double best = v;
        int where = at;
        wave_best(best, where);
        if (best == -HUGE_VAL) break;
        if (lane == picks) mine = where;
        if (where == at) {  // this lane's: the next of its own
            by_e[at] = -HUGE_VAL;
            mine_best(v, at);
        }
    }
    // renormalised sums start from the largest chosen logit: scores that underflow keep their shares
    const float own = mine >= 0 ? logit(p, row, mine) : NONE, top = group_max<64>(own);
    double w = 0.0;
    if (mine >= 0)
        w = p.renormalise && (p.score == SCORE_SOFTMAX || top < -300.0f) ? exp(double(own) - double(top)) : score(own, p.score, m);
    if (p.renormalise) {
        double sum = w;
#pragma unroll
        for (int x = 1; x < 64; x *= 2) sum += __shfl_xor(sum, x);
        w = mine >= 0 ? w / sum : 0.0;
    }
    if (lane < p.top_k) {
        p.ids[row * p.top_k + lane] = mine;
        p.weights[row * p.top_k + lane] = float(double(p.scale) * w);
    }
    wave_sync();
}

// What one wave holds in LDS: the choices by expert, a list of its tokens' candidates, and what one token's experts are
// chosen by in fp64.
template <int LPT, int V>
struct RouteLds {
    static constexpr int CAP = 4 * LPT;  // candidates of a token, whose fp64 choices lie in the place of c
    static constexpr int AREA = V >= 8 ? LPT * V : 2 * CAP;  // of a token in c
    float c[64 / LPT * AREA];
    double by_e[LPT * V];
    uint16_t e[64 / LPT][CAP];       // candidates
    uint16_t chosen[64 / LPT][CAP];  // in order
};

// LPT lanes a token (16, 32 or 64), four neighbouring experts a vector, V experts a lane: lanes hold few experts each, in
// registers, and a wave 64 / LPT tokens.  One lane a pick at least: the largest of each lane's own bound the choice, where
// there are less than two a pick the largest two (33530 tokens, top 14 of 64 in groups: 45 us with 32 lanes and
// their largest alone, 16.7 with 16 lanes).  64 lanes keep to the largest alone: with the two 40 of 64 experts take 38 us
// for 24 (at five waves a SIMD they spill 16 to 22 registers up to 512 experts) and 8 of 1024 98 for 96, but 40 of 1024
// 187 for 228.
//
// Bound by vector instructions, which issue in 0.8 to 1.0 of a SIMD's cycles throughout: 65536 tokens, top 8 of 256 fp32
// (71 MB: 14 us at a copy's rate): by the logits 16.9 us (494 instructions a wave), sigmoid and bias 24 (626), softmax and
// bias 27.6 (641); sigmoid, bias and the best 4 of 8 groups 31 (4 of 16: 33), of which the groups are a quarter.  Each pick
// by a reduction over the lanes, in fp64, cost 1988 there.  One token of 64 experts: 3.0 us, the launch, behind the host's
// 9.  Few experts leave most of a token's lanes without any, at the same instructions: 2 of 8 and 4 of 32 12.4 us (403), for
// 0.6 and 2.1 at a copy's rate.  A wave of 64 lanes has one token for as many (65536 x 1024 bf16, top 8: 96 us, 729 a wave;
// 28 at a copy's rate); of its 13 KB of LDS there three workgroups fit a CU.  Five waves a SIMD: at 32 lanes up to
// 256 experts 13 registers are kept in scratch for them, which costs nothing that shows (24 of 256 with sigmoid and bias
// 52.6 us, 52.2 at four waves without scratch; 24 of 128 36.4 and 36.4).
//
// Choices are first formed in fp32 (c, whose error is below `slack` / 2).  Of the LPT lanes' largest, the
// top_k-th is no more than the top_k-th largest of all, and the same holds for the largest two of each, so only
// experts within the slack of it can be chosen: a dozen of 256.  These candidates alone are ordered, each by counting
// those before it; where two neighbours in that order lie within the slack, the token's candidates are evaluated and ordered
// in fp64.
// Groups whose values leave their choice open are resolved by kept_groups, and tokens that have more candidates
// than there is room for (as where all logits are equal) are left to route_token: whole waves, in fp64 (65536 tokens of 256
// equal logits: 150 to 237 us).
template <int LPT, int V>
__global__ __launch_bounds__(256, 5) void route_kernel(RouteParams p, int64_t row0) {
    using Lds = RouteLds<LPT, V>;
    constexpr int TPW = 64 / LPT, CAP = Lds::CAP, N = V / 4;
    __shared__ Lds lds4[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sl = lane % LPT, tok = lane / LPT, first = tok * LPT;
    Lds& lds = lds4[wave];
    uint16_t* const list = lds.e[tok];
    uint16_t* const order = lds.chosen[tok];
    const int E = p.n_experts, K = p.top_k, G = p.n_groups, size = p.group_size;
    const bool sigmoid = p.score != SCORE_SOFTMAX, top2 = p.group_score == GROUP_TOP2;
    const bool by_score = p.bias || (G > 1 && top2);  // whether fp32 scores take part in the choice
    const bool sums = !sigmoid && (by_score || !p.renormalise);
    const int64_t r0 = (row0 / TPW + int64_t(blockIdx.x) * 4 + wave) * TPW;
    if (r0 >= p.n_tokens) return;
    const bool in = r0 + tok < p.n_tokens;
    const int64_t row = in ? r0 + tok : p.n_tokens - 1;  // lanes behind the last token do it again
    constexpr uint64_t TOKEN = LPT == 64 ? ~0ull : (1ull << LPT % 64) - 1;
    const float* bias = p.bias;
    // groups of V, 2 V .. 16 V experts: lane sl takes V neighbouring experts out of LDS, all of one group, for its value (the
    // registers' own vectors lie in N groups, whose pairs took 16 us of 36 where this takes 14 of 34).  The choice keeps
    // to the registers' layout: there the experts of few groups lie in more lanes, and bound it better (34 us, 53 else)
    const int part = size / V;
    const bool whole = G > 1 && size % V == 0 && part <= 16 && (part & (part - 1)) == 0;
    uint64_t kept = ~0ull;  // G > 1: a token's groups, one every 1 << shift bits
    int shift = 0;
    if (whole) shift = __builtin_ctz(part);
    else
        while (shift < 4 && (G << (shift + 1)) <= LPT) ++shift;
    auto lane_max = [](const float (&x)[V]) {
        float m = x[0];
#pragma unroll
        for (int v = 1; v < V; ++v) m = __builtin_fmaxf(m, x[v]);
        return m;
    };
    float l[V], c[V];
    float* const all = lds.c + tok * Lds::AREA;
    auto put4 = [&](float* to, int q, const float (&x)[V]) {
        *reinterpret_cast<float4*>(to + (q * LPT + sl) * 4) = make_float4(x[4 * q], x[4 * q + 1], x[4 * q + 2], x[4 * q + 3]);
    };
    if (E == LPT * V) {
#pragma unroll
        for (int q = 0; q < N; ++q)
            unpack4(l + 4 * q, load4<true>(p.logits, p.bf16, row * E + (q * LPT + sl) * 4, 4), p.bf16);
    } else {
#pragma unroll
        for (int q = 0; q < N; ++q) {
            const int col = (q * LPT + sl) * 4;
            unpack4(l + 4 * q, load4<false>(p.logits, p.bf16, row * E + col, E - col), p.bf16);
#pragma unroll
            for (int j = 0; j < 4; ++j) l[4 * q + j] = j < E - col ? l[4 * q + j] : NONE;
        }
    }
#pragma unroll
    for (int v = 0; v < V; ++v) l[v] = clean_logit(l[v]);
    Softmax soft{0.0f, 1.0};
    float z = 1.0f;
    if (!sigmoid) {
        const float most = group_max<LPT>(lane_max(l));
        soft.most = most > NONE ? most : 0.0f;
    }
    if (sums) {
        z = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            c[v] = __builtin_amdgcn_exp2f(1.44269504088896341f * (l[v] - soft.most));  // 0 where there is none
            z += c[v];
        }
        z = group_sum<LPT>(z);
        z = z > 0.0f ? z : 1.0f;
        soft.sum = double(z);
    }
    const float share = sigmoid ? 1.0f : 1.0f / z;  // no score is larger
    if (by_score) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            if (sigmoid) c[v] = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896341f * l[v]));
            else c[v] *= share;
        }
    }
    auto choices = [&] {
        if (!bias) {
            // bf16 logits are often equal: the lower half of their bits takes the expert's place in the order.  -0 becomes
            // 0, whose equal it is.
#pragma unroll
            for (int v = 0; v < V; ++v) {
                c[v] = l[v] + 0.0f;
                const uint32_t u = __float_as_uint(c[v]), e = (v / 4 * LPT + sl) * 4 + v % 4;
                if (p.bf16 && l[v] > NONE) c[v] = __uint_as_float(u | (int32_t(u) < 0 ? e : 1023 - e));
            }
            return;
        }
#pragma unroll
        for (int q = 0; q < N; ++q) {
            const int col = (q * LPT + sl) * 4;
            float b[4];
            unpack4(b, E == LPT * V ? load4<true>(bias, 0, col, 4) : load4<false>(bias, 0, col, E - col), 0);
            // 0 l is 0, or NaN where there is no expert; the maximum makes that and a bias's NaN -inf
#pragma unroll
            for (int j = 0; j < 4; ++j)
                c[4 * q + j] = __builtin_fmaxf(__builtin_fmaf(l[4 * q + j], 0.0f, c[4 * q + j] + b[j]), NONE);
        }
    };
    // Twice the error of a choice c in fp32, but for the 2^-24 |c| of its last addition.  Sigmoid: the exponent
    // s (1 - s) (1.3 |l| + 2) 2^-24, the sum and the reciprocal 3 s 2^-24: 3.2 2^-24 at most.  Softmax, of the largest score:
    // the exponential (2.3 |l - most| + 2) 2^-24, its sum 21 additions and the terms' own, 20 on average, and two roundings:
    // 47 2^-24.
    const float slack = by_score ? (sigmoid ? 4.76837158203125e-07f : 7.62939453125e-06f * share) : 0.0f;  // 2^-21, 2^-17

    if (G > 1) {
        const bool plain = top2 && !bias;  // groups by s, not by c
        if (!plain) {
            choices();
#pragma unroll
            for (int q = 0; q < N; ++q) put4(all, q, c);
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v) c[v] = l[v] > NONE ? c[v] : NONE;
        }
        // lanes sl >> shift = g come to hold the two largest of group g, best and second
        float best = NONE, second = NONE;
        if (plain) {
            // by s here, which leaves LDS to the choices behind
#pragma unroll
            for (int q = 0; q < N; ++q) put4(all, q, c);
        }
        wave_sync();
        const int h = 1 << shift, group = sl >> shift;
        if (whole) {
#pragma unroll
            for (int q = 0; q < N; ++q) {
                const float4 r = *reinterpret_cast<const float4*>(all + sl * V + (q + sl) % N * 4);  // other banks than its neighbours
                const float x[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    second = __builtin_amdgcn_fmed3f(best, second, x[j]);
                    best = __builtin_fmaxf(best, x[j]);
                }
            }
        } else if (group < G) {
            // 1 << shift lanes share a group of any size: every so many of its scores each, from a place of its own on
            const float* of = all + group * size;
#pragma unroll 4
            for (int i = sl & (h - 1); i < size; i += h) {
                const float v = of[i];
                second = __builtin_fmaxf(second, __builtin_fminf(best, v));
                best = __builtin_fmaxf(best, v);
            }
        }
        if (h >= 2) top2_step<0xb1>(best, second);   // quad_perm 1 0 3 2
        if (h >= 4) top2_step<0x4e>(best, second);   // quad_perm 2 3 0 1
        if (h >= 8) top2_step<0x141>(best, second);  // row_half_mirror
        if (h >= 16) top2_step<0x140>(best, second);  // row_mirror
        // A group without an expert (none) counts for nothing, whether it is kept or not.  Groups are left open where equal
        // ones make more than top_groups, and where the worst kept and the best other lie within their errors: each
        // the slack, 2^-24 of its terms' sizes and of itself
        const bool two = top2 && second > NONE, none = best == NONE;
        const float value = finite_value(two ? best + second : best);
        const bool keep = (group_larger<LPT>(value, value) >> shift) < p.top_groups && sl >> shift < G;
        kept = __ballot(keep) >> first;  // other tokens' behind
        bool open = (int(group_sum<LPT>(keep && !none ? 1.0f : 0.0f)) >> shift) > p.top_groups;
        if (by_score) {
            const float worst = -group_max<LPT>(keep && !none ? -value : NONE);
            const float next = group_max<LPT>(keep || none ? NONE : value);
            const float sizes = group_max<LPT>(none ? 0.0f : __builtin_fabsf(best) + (two ? __builtin_fabsf(second) : 0.0f));
            const float near = (top2 ? 2.0f : 1.0f) * (slack + 1.1920928955078125e-07f * sizes);
            open |= next > NONE && !(worst - next > near);
        }
        if (plain) {
            choices();
#pragma unroll
            for (int q = 0; q < N; ++q) put4(all, q, c);
        }
        for (uint64_t left = __ballot(open && in); left; left &= ~(TOKEN << (__builtin_ctzll(left) / LPT * LPT))) {
            const int t = __builtin_ctzll(left) / LPT;
            const uint64_t exact = kept_groups(p, r0 + t, shift, lds.by_e);
            if (tok == t) kept = exact;
        }
        // the choices come back from LDS: in registers they would be held beside what fp64 needs
        wave_sync();
#pragma unroll
        for (int q = 0; q < N; ++q) {
            const float4 r = *reinterpret_cast<const float4*>(all + (q * LPT + sl) * 4);
            c[4 * q] = r.x;
            c[4 * q + 1] = r.y;
            c[4 * q + 2] = r.z;
            c[4 * q + 3] = r.w;
        }
        if (whole) {
            const int to = __builtin_ctz(size / 4);  // 4 << to experts a group: of a vector's
#pragma unroll
            for (int q = 0; q < N; ++q) {
                const int g = (q * LPT + sl) >> to << shift;
                const bool k = (LPT == 64 ? uint32_t(kept >> g) : uint32_t(kept) >> g) & 1;
#pragma unroll
                for (int j = 0; j < 4; ++j) c[4 * q + j] = k ? c[4 * q + j] : NONE;
            }
        } else {
            const uint32_t inverse = ((1u << 20) + size - 1) / size;  // e / size = e inverse >> 20 for e < 1024
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const uint32_t g = uint32_t((v / 4 * LPT + sl) * 4 + v % 4) * inverse >> 20;
                c[v] = kept >> (g << shift & 63) & 1 ? c[v] : NONE;
            }
        }
    } else {
        choices();
#pragma unroll
        for (int q = 0; q < N; ++q) put4(all, q, c);
    }
    // candidates: not below the top_k-th largest of the lanes' largest, less the slack; or of their largest two, where lanes
    // are few, or hold the experts of few groups, so that too many are left to be ordered over the lanes (us, 65536 tokens over
    // 256 experts, 4 of 8 groups 34 -> 31, 4 of 16 48 -> 33; where the largest leave less, their two cost 2 to 3 more)
    const float most = finite_value(lane_max(c));
    const int larger = group_larger<LPT>(most, most);
    bool two = LPT < 64 && 2 * K > LPT;
    uint32_t live;
    int n, at;
    for (;;) {
        float bar = larger < K ? -most : NONE;
        if (LPT < 64 && two) {
            float a = NONE, b = NONE;  // the largest, the second
#pragma unroll
            for (int v = 0; v < V; ++v) {
                float x = c[v];
                asm volatile("" : "+v"(x));  // of this branch alone: else the compiler takes part of it into the maximum above
                b = __builtin_amdgcn_fmed3f(a, b, x);
                a = __builtin_fmaxf(a, x);
            }
            b = finite_value(b);
            bar = larger + group_larger<LPT>(most, b) < K ? -most : NONE;
            if (group_larger<LPT>(b, most) + group_larger<LPT>(b, b) < K) bar = -b;  // no more than most
        }
        bar = -group_max<LPT>(bar);
        if (bias) bar -= slack + 4.76837158203125e-07f * __builtin_fabsf(bar);
        bar = __builtin_fmaxf(bar, -3.4028234663852886e38f);  // every expert there is
        live = 0;
#pragma unroll
        for (int v = 0; v < V; ++v) live = push_sign(live, c[v] - bar);
        live = ~live & ((1u << V) - 1);  // bit V - 1 - v: of c[v]
        n = __builtin_popcount(live);
        at = group_before<LPT>(n, sl);
        n = __shfl(at + n, first + LPT - 1);  // of the token
        if (LPT == 64 || two || !__any(n > 2 * LPT)) break;
        two = true;
    }
    const bool redo = n > CAP;  // left to route_token
    if (!redo)
        for (; live; live &= live - 1) {
            const int v = V - 1 - __builtin_ctz(live);
            list[at++] = uint16_t((v / 4 * LPT + sl) * 4 + v % 4);
        }
    int got = redo ? 0 : n;  // candidates of the token, and below the chosen
    int longest = got;
#pragma unroll
    for (int d = LPT; d < 64; d *= 2) longest = max(longest, __shfl_xor(longest, d));
    longest = __builtin_amdgcn_readfirstlane(longest);
    wave_sync();
    // Their order, in fp32 first: a lane has one or two of them where there are no more, and finds its places by counting;
    // where equal ones meet in a place, and where there are more, each counts those before it out of LDS.
    bool counted = false;
    if (LPT < 64 && longest <= LPT) {
        const int e = sl < got ? list[sl] : 0;
        const float x = sl < got ? finite_value(all[e]) : NONE;
        const int before = group_larger<LPT>(x, x);
        counted = !__any(__builtin_popcount(group_or<LPT>(sl < got ? 1u << before : 0)) != got);
        if (counted && sl < got) order[before] = uint16_t(e);
    } else if (LPT < 64 && longest <= 2 * LPT) {
        const bool one = sl < got, two = sl + LPT < got;
        const int e = one ? list[sl] : 0, f = two ? list[sl + LPT] : 0;
        const float x = one ? finite_value(all[e]) : NONE, y = two ? finite_value(all[f]) : NONE;
        const int before = group_larger<LPT>(x, x) + group_larger<LPT>(x, y);
        const int behind = group_larger<LPT>(y, x) + group_larger<LPT>(y, y);
        if constexpr (LPT == 16) {
            const uint32_t places = group_or<LPT>((one ? 1u << before : 0) | (two ? 1u << behind : 0));
            counted = !__any(__builtin_popcount(places) != got);
        } else {
            // more places than bits: their sum is short of 0 + 1 + ... where two meet
            const float places = (one ? float(before) : 0.0f) + (two ? float(behind) : 0.0f);
            counted = !__any(group_sum<LPT>(places) != 0.5f * float(got) * float(got - 1));
        }
        if (counted && one) order[before] = uint16_t(e);
        if (counted && two) order[behind] = uint16_t(f);
    }
    if (!counted) {
        for (int i = sl; i < got; i += LPT) {
            const int e = list[i];
            const float x = all[e];
            int before = 0;
            for (int o = 0; o < got; ++o) {
                const int f = list[o];
                before += all[f] > x || (all[f] == x && f < e);
            }
            order[before] = uint16_t(e);
        }
    }
    wave_sync();
    if (bias) {
        // two neighbours in the order that lie within the slack, and are not of equal logits and biases.  The errors of
        // a softmax's sum and its reciprocal, 43 2^-24, are the same factor in both: of the difference of their scores,
        // which is that of the biases where the choices are close; beside it are 3 2^-24 of the largest score in each.
        bool near = false;
        for (int i = sl; i + 1 < got; i += LPT) {
            const int e = order[i], f = order[i + 1];
            const float x = all[e], y = all[f];
            if (x - y < slack + 2.384185791015625e-07f * __builtin_fabsf(x)) {
                bool open = logit(p, row, e) != logit(p, row, f) || bias[e] != bias[f];
                if (!sigmoid)  // 2^-21, 2^-22, 2^-17
                    open &= x - y < 4.76837158203125e-07f * share + 2.384185791015625e-07f * __builtin_fabsf(x) +
                                        7.62939453125e-06f * __builtin_fabsf(bias[e] - bias[f]);
                near |= open;
            }
        }
        if (__any(near)) {
            // in fp64, in the place of the fp32 choices, with the softmax's sum formed in fp64 too
            if (!sigmoid) {
                double t = 0.0;
#pragma unroll 4
                for (int e = sl; e < E; e += LPT) {
                    const float x = logit(p, row, e);
                    t += x > NONE ? exp(double(x) - double(soft.most)) : 0.0;
                }
#pragma unroll
                for (int d = 1; d < LPT; d *= 2) t += __shfl_xor(t, d);
                soft.sum = t > 0.0 ? t : 1.0;
            }
            double* const exact = reinterpret_cast<double*>(all);
            wave_sync();
            for (int i = sl; i < got; i += LPT) exact[i] = choice(p, logit(p, row, list[i]), list[i], soft);
            wave_sync();
            for (int i = sl; i < got; i += LPT) {
                const double x = exact[i];
                const int e = list[i];
                int before = 0;
                for (int o = 0; o < got; ++o) before += exact[o] > x || (exact[o] == x && list[o] < e);
                order[before] = uint16_t(e);
            }
            wave_sync();
        }
    }
    got = min(got, K);
    // weights of the chosen, a lane each
    const int pick = sl < got ? order[sl] : -1;
    float lg = NONE;
    if (sl < got) {
        const uint32_t u = __float_as_uint(all[pick]);  // without a bias: the logit, with its place if it has one
        lg = bias ? logit(p, row, pick) : __uint_as_float(p.bf16 && (u & 0xffffu) != 0xffffu ? u & 0xffff0000u : u);
    }
    // renormalised from the largest chosen logit, below 0 for sigmoids: shares keep their bits where scores underflow
    const float top = p.renormalise ? group_max<LPT>(lg) : soft.most;
    float w = sigmoid ? sigmoid_part(lg, __builtin_fminf(top, 0.0f)) : expf(lg - top);
    w = sl < got ? w : 0.0f;
    if (p.renormalise || !sigmoid) {
        const float total = p.renormalise ? group_sum<LPT>(w) : z;
        w = sl < got ? w / total : 0.0f;
    }
    uint64_t left = __ballot(redo && in);
    if (in && sl < K && !(left >> first & TOKEN)) {
        p.weights[row * K + sl] = p.scale * w;
        p.ids[row * K + sl] = pick;
    }
    for (; left; left &= ~(TOKEN << (__builtin_ctzll(left) / LPT * LPT))) {
        const int src = __builtin_ctzll(left);
        const uint64_t of = uint64_t(uint32_t(__shfl(int(kept >> 32), src))) << 32 | uint32_t(__shfl(int(kept), src));
        route_token(p, r0 + src / LPT, of, shift, lds.by_e);
    }
}

// v of lane J of every row of 16 (of the LPT lanes of a token).
template <int LPT, int J>
__device__ __forceinline__ int of_lane(int v, int first) {
    if constexpr (LPT == 16) return __builtin_amdgcn_mov_dpp(v, 0x150 + J, 0xf, 0xf, true);  // row_newbcast
    else return __shfl(v, first + J);
}
// The sum of d over the token's entries of this lane's expert, in their order.
template <int LPT, int J = 0>
__device__ __forceinline__ float of_expert(int id, float d, int top_k, int first, float sum = 0.0f) {
    if constexpr (J < LPT) {
        if (J < top_k) {
            const int i = of_lane<LPT, J>(id, first);
            const float x = __int_as_float(of_lane<LPT, J>(__float_as_int(d), first));
            return of_expert<LPT, J + 1>(id, d, top_k, first, i == id ? sum + x : sum);
        }
    }
    return sum;
}

// The gradient for up to 1024 experts: LPT lanes a token, as route_kernel has them.  Lane j of a token has its entry
// j; what the entries give their experts passes through LDS, summed in the entries' order first, so that no atomics
// are needed and an expert may be there twice.  Only the plain softmax reads the other experts' logits: else theirs is
// 0.  65536 x 64 bf16, plain softmax: 8.1 us for 19 MB, 2.3 TB/s, of which the launch and its ends are half
// (a wave a token that looks through its entries for each expert: 88).  65536 x 256 fp32, top 8: plain softmax 28.7 for
// 138 MB, 4.8 TB/s; renormalised, and the sigmoid both ways, 24.4 for 73 MB (the chosen logits alone are read, each in a line
// of its own).  65536 x 8 takes 7.6, x 32 8.1, the instructions of lanes that hold no expert.
template <int LPT, int V>
__global__ __launch_bounds__(256) void route_bwd_kernel(RouteBwdParams p, int64_t row0) {
    constexpr int TPW = 64 / LPT, N = V / 4;
    __shared__ float s_own[4][64 * V];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sl = lane % LPT, tok = lane / LPT, first = tok * LPT;
    const int E = p.n_experts, K = p.top_k;
    const bool sigmoid = p.score != SCORE_SOFTMAX, every = !sigmoid && !p.renormalise;
    const int64_t r0 = (row0 / TPW + int64_t(blockIdx.x) * 4 + wave) * TPW;
    if (r0 >= p.n_tokens) return;
    const bool in = r0 + tok < p.n_tokens;
    const int64_t row = in ? r0 + tok : p.n_tokens - 1;  // lanes behind the last token do it again
    int id = -1;
    float d = 0.0f, lg = NONE;
    if (sl < K) {
        id = p.ids[row * K + sl];
        d = p.scale * p.dweights[row * K + sl];
    }
    float l[V], most = NONE, z = 1.0f;
    if (every) {
        if (E == LPT * V) {
#pragma unroll
            for (int q = 0; q < N; ++q)
                unpack4(l + 4 * q, load4<true>(p.logits, p.bf16, row * E + (q * LPT + sl) * 4, 4), p.bf16);
        } else {
#pragma unroll
            for (int q = 0; q < N; ++q) {
                const int col = (q * LPT + sl) * 4;
                unpack4(l + 4 * q, load4<false>(p.logits, p.bf16, row * E + col, E - col), p.bf16);
#pragma unroll
                for (int j = 0; j < 4; ++j) l[4 * q + j] = j < E - col ? l[4 * q + j] : NONE;
            }
        }
    }
    float* const own = s_own[wave] + tok * (LPT * V);
#pragma unroll
    for (int q = 0; q < N; ++q) *reinterpret_cast<float4*>(own + (q * LPT + sl) * 4) = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    id = id >= 0 && id < E ? id : -1;
    if (id >= 0) lg = clean_logit(load_elem(p.logits, p.bf16, row * E + id));
    id = lg > NONE ? id : -1;  // an expert that is masked takes no part
    d = id >= 0 ? d : 0.0f;
    if (every) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            l[v] = clean_logit(l[v]);
            most = __builtin_fmaxf(most, l[v]);
        }
        most = group_max<LPT>(most);
        most = most > NONE ? most : 0.0f;
        z = 0.0f;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            l[v] = __builtin_amdgcn_exp2f(1.44269504088896341f * (l[v] - most));  // 0 where there is none
            z += l[v];
        }
        z = group_sum<LPT>(z);
        z = z > 0.0f ? z : 1.0f;
    } else if (p.renormalise) {
        most = group_max<LPT>(lg);
    }
    // this entry's share of d; all: what the softmax takes from every expert's
    float s = sigmoid ? sigmoid_part(lg, p.renormalise ? __builtin_fminf(most, 0.0f) : 0.0f) : expf(lg - most), all = 0.0f;
    s = id < 0 ? 0.0f : s;
    const float rest = sigmoid ? sigmoid_part(-lg, 0.0f) : 1.0f;  // 1 - s
    if (p.renormalise) {
        const float total = group_sum<LPT>(s);
        s = id < 0 ? 0.0f : s / total;
        const float mean = group_sum<LPT>(d * s);  // of all lanes: no condition around it
        d = id < 0 ? 0.0f : s * (d - mean) * rest;
    } else if (sigmoid) {
        d = id < 0 ? 0.0f : d * s * rest;
    } else {
        all = group_sum<LPT>(d * (s / z));
    }
    const float sum = of_expert<LPT>(id, d, K, first);
    wave_sync();
    if (id >= 0) own[id] = sum;  // entries of one expert write the same
    wave_sync();
    const float share = 1.0f / z;
#pragma unroll
    for (int q = 0; q < N; ++q) {
        const int col = (q * LPT + sl) * 4;
        const float4 o = *reinterpret_cast<const float4*>(own + col);
        float g[4] = {o.x, o.y, o.z, o.w};
        if (every) {
#pragma unroll
            for (int j = 0; j < 4; ++j) g[j] = l[4 * q + j] * share * (g[j] - all);
        }
        if (!in) continue;
        if (E == LPT * V) store4<true>(p.dlogits, p.d_bf16, row * E + col, 4, g);
        else store4<false>(p.dlogits, p.d_bf16, row * E + col, E - col, g);
    }
}

// The gradient for any number of experts: a wave a token, whose experts look through the entries where any is one of their
// 64 (4096 x 2048 bf16, top 8: 40 us, 15 renormalised; 34 MB are 7 at a copy's rate).
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
        // this entry's part of d, and what is taken from every expert's
        float s = sigmoid ? sigmoid_part(l, p.renormalise ? __builtin_fminf(most, 0.0f) : 0.0f) : expf(l - most), all = 0.0f;
        s = id < 0 ? 0.0f : s;
        if (p.renormalise) {
            const float total = group_sum<64>(s);
            s = id < 0 ? 0.0f : s / total;
            d = s * (d - group_sum<64>(d * s));
        } else if (!sigmoid) {
            all = group_sum<64>(d * (s / sum));
        }
        for (int e = lane; e - lane < E; e += 64) {
            float own = 0.0f;
            const bool any = __any(id >= 0 && id >> 6 == e >> 6);  // an entry of these 64 experts
            for (int j = 0; any && j < K; ++j) {
                const int i = __shfl(id, j);
                const float v = __shfl(d, j);
                if (i == e) own += v;
            }
            if (e >= E) continue;
            float g = 0.0f;
            if (!any && (sigmoid || p.renormalise)) {
                store_elem(p.dlogits, p.d_bf16, row * E + e, 0.0f);
                continue;
            }
            const float v = at(e);
            if (v > NONE) {
                if (sigmoid) {
                    const float rest = sigmoid_part(-v, 0.0f);  // 1 - s
                    g = own == 0.0f ? 0.0f : p.renormalise ? own * rest : own * sigmoid_part(v, 0.0f) * rest;
                } else {
                    g = p.renormalise ? own : expf(v - most) / sum * (own - all);
                }
            }
            store_elem(p.dlogits, p.d_bf16, row * E + e, g);
        }
    }
}

}  // namespace

namespace {

// Calls launch(lanes, experts a lane) for `need` lanes a token at least; false where no kernel holds the token.
template <class F>
bool token_shape(int32_t n_experts, int need, F launch) {
    auto of = [&](auto lpt) {
        using L = decltype(lpt);
        if (n_experts <= 4 * L::value) launch(lpt, std::integral_constant<int, 4>{});
        else if (n_experts <= 8 * L::value) launch(lpt, std::integral_constant<int, 8>{});
        else launch(lpt, std::integral_constant<int, 16>{});
        return true;
    };
    const int lanes = std::max(need, (n_experts + 15) / 16);
    if (lanes <= 16) return of(std::integral_constant<int, 16>{});
    if (lanes <= 32) return of(std::integral_constant<int, 32>{});
    return lanes <= 64 && of(std::integral_constant<int, 64>{});
}

// Launches kernel<<<, 256>>>(p, first token) for `per` tokens a workgroup: a launch holds less than 2^32 threads.
template <class K, class P>
void launch_tokens(K kernel, const P& p, int per, hipStream_t stream) {
    constexpr int64_t most = int64_t(1) << 23;
    for (int64_t row0 = 0; row0 < p.n_tokens; row0 += most * per) {
        const unsigned grid = unsigned(std::min<int64_t>((p.n_tokens - row0 + per - 1) / per, most));
        hipLaunchKernelGGL(kernel, dim3(grid), dim3(256), 0, stream, p, row0);
    }
}

}  // namespace

hipError_t run_route(const RouteParams& args, const DeviceInfo& dev, hipStream_t stream) {
    RouteParams p = args;
    if (p.top_groups == p.n_groups) {  // every group is kept
        p.n_groups = p.top_groups = 1;
        p.group_size = p.n_experts;
    }
    // lanes a token: one at least a pick and a group
    if (token_shape(p.n_experts, std::max(p.top_k, p.n_groups), [&](auto lpt, auto v) {
            launch_tokens(route_kernel<lpt.value, v.value>, p, 256 / lpt.value, stream);
        }))
        return hipGetLastError();
    const unsigned grid = unsigned(std::min<int64_t>(p.n_tokens, 8 * std::max(dev.cu_count, 1)));
    hipLaunchKernelGGL(route_any_kernel, dim3(grid), dim3(ANY), 0, stream, p);
    return hipGetLastError();
}

hipError_t run_route_backward(const RouteBwdParams& p, const DeviceInfo& dev, hipStream_t stream) {
    if (token_shape(p.n_experts, p.top_k, [&](auto lpt, auto v) {
            launch_tokens(route_bwd_kernel<lpt.value, v.value>, p, 256 / lpt.value, stream);
        }))
        return hipGetLastError();
    const unsigned grid = unsigned(std::min<int64_t>((p.n_tokens + 3) / 4, 8 * std::max(dev.cu_count, 1)));
    hipLaunchKernelGGL(route_bwd_any_kernel, dim3(grid), dim3(256), 0, stream, p);
    return hipGetLastError();
}

}  // namespace fff

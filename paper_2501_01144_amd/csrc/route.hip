// The router of a sparse layer and the plan of its experts' products (formulas and arrays in include/dfp4.h).
//
// A wave takes a token: PER experts a lane (expert 64 j + lane).  Choices are by 64-bit keys that order as the scores do, the largest of a
// wave by its upper halves first (DPP) and the lower ones only where several lanes share it, which is all but never.
// Scores are in 64 bits because a choice is a whole number: next to a border fp32 would take another expert than the formula does.
#include "experts.h"

namespace dfp4 {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;

__device__ __forceinline__ float as_f(uint32_t u) { return __builtin_bit_cast(float, u); }

template <int CTRL>
__device__ __forceinline__ uint32_t across(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true); }
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
    v = max(v, across<0xB1>(v));
    v = max(v, across<0x4E>(v));
    v = max(v, across<0x141>(v));
    v = max(v, across<0x140>(v));
    const uint32_t a = max((uint32_t)__builtin_amdgcn_readlane((int)v, 0), (uint32_t)__builtin_amdgcn_readlane((int)v, 16));
    const uint32_t b = max((uint32_t)__builtin_amdgcn_readlane((int)v, 32), (uint32_t)__builtin_amdgcn_readlane((int)v, 48));
    return max(a, b);
}
__device__ __forceinline__ double wave_sum(double v) {
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) v += __shfl_xor(v, x);
    return v;
}

// 64-bit integers that order as the numbers do; 0 is below all, NaN 1
__device__ __forceinline__ uint64_t key_of(double v) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint64_t k = (b >> 63) ? ~b : b | 0x8000000000000000ull;
    return v == v ? k : 1ull;
}
// The largest key of a wave, in all lanes
__device__ __forceinline__ uint64_t wave_max(uint64_t k) {
    const uint32_t hi = wave_max((uint32_t)(k >> 32));
    const uint64_t same = __ballot((uint32_t)(k >> 32) == hi);
    uint32_t lo;
    if (__popcll(same) == 1) lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)k, __ffsll((unsigned long long)same) - 1);
    else lo = wave_max((uint32_t)(k >> 32) == hi ? (uint32_t)k : 0u);
    return (uint64_t)hi << 32 | lo;
}

template <int PER>
__global__ __launch_bounds__(kThreads) void route_kernel(RouteArgs a) {
    __shared__ double s_score[kWaves][64 * PER];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t token = (int64_t)blockIdx.x * kWaves + wave;
    const bool on = token < a.tokens;
    const int E = a.experts;
    double s[PER];
    {
        float x[PER], top = -__builtin_inff();
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int e = 64 * j + lane;
            x[j] = -__builtin_inff();
            if (on && e < E) {
                const int64_t at = token * a.ld + e;
                x[j] = a.bf16 ? as_f((uint32_t)static_cast<const uint16_t*>(a.logits)[at] << 16) : static_cast<const float*>(a.logits)[at];
                x[j] = x[j] == x[j] ? fminf(x[j], 3.402823466e38f) : -__builtin_inff();
            }
            top = fmaxf(top, x[j]);
        }
        if (a.sigmoid) {
#pragma unroll
            for (int j = 0; j < PER; ++j) s[j] = 1.0 / (1.0 + exp(-(double)x[j]));
        } else {
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
            double sum = 0.0;
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                s[j] = top == -__builtin_inff() ? 0.0 : exp((double)x[j] - (double)top);
                sum += s[j];
            }
            sum = wave_sum(sum);
#pragma unroll
            for (int j = 0; j < PER; ++j) s[j] = sum > 0.0 ? s[j] / sum : 0.0;
        }
    }
    uint64_t key[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int e = 64 * j + lane;
        const double c = a.bias && e < E ? s[j] + (double)a.bias[e] : s[j];
        key[j] = e < E ? key_of(c) : 0;
        if (a.groups > 1) s_score[wave][e] = c;
    }
    if (a.groups > 1) {
        __syncthreads();
        // a lane a group
        const int size = E / a.groups;
        double first = -__builtin_inf(), second = -__builtin_inf();
        if (lane < a.groups) {
            for (int i = 0; i < size; ++i) {
                double c = s_score[wave][lane * size + i];
                c = c == c ? c : -__builtin_inf();
                second = fmax(second, fmin(first, c));
                first = fmax(first, c);
            }
        }
        const uint64_t mine = lane < a.groups ? key_of(a.best == 2 ? first + second : first) : 0;
        int better = 0;
        for (int g = 0; g < a.groups; ++g) {
            const uint64_t other = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(mine >> 32), g) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)mine, g);
            better += other > mine || (other == mine && g < lane) ? 1 : 0;
        }
        const uint64_t stays = __ballot(lane < a.groups && better < a.kept);
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int e = 64 * j + lane;
            if (e < E && !((stays >> (e / size)) & 1)) key[j] = 0;
        }
        __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < PER; ++j) s_score[wave][64 * j + lane] = s[j];
    int chosen = 0;                                       // lane j: the j-th
    for (int i = 0; i < a.k; ++i) {
        uint64_t best = key[0];
#pragma unroll
        for (int j = 1; j < PER; ++j) best = best > key[j] ? best : key[j];
        best = wave_max(best);
        // the lowest index that has it
        int e = 0;
#pragma unroll
        for (int j = PER - 1; j >= 0; --j) {
            const uint64_t has = __ballot(key[j] == best);
            if (has) e = 64 * j + __ffsll((unsigned long long)has) - 1;
        }
        if (lane == i) chosen = e;
#pragma unroll
        for (int j = 0; j < PER; ++j)
            if (64 * j + lane == e) key[j] = 0;
    }
    __syncthreads();
    const double mine = lane < a.k ? s_score[wave][chosen] : 0.0;
    double total = 1.0;
    if (a.renormalize) {
        total = 0.0;
        for (int i = 0; i < a.k; ++i) total += __shfl(mine, i);
    }
    if (on && lane < a.k) {
        a.ids[token * a.k + lane] = chosen;
        a.weights[token * a.k + lane] = (float)(total > 0.0 ? mine / total * (double)a.scale : 0.0);
    }
}

// ---- plan

constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64;

// A workgroup an expert.  Each counts all ids (LDS), which gives it its first row and group; a wave then finds the expert's pairs in
// its share of the ids, first how many, then where.
__global__ __launch_bounds__(kPlanThreads) void expert_plan_kernel(const int32_t* __restrict__ ids, PlanView v, int64_t pairs, int experts, int64_t groups) {
    __shared__ uint32_t s_count[kMaxExperts], s_first[kPlanWaves];
    __shared__ uint32_t s_sum[2][kPlanWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int mine = (int)blockIdx.x;
    for (int e = tid; e < experts; e += kPlanThreads) s_count[e] = 0;
    __syncthreads();
    // (whole waves' shares of 64 ids, in order)
    const int64_t per = (pairs + 64 * kPlanWaves - 1) / (64 * kPlanWaves) * 64, lo = wave * per, hi = lo + per < pairs ? lo + per : pairs;
    uint32_t found = 0;
    for (int64_t i0 = lo; i0 < hi; i0 += 64) {
        const int64_t i = i0 + lane;
        const uint32_t id = i < hi ? (uint32_t)ids[i] : 0xffffffffu;
        if (id < (uint32_t)experts) atomicAdd(&s_count[id], 1u);
        else if (mine == 0 && i < hi) v.place[i] = -1;
        found += __popcll(__ballot(id == (uint32_t)mine));
    }
    if (lane == 0) s_first[wave] = found;
    __syncthreads();
    // rows and groups before this expert's, and in all
    auto sums = [&](int end, uint32_t& rows, uint32_t& groups_before) {
        uint32_t r = 0, g = 0;
        for (int e = tid; e < end; e += kPlanThreads) {
            r += s_count[e];
            g += (s_count[e] + kGroupRows - 1) / kGroupRows;
        }
        for (int x = 1; x < 64; x <<= 1) {
            r += __shfl_xor(r, x);
            g += __shfl_xor(g, x);
        }
        __syncthreads();
        if (lane == 0) s_sum[0][wave] = r, s_sum[1][wave] = g;
        __syncthreads();
        rows = groups_before = 0;
        for (int w = 0; w < kPlanWaves; ++w) rows += s_sum[0][w], groups_before += s_sum[1][w];
    };
    uint32_t row0, group0;
    sums(mine, row0, group0);
    const uint32_t count = s_count[mine], my_groups = (count + kGroupRows - 1) / kGroupRows;
    if (tid == 0) {
        v.offsets[mine] = (int32_t)row0;
    }
    for (uint32_t g = tid; g < my_groups; g += kPlanThreads)
        v.groups[group0 + g] = PlanGroup{mine, (int32_t)(row0 + g * kGroupRows), (int32_t)min(count - g * kGroupRows, (uint32_t)kGroupRows), 0};
    for (uint32_t r = tid; r < count; r += kPlanThreads) v.row_at[row0 + r] = (int32_t)(group0 * kGroupRows + r);
    if (mine == experts - 1) {
        const uint32_t rows = row0 + count, used = group0 + my_groups;
        if (tid == 0) {
            v.offsets[experts] = (int32_t)rows;
            *v.used = (int32_t)used;
        }
        for (int64_t g = used + tid; g < groups; g += kPlanThreads) v.groups[g] = PlanGroup{0, 0, 0, 0};
        for (int64_t r = (int64_t)rows + tid; r < pairs; r += kPlanThreads) v.order[r] = v.row_at[r] = -1;
    }
    uint32_t at = row0;
    for (int w = 0; w < wave; ++w) at += s_first[w];
    for (int64_t i0 = lo; i0 < hi; i0 += 64) {
        const int64_t i = i0 + lane;
        const bool is = i < hi && ids[i] == mine;
        const uint64_t all = __ballot(is);
        if (is) {
            const uint32_t row = at + (uint32_t)__popcll(all & ((1ull << lane) - 1));
            v.order[row] = (int32_t)i;
            v.place[i] = (int32_t)row;
        }
        at += (uint32_t)__popcll(all);
    }
}

}  // namespace

int launch_route(const RouteArgs& a, hipStream_t stream) {
    const dim3 grid((uint32_t)((a.tokens + kWaves - 1) / kWaves)), block(kThreads);
    if (a.experts <= 64) hipLaunchKernelGGL((route_kernel<1>), grid, block, 0, stream, a);
    else if (a.experts <= 128) hipLaunchKernelGGL((route_kernel<2>), grid, block, 0, stream, a);
    else if (a.experts <= 256) hipLaunchKernelGGL((route_kernel<4>), grid, block, 0, stream, a);
    else if (a.experts <= 512) hipLaunchKernelGGL((route_kernel<8>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((route_kernel<16>), grid, block, 0, stream, a);
    return check_launch();
}

int launch_expert_plan(const int32_t* ids, const dfp4_plan& p, hipStream_t stream) {
    const int64_t pairs = p.tokens * p.k;
    hipLaunchKernelGGL(expert_plan_kernel, dim3((uint32_t)p.experts), dim3(kPlanThreads), 0, stream, ids, plan_view(p), pairs, (int)p.experts, plan_groups(pairs, p.experts));
    return check_launch();
}

}  // namespace dfp4

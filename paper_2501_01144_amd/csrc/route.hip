// The router of a sparse layer and the plan of its experts' products (formulas and arrays in include/dfp4.h).
//
// A wave takes a token: PER experts a lane (expert 64 j + lane).  Choices are by 32-bit keys that order as the scores do; where several are the largest,
// which for scores in 64 bits is all but never, by the scores themselves.  Scores are in 64 bits because a choice is a whole number: next to a
// border fp32 would take another expert than the formula does.  Without a bias, and where groups go by one score, the order is the logits', and
// only what the weights need is computed.
// Bound by latency (k rounds of a maximum over the wave, each waiting for the one before): 16384 tokens of 8 of 256 18.8 us (with 64-bit keys, all
// scores computed, 25.5); route_logits_kernel 9.2, vector instructions busy 35 % of the time, waves waiting half of theirs.
#include <type_traits>
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

// Integers that order as the numbers do; 0 is below all, NaN 1
__device__ __forceinline__ uint32_t key_of(float v) {
    const uint32_t b = __builtin_bit_cast(uint32_t, v + 0.0f);       // (zeros are alike)
    const uint32_t k = (b >> 31) ? ~b : b | 0x80000000u;
    return v == v ? k : 1u;
}
__device__ __forceinline__ uint64_t key_of(double v) {
    const uint64_t b = __builtin_bit_cast(uint64_t, v + 0.0);
    const uint64_t k = (b >> 63) ? ~b : b | 0x8000000000000000ull;
    return v == v ? k : 1ull;
}
__device__ __forceinline__ uint64_t wave_max(uint64_t k) {
    const uint32_t hi = wave_max((uint32_t)(k >> 32));
    return (uint64_t)hi << 32 | wave_max((uint32_t)(k >> 32) == hi ? (uint32_t)k : 0u);
}

template <int PER>
__global__ __launch_bounds__(kThreads) void route_kernel(RouteArgs a) {
    __shared__ double s_score[kWaves][64 * PER];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t token = (int64_t)blockIdx.x * kWaves + wave;
    const bool on = token < a.tokens;
    const int E = a.experts;
    const bool by_logit = !a.bias && (a.groups == 1 || a.best == 1);
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
    double sum = 1.0;                                     // of softmax
    auto score = [&](float v) { return a.sigmoid ? 1.0 / (1.0 + exp(-(double)v)) : top == -__builtin_inff() ? 0.0 : exp((double)v - (double)top) / sum; };
    if (!a.sigmoid) {
        const uint32_t k = wave_max(key_of(top));
        top = as_f((k >> 31) ? k & 0x7fffffffu : ~k);
        if (!by_logit || !a.renormalize) {
            double t = 0.0;
#pragma unroll
            for (int j = 0; j < PER; ++j) t += score(x[j]);
            t = wave_sum(t);
            sum = t > 0.0 ? t : 1.0;
        }
    }
    // what is chosen by: the logit, or c in 64 bits (in LDS) and its rounding to 32
    uint32_t key[PER];
    if (by_logit) {
#pragma unroll
        for (int j = 0; j < PER; ++j) key[j] = 64 * j + lane < E ? key_of(x[j]) : 0;
    } else {
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const int e = 64 * j + lane;
            double c = score(x[j]);
            if (a.bias && e < E) c += (double)a.bias[e];
            s_score[wave][e] = c;
            key[j] = e < E ? key_of((float)c) : 0;
        }
    }
    if (a.groups > 1) {
        // a lane a group
        const int size = E / a.groups;
        uint64_t mine = 0;
        if (by_logit) {
#pragma unroll
            for (int j = 0; j < PER; ++j) s_score[wave][64 * j + lane] = (double)x[j];
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        if (lane < a.groups) {
            double first = -__builtin_inf(), second = -__builtin_inf();
#pragma unroll 4
            for (int i = 0; i < size; ++i) {
                double c = s_score[wave][lane * size + i];
                c = c == c ? c : -__builtin_inf();
                second = fmax(second, fmin(first, c));
                first = fmax(first, c);
            }
            mine = key_of(a.best == 2 ? first + second : first);
        }
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
    }
    int chosen = 0;                                       // lane j: the j-th, and its logit
    float logit = 0.0f;
    for (int i = 0; i < a.k; ++i) {
        uint32_t m = key[0];
#pragma unroll
        for (int j = 1; j < PER; ++j) m = max(m, key[j]);
        m = wave_max(m);
        int e = 0, several = 0;
#pragma unroll
        for (int j = PER - 1; j >= 0; --j) {
            const uint64_t has = __ballot(key[j] == m);
            several += (int)__popcll(has);
            if (has) e = 64 * j + __ffsll((unsigned long long)has) - 1;         // the lowest
        }
        if (several > 1 && !by_logit) {
            uint64_t best = 0;
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                const uint64_t k = key[j] == m ? key_of(s_score[wave][64 * j + lane]) : 0;
                best = best > k ? best : k;
            }
            best = wave_max(best);
#pragma unroll
            for (int j = PER - 1; j >= 0; --j) {
                const uint64_t has = __ballot(key[j] == m && key_of(s_score[wave][64 * j + lane]) == best);
                if (has) e = 64 * j + __ffsll((unsigned long long)has) - 1;
            }
        }
        float v = 0.0f;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            if (e >> 6 == j) v = x[j];
            if (64 * j + lane == e) key[j] = 0;
        }
        v = as_f((uint32_t)__builtin_amdgcn_readlane(__builtin_bit_cast(int, v), e & 63));
        if (lane == i) chosen = e, logit = v;
    }
    const double mine = lane < a.k ? score(logit) : 0.0;
    double total = 1.0;
    if (a.renormalize) {
        total = 0.0;
        for (int i = 0; i < a.k; ++i) {
            const uint64_t b = __builtin_bit_cast(uint64_t, mine);
            total += __builtin_bit_cast(double, (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(b >> 32), i) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)b, i));
        }
    }
    if (on && lane < a.k) {
        a.ids[token * a.k + lane] = chosen;
        a.weights[token * a.k + lane] = (float)(total > 0.0 ? mine / total * (double)a.scale : 0.0);
    }
}

// The same where the order is the logits', without groups, up to 256 experts and 16 of them: a token has 16 lanes, PER experts in a row each, so that a wave
// takes four and no scalar instruction is in a round.  bf16: a key has the logit above the expert's number, so that no two are alike.
template <int PER, bool BF16>
__global__ __launch_bounds__(kThreads) void route_logits_kernel(RouteArgs a) {
    const int lane = threadIdx.x & 63, l = lane & 15;
    const int64_t token = (int64_t)blockIdx.x * (kThreads / 16) + (threadIdx.x >> 4);
    const bool on = token < a.tokens;
    const int E = a.experts, first = l * PER;
    uint32_t raw[PER];                                    // bits, bf16 in the upper half
    {
        constexpr int kEach = BF16 ? 2 : 4, kVec = PER * kEach < 16 ? PER * kEach : 16;
        const uint8_t* row = static_cast<const uint8_t*>(a.logits) + ((on ? token : 0) * a.ld + first) * kEach;
        if (first + PER <= E) {
            // (rows may begin anywhere)
            uint8_t bytes[PER * kEach];
#pragma unroll
            for (int i = 0; i < PER * kEach; i += kVec) __builtin_memcpy(bytes + i, row + i, kVec);
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                if constexpr (BF16) {
                    uint16_t v;
                    __builtin_memcpy(&v, bytes + 2 * j, 2);
                    raw[j] = (uint32_t)v << 16;
                } else {
                    __builtin_memcpy(&raw[j], bytes + 4 * j, 4);
                }
            }
        } else {
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                raw[j] = 0;
                if (first + j < E) {
                    if constexpr (BF16) raw[j] = (uint32_t)reinterpret_cast<const uint16_t*>(row)[j] << 16;
                    else raw[j] = reinterpret_cast<const uint32_t*>(row)[j];
                }
            }
        }
    }
    // keys; NaN is -infinity, +infinity (f32) the largest number
    uint32_t key[PER];
    float x[PER];
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        x[j] = as_f(raw[j]);
        x[j] = x[j] == x[j] ? x[j] : -__builtin_inff();
        if constexpr (!BF16) x[j] = fminf(x[j], 3.402823466e38f);
        const uint32_t k = key_of(x[j]);
        key[j] = first + j >= E ? 0 : BF16 ? (k & 0xffff0000u) | (uint32_t)(0xffff - (first + j)) : k;
    }
    auto value_of = [](uint32_t k) { return fminf(as_f((k >> 31) ? k & 0x7fffffffu : ~k), 3.402823466e38f); };
    int chosen = 0;                                       // lane i of the 16: the i-th, and its logit
    float logit = -__builtin_inff(), top = 0.0f;
    for (int i = 0; i < a.k; ++i) {
        uint32_t m = key[0];
#pragma unroll
        for (int j = 1; j < PER; ++j) m = max(m, key[j]);
        m = max(m, across<0xB1>(m));
        m = max(m, across<0x4E>(m));
        m = max(m, across<0x141>(m));
        m = max(m, across<0x140>(m));
        int e;
        float v;
        if constexpr (BF16) {
            e = 0xffff - (int)(m & 0xffffu);
            // (the lower half of a negative number's key is ones)
            v = value_of((m >> 31) ? m & 0xffff0000u : m | 0xffffu);
#pragma unroll
            for (int j = 0; j < PER; ++j) key[j] = key[j] == m ? 0 : key[j];
        } else {
            uint32_t at = 0xffff;                         // the lowest of those that have it
#pragma unroll
            for (int j = PER - 1; j >= 0; --j) at = key[j] == m ? (uint32_t)(first + j) : at;
            uint32_t low = at;
            low = min(low, across<0xB1>(low));
            low = min(low, across<0x4E>(low));
            low = min(low, across<0x141>(low));
            low = min(low, across<0x140>(low));
            e = (int)low;
            v = value_of(m);
#pragma unroll
            for (int j = 0; j < PER; ++j) key[j] = (uint32_t)(first + j) == low ? 0 : key[j];
        }
        if (i == 0) top = v;
        if (l == i) chosen = e, logit = v;
    }
    auto sum16 = [](double t) {
#pragma unroll
        for (int d = 1; d < 16; d <<= 1) t += __shfl_xor(t, d);
        return t;
    };
    double sum = 1.0;                                     // of softmax
    auto score = [&](float v) { return a.sigmoid ? 1.0 / (1.0 + exp(-(double)v)) : top == -__builtin_inff() ? 0.0 : exp((double)v - (double)top) / sum; };
    if (!a.sigmoid && !a.renormalize) {
        double t = 0.0;
#pragma unroll
        for (int j = 0; j < PER; ++j) t += first + j < E ? score(fminf(x[j], 3.402823466e38f)) : 0.0;
        t = sum16(t);
        sum = t > 0.0 ? t : 1.0;
    }
    const double mine = l < a.k ? score(logit) : 0.0, total = a.renormalize ? sum16(mine) : 1.0;
    if (on && l < a.k) {
        a.ids[token * a.k + l] = chosen;
        a.weights[token * a.k + l] = (float)(total > 0.0 ? mine / total * (double)a.scale : 0.0);
    }
}

// ---- plan

constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64;

// sums over the lanes up to each
__device__ __forceinline__ uint32_t wave_scan(uint32_t v) {
    auto add = [&](auto ctrl, auto rows) { v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, decltype(rows)::value, 0xf, false); };
    using std::integral_constant;
    add(integral_constant<int, 0x111>{}, integral_constant<int, 0xf>{});      // from 1, 2, 4, 8 lanes before, within 16
    add(integral_constant<int, 0x112>{}, integral_constant<int, 0xf>{});
    add(integral_constant<int, 0x114>{}, integral_constant<int, 0xf>{});
    add(integral_constant<int, 0x118>{}, integral_constant<int, 0xf>{});
    add(integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});      // the last lane of 16 to the 16 after it, of 32 to the other 32
    add(integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});
    return v;
}

constexpr int64_t kRecount = 16384;                                 // pairs up to which every workgroup counts all, which spares a launch

// entries of one of the plan's lists, every `by`-th
constexpr uint32_t kListSerial = 512;                               // rows of an expert up to which one thread writes them
__device__ __forceinline__ void list_entries(PlanGroup* to, int list, int expert, uint32_t row0, uint32_t total, uint32_t group0, uint32_t from, uint32_t by) {
    const uint32_t rows = list == 0 ? kListRows[0] : list == 1 ? kListRows[1] : kListRows[2], n = (total + rows - 1) / rows;
    for (uint32_t g = from; g < n; g += by)
        to[g] = PlanGroup{expert, (int32_t)(row0 + g * rows), (int32_t)min(total - g * rows, rows), (int32_t)(group0 * kGroupRows + g * rows)};
}

// A stable counting sort, bound by latency: 131072 pairs of 256 experts 2.8 + 9.3 us (a workgroup an expert, each looking at all ids: 76); a few pairs
// 3 to 5.  A workgroup takes a share of the pairs, 16 waves in turn; where there are several, each counts all pairs, or a first
// kernel has counted each share's experts.  Every workgroup knows all counts then, and with them each expert's first row and its entries of the lists; a wave ranks its pairs 64 at
// a time by comparing bits of their experts.
__global__ __launch_bounds__(kPlanThreads) void expert_count_kernel(const int32_t* __restrict__ ids, int32_t* counts, int64_t pairs, int64_t share, int experts) {
    __shared__ int32_t s_count[kMaxExperts];
    for (int e = threadIdx.x; e < experts; e += kPlanThreads) s_count[e] = 0;
    __syncthreads();
    const int64_t lo = blockIdx.x * share, hi = min(pairs, lo + share);
    for (int64_t i = lo + threadIdx.x; i < hi; i += kPlanThreads) {
        const uint32_t id = (uint32_t)ids[i];
        if (id < (uint32_t)experts) atomicAdd(&s_count[id], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < experts; e += kPlanThreads) counts[(int64_t)blockIdx.x * experts + e] = s_count[e];
}

__global__ __launch_bounds__(kPlanThreads) void expert_plan_kernel(const int32_t* __restrict__ ids, PlanView v, int64_t pairs, int64_t share, int experts, int bits, int64_t most_blocks) {
    __shared__ uint32_t s_at[kPlanWaves][kMaxExperts];               // of a wave's pairs: how many, then the next row
    __shared__ uint32_t s_row[kMaxExperts], s_group[kMaxExperts], s_total[kMaxExperts], s_list[3][kMaxExperts];
    __shared__ uint4 s_sum[kPlanWaves];
    __shared__ uint32_t s_rows, s_blocks;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t lo = blockIdx.x * share, hi = min(pairs, lo + share);
    // (a wave's part of the share: whole rounds of 64)
    const int64_t per = share / kPlanWaves, wlo = min(hi, lo + wave * per), whi = min(hi, wlo + per);
    for (int w = 0; w < kPlanWaves; ++w)
        if (tid < experts) s_at[w][tid] = 0;
    if (tid < experts) s_total[tid] = s_list[0][tid] = 0;
    __syncthreads();
    if (gridDim.x > 1 && pairs <= kRecount) {
#pragma unroll 4
        for (int i = tid; i < (int)pairs; i += kPlanThreads) {
            const uint32_t id = (uint32_t)ids[i];
            if (id < (uint32_t)experts) {
                atomicAdd(&s_total[id], 1u);
                if (i < lo) atomicAdd(&s_list[0][id], 1u);
            }
        }
    }
    for (int64_t i = wlo + lane; i < whi; i += 64) {
        const uint32_t id = (uint32_t)ids[i];
        if (id < (uint32_t)experts) atomicAdd(&s_at[wave][id], 1u);
    }
    __syncthreads();
    // a thread an expert: pairs in all, and in the shares before
    const int e = tid;
    uint32_t total = 0, before = 0;
    if (e < experts) {
        if (gridDim.x > 1 && pairs <= kRecount) {
            total = s_total[e];
            before = s_list[0][e];
        } else if (gridDim.x > 1) {
#pragma unroll 16
            for (int b = 0; b < (int)gridDim.x; ++b) {
                const uint32_t n = (uint32_t)v.counts[(int64_t)b * experts + e];
                total += n;
                before += b < (int)blockIdx.x ? n : 0;
            }
        } else {
            for (int w = 0; w < kPlanWaves; ++w) total += s_at[w][e];
        }
    }
    uint32_t sum[4] = {total};                                       // of the experts up to this one: rows, entries of the lists
    uint32_t entries[3];
#pragma unroll
    for (int q = 0; q < 3; ++q) sum[q + 1] = entries[q] = (total + kListRows[q] - 1) / kListRows[q];
#pragma unroll
    for (int q = 0; q < 4; ++q) sum[q] = wave_scan(sum[q]);
    if (lane == 63) s_sum[wave] = make_uint4(sum[0], sum[1], sum[2], sum[3]);
    __syncthreads();
    for (int w = 0; w < (experts + 63) / 64; ++w) {
        const uint4 v = s_sum[w];
        if (w < wave) sum[0] += v.x, sum[1] += v.y, sum[2] += v.z, sum[3] += v.w;
    }
    if (e < experts) {
        const uint32_t row0 = sum[0] - total, group0 = sum[1] - entries[0];
        s_total[e] = total;
#pragma unroll
        for (int q = 0; q < 3; ++q) s_list[q][e] = sum[q + 1] - entries[q];
        s_row[e] = row0;
        s_group[e] = group0;
        uint32_t at = row0 + before;
        for (int w = 0; w < kPlanWaves; ++w) {
            const uint32_t n = s_at[w][e];
            s_at[w][e] = at;
            at += n;
        }
        if (e % (int)gridDim.x == (int)blockIdx.x) {                 // described by one of the workgroups
            v.offsets[e] = (int32_t)row0;
#pragma unroll
            for (int q = 0; q < 3; ++q) {
                if (total <= kListSerial) list_entries(v.list[q] + (sum[q + 1] - entries[q]), q, e, row0, total, group0, 0, 1);
                if (e == experts - 1) v.used[q] = (int32_t)sum[q + 1];
            }
            if (e == experts - 1) v.offsets[experts] = (int32_t)sum[0];
        }
        if (e == experts - 1) s_rows = sum[0], s_blocks = sum[3];
    }
    __syncthreads();
    // (experts of many rows: a wave each)
    for (int x = (int)blockIdx.x + (int)gridDim.x * wave; x < experts; x += (int)gridDim.x * kPlanWaves)
        if (s_total[x] > kListSerial)
            for (int q = 0; q < 3; ++q) list_entries(v.list[q] + s_list[q][x], q, x, s_row[x], s_total[x], s_group[x], lane, 64);
    for (int64_t i4 = wlo; i4 < whi; i4 += 256) {
        uint32_t next[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) next[q] = i4 + 64 * q + lane < whi ? (uint32_t)ids[i4 + 64 * q + lane] : 0xffffffffu;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (i4 + 64 * q >= whi) break;
            const int64_t i = i4 + 64 * q + lane;
            const uint32_t id = next[q];
            const bool is = id < (uint32_t)experts;
            uint64_t same = __ballot(is);
            for (int b = 0; b < bits; ++b) {
                const uint64_t set = __ballot((id >> b) & 1);
                same &= (id >> b) & 1 ? set : ~set;
            }
            if (i < whi) v.expert[i] = is ? (int32_t)id : -1;
            if (is) {
                const uint32_t row = s_at[wave][id] + (uint32_t)__popcll(same & ((1ull << lane) - 1));
                v.order[row] = (int32_t)i;
                v.row_at[row] = (int32_t)(s_group[id] * kGroupRows + row - s_row[id]);
                v.place[i] = (int32_t)row;
            } else if (i < whi) {
                v.place[i] = -1;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (is && (same >> lane) == 1) s_at[wave][id] += (uint32_t)__popcll(same);  // the last of them
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
    }
    if (blockIdx.x == 0)                                             // (as many as there can be are looked at where there is one token)
        for (int64_t g = s_blocks + tid; g < most_blocks; g += kPlanThreads) v.list[2][g] = PlanGroup{0, 0, 0, 0};
    // rows that no pair has
    for (int64_t r = s_rows + (int64_t)blockIdx.x * kPlanThreads + tid; r < pairs; r += (int64_t)gridDim.x * kPlanThreads) v.order[r] = -1;
}

}  // namespace

int launch_route(const RouteArgs& a, hipStream_t stream) {
    if (!a.bias && a.groups == 1 && a.experts <= 256 && a.k <= 16) {
        const dim3 by16((uint32_t)((a.tokens + kThreads / 16 - 1) / (kThreads / 16)));
        auto run = [&](auto per) {
            if (a.bf16) hipLaunchKernelGGL((route_logits_kernel<decltype(per)::value, true>), by16, dim3(kThreads), 0, stream, a);
            else hipLaunchKernelGGL((route_logits_kernel<decltype(per)::value, false>), by16, dim3(kThreads), 0, stream, a);
        };
        if (a.experts <= 16) run(std::integral_constant<int, 1>{});
        else if (a.experts <= 32) run(std::integral_constant<int, 2>{});
        else if (a.experts <= 64) run(std::integral_constant<int, 4>{});
        else if (a.experts <= 128) run(std::integral_constant<int, 8>{});
        else run(std::integral_constant<int, 16>{});
        return check_launch();
    }
    const dim3 grid((uint32_t)((a.tokens + kWaves - 1) / kWaves)), block(kThreads);
    if (a.experts <= 64) hipLaunchKernelGGL((route_kernel<1>), grid, block, 0, stream, a);
    else if (a.experts <= 128) hipLaunchKernelGGL((route_kernel<2>), grid, block, 0, stream, a);
    else if (a.experts <= 256) hipLaunchKernelGGL((route_kernel<4>), grid, block, 0, stream, a);
    else if (a.experts <= 512) hipLaunchKernelGGL((route_kernel<8>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((route_kernel<16>), grid, block, 0, stream, a);
    return check_launch();
}

int launch_expert_plan(const int32_t* ids, const dfp4_plan& p, hipStream_t stream) {
    const int64_t pairs = p.tokens * p.k, share = plan_share(pairs), shares = plan_shares(pairs);
    const PlanView v = plan_view(p);
    int bits = 0;
    while ((1 << bits) < p.experts) ++bits;
    if (shares > 1 && pairs > kRecount) hipLaunchKernelGGL(expert_count_kernel, dim3((uint32_t)shares), dim3(kPlanThreads), 0, stream, ids, v.counts, pairs, share, (int)p.experts);
    hipLaunchKernelGGL(expert_plan_kernel, dim3((uint32_t)shares), dim3(kPlanThreads), 0, stream, ids, v, pairs, share, (int)p.experts, bits,
                       p.tokens == 1 ? plan_list(pairs, p.experts, 2) : 0);
    return check_launch();
}

}  // namespace dfp4

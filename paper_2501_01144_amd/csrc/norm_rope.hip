// Norms of queries and keys per head and their rotation by position, in one pass (formulas in include/dfp4.h).
//
// Bound by memory: 4 bytes an element.  A head is head_dim / 8 lanes of eight elements, rounded up to a power of two for the sum of
// squares (within a row of 16 lanes by DPP).  A lane has both elements of its pairs: with pairs rotary / 2 apart 4 + 4 elements (8 bytes
// a load, so that nothing moves between lanes), else eight in a row.  Its place in a head, and so its cosines and weights, are the same
// for all heads: they are in registers.  A workgroup takes as many tokens as it has threads for their cosines and sines, which it
// computes at once and hands over in LDS, and a share of their heads: all where there are many tokens, 16 where there are few.
// 8192 tokens, 32 + 8 heads of 128 (168 MB) 42 us = 4.0 TB/s (a copy: 5.2).  One token a workgroup, pairs exchanged by shuffles and
// cosines read for every head took 96; loads one head ahead, ending with each token, 58.
#include "paged.h"

namespace dfp4 {

namespace {

constexpr int kThreads = 256;

typedef __bf16 v4b __attribute__((ext_vector_type(4)));

__device__ __forceinline__ float as_f(uint32_t u) { return __builtin_bit_cast(float, u); }

template <int CTRL>
__device__ __forceinline__ float across(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
// sum over LANES neighbouring lanes: neighbours 1 and 2 apart, then mirrored in 8 and in 16 lanes, then 16 apart
template <uint32_t LANES>
__device__ __forceinline__ float head_sum(float v) {
    v += across<0xB1>(v);
    v += across<0x4E>(v);
    if constexpr (LANES >= 8) v += across<0x141>(v);
    if constexpr (LANES >= 16) v += across<0x140>(v);
    if constexpr (LANES >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
        v = as_f(r[0]) + as_f(r[1]);
    }
    return v;
}

struct Launch {
    NormRopeArgs a;
    int tokens, passes;          // tokens of a workgroup; heads of a token: passes * kThreads / LANES
};

template <uint32_t LANES>                                            // of a head
__global__ __launch_bounds__(kThreads) void norm_rope_kernel(Launch p) {
    const NormRopeArgs& a = p.a;
    __shared__ __attribute__((aligned(16))) float s_cos[kThreads], s_sin[kThreads];      // [token][pair]
    constexpr int kHeads = kThreads / (int)LANES;                    // at a time
    const uint32_t tid = threadIdx.x, sub = tid % LANES, half = (uint32_t)a.rotary / 2u;
    const int t0 = (int)blockIdx.x * p.tokens, tokens = min(p.tokens, a.tokens - t0);
    if (tid < (uint32_t)tokens * half) {
        // the angle in turns, in 64 bits: a position of 2^20 and a frequency of 1 leave 32 of their bits to the fraction
        const double turns = (double)a.positions[t0 + (int)(tid / half)] * (double)a.inv_freq[tid % half] * 0.15915494309189533577;
        sincospif(2.0f * (float)(turns - rint(turns)), &s_sin[tid], &s_cos[tid]);
    }
    // the lane's elements: d0 .. d0 + 3 and d1 .. d1 + 3
    const bool in = sub * 8u < (uint32_t)a.head_dim, turn = a.interleaved ? sub * 8u < (uint32_t)a.rotary : sub * 4u < half;
    const uint32_t d0 = !in ? 0u : !a.interleaved && turn ? sub * 4u : sub * 8u, d1 = !in ? 4u : !a.interleaved && turn ? d0 + half : d0 + 4u;
    float wq[8], wk[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t d = (j < 4 ? d0 : d1 - 4u) + j;
        wq[j] = a.q_weight ? a.q_weight[d] : 1.0f;
        wk[j] = a.k_weight ? a.k_weight[d] : 1.0f;
    }
    __syncthreads();
    const int heads = a.heads + a.kv_heads, first = (int)blockIdx.y * p.passes * kHeads + (int)(tid / LANES), end = min(heads, first + p.passes * kHeads);
    const float per = 1.0f / (float)a.head_dim;
    // two heads ahead, over all heads of all tokens
    uint2 next[2][2] = {};
    int load_n = 0, load_h = first;
    auto load = [&](uint2 (&to)[2]) {
        if (in && load_n < tokens && load_h < end) {
            const int64_t t = t0 + load_n;
            const uint16_t* from = load_h < a.heads ? a.q + t * a.q_stride + (int64_t)load_h * a.q_head_stride
                                                    : a.k + t * a.k_stride + (int64_t)(load_h - a.heads) * a.k_head_stride;
            to[0] = *reinterpret_cast<const uint2*>(from + d0);
            to[1] = *reinterpret_cast<const uint2*>(from + d1);
        }
        load_h += kHeads;
        if (load_h - first == p.passes * kHeads) load_h = first, ++load_n;
    };
    load(next[0]);
    load(next[1]);
    for (int n = 0; n < tokens; ++n) {
        const int64_t t = t0 + n;
        float c[4] = {1, 1, 1, 1}, s[4] = {0, 0, 0, 0};              // pair by pair (interleaved: elements 2 j, 2 j + 1)
        if (turn) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                c[j] = s_cos[n * half + sub * 4u + j];
                s[j] = s_sin[n * half + sub * 4u + j];
            }
        }
        for (int i = 0; i < p.passes; ++i) {
            const int h = first + i * kHeads;
            const uint32_t u[4] = {next[0][0].x, next[0][0].y, next[0][1].x, next[0][1].y};
            next[0][0] = next[1][0];
            next[0][1] = next[1][1];
            load(next[1]);
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = as_f((j & 1) ? u[j / 2] & 0xffff0000u : u[j / 2] << 16);
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) sum += x[j] * x[j];
            const bool is_q = h < a.heads;
            if (is_q ? a.q_weight != nullptr : a.k_weight != nullptr) {
                // (lanes of a head that are beyond head_dim hold zeros)
                float mean = head_sum<LANES>(sum) * per + a.eps;
                if (__any(mean < 0x1p-100f || mean == __builtin_inff())) {
                    // squares beyond the range of fp32 (from |x| of about 2^60 on, or below 2^-50 with as small an eps): of numbers
                    // scaled by a power of two
                    const float by = mean == __builtin_inff() ? 0x1p-70f : mean < 0x1p-100f ? 0x1p100f : 1.0f;
                    sum = 0.0f;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        x[j] *= by;
                        sum += x[j] * x[j];
                    }
                    mean = head_sum<LANES>(sum) * per + a.eps * by * by;
                }
                const float r = __builtin_amdgcn_rsqf(mean);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] *= r * (is_q ? wq[j] : wk[j]);
            }
            float y[8];
            if (a.interleaved) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    y[2 * j] = x[2 * j] * c[j] - x[2 * j + 1] * s[j];
                    y[2 * j + 1] = x[2 * j + 1] * c[j] + x[2 * j] * s[j];
                }
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    y[j] = x[j] * c[j] - x[4 + j] * s[j];
                    y[4 + j] = x[4 + j] * c[j] + x[j] * s[j];
                }
            }
            if (in && h < end) {
                uint16_t* dst = is_q ? a.q_out + (t * a.heads + h) * a.head_dim : a.k_out + (t * a.kv_heads + (h - a.heads)) * a.head_dim;
                v4b o[2];
#pragma unroll
                for (int j = 0; j < 8; ++j) o[j / 4][j % 4] = (__bf16)y[j];
                *reinterpret_cast<v4b*>(dst + d0) = o[0];
                *reinterpret_cast<v4b*>(dst + d1) = o[1];
            }
        }
    }
}

}  // namespace

int launch_norm_rope(const NormRopeArgs& a, hipStream_t stream) {
    const int lanes = a.head_dim <= 32 ? 4 : a.head_dim <= 64 ? 8 : a.head_dim <= 128 ? 16 : 32, at_once = kThreads / lanes;
    const int rounds = (a.heads + a.kv_heads + at_once - 1) / at_once, fit = a.rotary > 0 ? kThreads / (a.rotary / 2) : 4;
    const int cus = device_cu_count();
    // As many tokens a workgroup as leave four workgroups to a compute unit; with fewer workgroups than that a pass of heads to each
    // (one token, 40 heads: three workgroups, 3.3 us of kernel; all heads in one 6.2).
    int tokens = a.tokens / (4 * cus);
    tokens = tokens < 1 ? 1 : tokens < fit ? tokens : fit;
    const int64_t groups = ((int64_t)a.tokens + tokens - 1) / tokens;
    const int passes = groups >= 4 * cus ? rounds : 1;
    const int64_t most = ((int64_t)1 << 32) / kThreads - 1;          // workgroups of a launch: fewer than 2^32 threads
    for (int64_t at = 0; at < groups; at += most) {
        const int64_t t = at * tokens, left = groups - at < most ? groups - at : most;
        Launch p{a, tokens, passes};
        p.a.tokens = (int)(a.tokens - t < left * tokens ? a.tokens - t : left * tokens);
        p.a.q += t * a.q_stride, p.a.k += t * a.k_stride, p.a.positions += t;
        p.a.q_out += t * a.heads * a.head_dim, p.a.k_out += t * a.kv_heads * a.head_dim;
        const dim3 grid((uint32_t)left, (uint32_t)((rounds + passes - 1) / passes)), block(kThreads);
        if (lanes == 4) hipLaunchKernelGGL((norm_rope_kernel<4>), grid, block, 0, stream, p);
        else if (lanes == 8) hipLaunchKernelGGL((norm_rope_kernel<8>), grid, block, 0, stream, p);
        else if (lanes == 16) hipLaunchKernelGGL((norm_rope_kernel<16>), grid, block, 0, stream, p);
        else hipLaunchKernelGGL((norm_rope_kernel<32>), grid, block, 0, stream, p);
    }
    return check_launch();
}

}  // namespace dfp4

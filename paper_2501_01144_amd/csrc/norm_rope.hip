// Norms of queries and keys per head and their rotation by position, in one pass (formulas in include/dfp4.h).
//
// A head is head_dim / 8 lanes of 8 elements (16 bytes), rounded up to a power of two for the sum of squares.  A workgroup takes
// one token; its cosines and sines, alike for all heads, are computed once and kept in LDS.  Bound by memory: 4 bytes an element.
#include "paged.h"

namespace dfp4 {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float as_f(uint32_t u) { return __builtin_bit_cast(float, u); }
__device__ __forceinline__ uint32_t bf16_bits(float x) {             // round to nearest even; the inputs are finite
    const uint32_t u = __builtin_bit_cast(uint32_t, x);
    return (u + 0x7fffu + ((u >> 16) & 1u)) >> 16;
}

template <uint32_t LANES>                                            // of a head
__global__ __launch_bounds__(kThreads) void norm_rope_kernel(NormRopeArgs a) {
    __shared__ float s_cos[128], s_sin[128];
    const uint32_t tid = threadIdx.x, sub = tid % LANES, half = (uint32_t)a.rotary / 2u;
    const int t = (int)blockIdx.x;
    for (uint32_t j = tid; j < half; j += kThreads) {
        // the angle in turns, in 64 bits: a position of 2^20 and a frequency of 1 leave 32 of their bits to the fraction
        const double turns = (double)a.positions[t] * (double)a.inv_freq[j] * 0.15915494309189533577;
        const float frac = (float)(turns - rint(turns));
        sincospif(2.0f * frac, &s_sin[j], &s_cos[j]);
    }
    __syncthreads();
    const uint32_t d0 = sub * 8u;
    const bool in = d0 < (uint32_t)a.head_dim;
    const int heads = a.heads + a.kv_heads;
    for (int h = (int)(tid / LANES); h < (heads + (int)(kThreads / LANES) - 1) / (int)(kThreads / LANES) * (int)(kThreads / LANES); h += (int)(kThreads / LANES)) {
        const bool is_q = h < a.heads, on = in && h < heads;
        const uint16_t* src = is_q ? a.q + (int64_t)t * a.q_stride + (int64_t)h * a.q_head_stride
                                   : a.k + (int64_t)t * a.k_stride + (int64_t)(h - a.heads) * a.k_head_stride;
        const float* w = is_q ? a.q_weight : a.k_weight;
        uint4 raw = make_uint4(0, 0, 0, 0);
        if (on) raw = *reinterpret_cast<const uint4*>(src + d0);
        const uint32_t u[4] = {raw.x, raw.y, raw.z, raw.w};
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = as_f((j & 1) ? u[j / 2] & 0xffff0000u : u[j / 2] << 16);
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += x[j] * x[j];
#pragma unroll
        for (uint32_t m = 1; m < LANES; m *= 2) sum += __shfl_xor(sum, (int)m);
        if (w) {
            const float r = 1.0f / sqrtf(sum / (float)a.head_dim + a.eps);
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] *= r * (in ? w[d0 + j] : 0.0f);
        }
        float y[8];
        if (a.interleaved) {
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const uint32_t p = (d0 + j) / 2u;
                const bool turn = d0 + j < (uint32_t)a.rotary;
                const float c = turn ? s_cos[p] : 1.0f, s = turn ? s_sin[p] : 0.0f;
                y[j] = x[j] * c - x[j + 1] * s;
                y[j + 1] = x[j + 1] * c + x[j] * s;
            }
        } else {
            // the other element of a pair lies half / 8 lanes on or back (rotary is a multiple of 16)
            const bool turn = d0 < (uint32_t)a.rotary, upper = d0 >= half;
            const uint32_t lane = tid & 63u, other = turn ? (upper ? lane - half / 8u : lane + half / 8u) : lane;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float o = __shfl(x[j], (int)other);
                const uint32_t p = turn ? d0 + j - (upper ? half : 0u) : 0u;
                const float c = turn ? s_cos[p] : 1.0f, s = turn ? s_sin[p] : 0.0f;
                y[j] = x[j] * c + (upper ? o * s : -o * s);
            }
        }
        if (on) {
            uint32_t o[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] = bf16_bits(y[2 * j]) | (bf16_bits(y[2 * j + 1]) << 16);
            uint16_t* dst = is_q ? a.q_out + ((int64_t)t * a.heads + h) * a.head_dim : a.k_out + ((int64_t)t * a.kv_heads + (h - a.heads)) * a.head_dim;
            *reinterpret_cast<uint4*>(dst + d0) = make_uint4(o[0], o[1], o[2], o[3]);
        }
    }
}

}  // namespace

int launch_norm_rope(const NormRopeArgs& a, hipStream_t stream) {
    const dim3 grid((uint32_t)a.tokens), block(kThreads);
    if (a.head_dim <= 32) hipLaunchKernelGGL((norm_rope_kernel<4>), grid, block, 0, stream, a);
    else if (a.head_dim <= 64) hipLaunchKernelGGL((norm_rope_kernel<8>), grid, block, 0, stream, a);
    else if (a.head_dim <= 128) hipLaunchKernelGGL((norm_rope_kernel<16>), grid, block, 0, stream, a);
    else hipLaunchKernelGGL((norm_rope_kernel<32>), grid, block, 0, stream, a);
    return check_launch();
}

}  // namespace dfp4

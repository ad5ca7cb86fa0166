// Norms before and after a block with its gate and the residual, in one pass (formulas in include/dfp4.h).
//
// Bound by memory: 8 bytes an element (bf16 residual, no gate).  A row stays in registers between the two sums: eight elements a lane and
// pass, a workgroup (or, up to 512 elements, a wave) a row.  8192 x 4096 (268 MB) 51 us = 5.2 TB/s, what a large copy reaches; the kernel alone 40, its
// outputs then in the last cache.
#include "experts.h"

namespace dfp4 {

namespace {

typedef __bf16 v8b __attribute__((ext_vector_type(8)));

__device__ __forceinline__ float as_f(uint32_t u) { return __builtin_bit_cast(float, u); }
template <int CTRL>
__device__ __forceinline__ float across(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
__device__ __forceinline__ float lane_of(float v, int lane) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}
__device__ __forceinline__ float wave_sum(float v) {
    v += across<0xB1>(v);
    v += across<0x4E>(v);
    v += across<0x141>(v);
    v += across<0x140>(v);
    return (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
}

template <int WAVES>
__device__ __forceinline__ float row_sum(float v, float* s) {
    v = wave_sum(v);
    if constexpr (WAVES > 1) {
        __syncthreads();                                 // what was read of `s` before is done with
        if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
        __syncthreads();
        v = s[0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v += s[w];
    }
    return v;
}

__device__ __forceinline__ void widen(uint4 u, float (&x)[8]) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = as_f((j & 1) ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
}

// x -> x / sqrt(mean(x^2) + eps) in the row's registers
template <int WAVES, int PASSES>
__device__ __forceinline__ void normalize(float (&x)[PASSES][8], float per, float eps, float* s) {
    auto sum = [&] {
        float t = 0.0f;
#pragma unroll
        for (int i = 0; i < PASSES; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) t += x[i][j] * x[i][j];
        return row_sum<WAVES>(t, s);
    };
    float mean = sum() * per + eps;
    if (mean < 0x1p-100f || mean == __builtin_inff()) {  // (the same for the whole row)
        // squares beyond the range of fp32: of numbers scaled by a power of two, below 2^48 then, so that 2^14 squares have a sum
        const float by = mean == __builtin_inff() ? 0x1p-80f : 0x1p100f;
#pragma unroll
        for (int i = 0; i < PASSES; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) x[i][j] *= by;
        mean = sum() * per + eps * by * by;
    }
    const float r = __builtin_amdgcn_rsqf(mean);
#pragma unroll
    for (int i = 0; i < PASSES; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) x[i][j] *= r;
}

// WAVES of a row: 1 (four rows a workgroup) or 4
template <int WAVES, int PASSES, bool WIDE>
__global__ __launch_bounds__(256) void add_norm_kernel(AddNormArgs a) {
    __shared__ float s_sum[4];
    constexpr int kThreads = 64 * WAVES;
    const int sub = threadIdx.x % kThreads;
    const int64_t row = (int64_t)blockIdx.x * (256 / kThreads) + threadIdx.x / kThreads;
    if (WAVES == 1 && row >= a.tokens) return;
    const float per = 1.0f / (float)a.dim;
    float z[PASSES][8];
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int d = (i * kThreads + sub) * 8;
        widen(d < a.dim ? *reinterpret_cast<const uint4*>(a.y + row * a.y_ld + d) : make_uint4(0, 0, 0, 0), z[i]);
    }
    float r[PASSES][8];
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int d = (i * kThreads + sub) * 8;
        if constexpr (WIDE) {
            const float4* from = reinterpret_cast<const float4*>(static_cast<const float*>(a.residual) + row * a.residual_ld + d);
            const float4 lo = d < a.dim ? from[0] : make_float4(0, 0, 0, 0), hi = d < a.dim ? from[1] : make_float4(0, 0, 0, 0);
            r[i][0] = lo.x, r[i][1] = lo.y, r[i][2] = lo.z, r[i][3] = lo.w, r[i][4] = hi.x, r[i][5] = hi.y, r[i][6] = hi.z, r[i][7] = hi.w;
        } else {
            widen(d < a.dim ? *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.residual) + row * a.residual_ld + d) : make_uint4(0, 0, 0, 0), r[i]);
        }
    }
    if (a.post) normalize<WAVES, PASSES>(z, per, a.eps, s_sum);
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int d = (i * kThreads + sub) * 8;
        if (d >= a.dim) continue;
        if (a.post) {
#pragma unroll
            for (int j = 0; j < 8; ++j) z[i][j] *= a.post[d + j];
        }
        if (a.gate) {
            float g[8];
            widen(*reinterpret_cast<const uint4*>(a.gate + row * a.gate_ld + d), g);
#pragma unroll
            for (int j = 0; j < 8; ++j) z[i][j] *= g[j];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) r[i][j] += a.scale * z[i][j];
        if constexpr (WIDE) {
            float4* to = reinterpret_cast<float4*>(static_cast<float*>(a.residual_out) + row * a.dim + d);
            to[0] = make_float4(r[i][0], r[i][1], r[i][2], r[i][3]);
            to[1] = make_float4(r[i][4], r[i][5], r[i][6], r[i][7]);
        } else {
            v8b o;
#pragma unroll
            for (int j = 0; j < 8; ++j) o[j] = (__bf16)r[i][j];
            *reinterpret_cast<v8b*>(static_cast<uint16_t*>(a.residual_out) + row * a.dim + d) = o;
        }
    }
    normalize<WAVES, PASSES>(r, per, a.eps, s_sum);
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int d = (i * kThreads + sub) * 8;
        if (d >= a.dim) continue;
        v8b o;
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j] = (__bf16)(r[i][j] * a.weight[d + j]);
        *reinterpret_cast<v8b*>(a.normed + row * a.dim + d) = o;
    }
}

}  // namespace

int launch_add_norm(const AddNormArgs& a, hipStream_t stream) {
    const bool one_wave = a.dim <= 512;
    const int64_t per = one_wave ? 4 : 1, most = ((int64_t)1 << 24) - 1;          // workgroups of a launch: fewer than 2^32 threads
    for (int64_t at = 0; at < a.tokens; at += most * per) {
        const int64_t left = a.tokens - at < most * per ? a.tokens - at : most * per;
        AddNormArgs p = a;
        p.tokens = left;
        p.y += at * a.y_ld;
        const int64_t size = a.wide ? 4 : 2;
        p.residual = static_cast<const uint8_t*>(a.residual) + at * a.residual_ld * size;
        p.residual_out = static_cast<uint8_t*>(a.residual_out) + at * a.dim * size;
        if (p.gate) p.gate += at * a.gate_ld;
        p.normed += at * a.dim;
        const dim3 grid((uint32_t)((left + per - 1) / per)), block(256);
        auto run = [&](auto waves, auto passes) {
            if (a.wide) hipLaunchKernelGGL((add_norm_kernel<decltype(waves)::value, decltype(passes)::value, true>), grid, block, 0, stream, p);
            else hipLaunchKernelGGL((add_norm_kernel<decltype(waves)::value, decltype(passes)::value, false>), grid, block, 0, stream, p);
        };
        std::integral_constant<int, 1> i1;
        std::integral_constant<int, 2> i2;
        std::integral_constant<int, 4> i4;
        std::integral_constant<int, 8> i8;
        if (one_wave) run(i1, i1);
        else if (a.dim <= 2048) run(i4, i1);
        else if (a.dim <= 4096) run(i4, i2);
        else if (a.dim <= 8192) run(i4, i4);
        else run(i4, i8);
    }
    return check_launch();
}

}  // namespace dfp4

// Attention of new tokens over the paged 4-bit cache (formulas and layouts: include/dfp4.h, paged.h).
//
// Rows of a (sequence, KV head) are its new tokens times the query heads of the group, so that they share keys and values.
// With tokens as rows and query rows as columns, softmax statistics of a query are one number a lane: S^T = K Q^T and O^T = V^T P^T, both on
// 16 x 16 x 32 in bf16.  Every DialectFP4 magnitude 0.5 u is an E4M3 number: eight vector instructions make a dword of codes FP8 bytes, and
// these become bf16 with their block's scale in one conversion for two (exact).  A query goes in as it is, a probability as the sum of two bf16
// numbers (one where there are many rows; as two FP8 numbers it has 8 bits down to 2^-19 of the largest and fewer below, which shows where the
// values at the largest are zero).
// (Keys on the block-scaled instruction in FP8, against a query as the sum of two FP8 numbers, take as many matrix clocks and no conversions: 117
// instead of 118 us for 48 sequences of 8192, 511 instead of 540 for 2048 tokens over 16384.  But that instruction leaves a score off by up to 2.8e-4 of
// its largest product, and a query's elements lose bits from 2^-14 of their block's largest on; in bf16 it is off by 2^-21 of sum |q||k|.)
// Both leave in lane (g, c) rows 4 g .. 4 g + 3 of column c, and O^T may take its 128 tokens in any order.  So row 4 g + i of tile t
// (0 .. 7) of S^T is token 32 g + 4 t + i of a step of 128: a lane has the scores of the chunk of 32 whose values it expands and
// whose probabilities it supplies, and nothing moves between lanes.
//
// Values of the sequence's last, incomplete chunk of 32 are bf16 and are multiplied as they are, at the end.
#include <type_traits>
#include <utility>

#include "paged.h"

namespace dfp4 {

namespace {

constexpr int kThreads = 256, kWaves = 4;

typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef __bf16 v2b __attribute__((ext_vector_type(2)));
typedef __bf16 v8b __attribute__((ext_vector_type(8)));

__device__ __forceinline__ float as_f(uint32_t u) { return __builtin_bit_cast(float, u); }
__device__ __forceinline__ uint32_t as_u(float f) { return __builtin_bit_cast(uint32_t, f); }

// E4M3 bytes of the magnitudes 0.5 u of every dialect
struct F8Rows { uint8_t b[kDialects][8]; };
constexpr F8Rows make_f8_rows() {
    F8Rows r{};
    for (int d = 0; d < kDialects; ++d)
        for (int j = 0; j < 8; ++j) {
            const int u = kBook[d][j], top = u >= 8 ? 3 : u >= 4 ? 2 : u >= 2 ? 1 : 0;
            r.b[d][j] = u == 0 ? 0 : (uint8_t)(((top - 1 + 7) << 3) | ((u << (3 - top)) & 7));
        }
    return r;
}
__device__ const F8Rows g_f8_rows = make_f8_rows();

template <class F, int... I>
__device__ __forceinline__ void each(F&& f, std::integer_sequence<int, I...>) { (f(std::integral_constant<int, I>{}), ...); }
template <int N, class F>
__device__ __forceinline__ void each(F&& f) { each(f, std::make_integer_sequence<int, N>{}); }

// N dwords of codes of a scale and a dialect to bf16: fragments of N instructions, elements 8 q .. 8 q + 7 in the q-th
template <int N>
__device__ __forceinline__ void expand_bf16(const uint32_t* w, uint2 row, uint32_t ebyte, v8b* v) {
    const float scale = as_f(ebyte << 23);                          // the conversion goes by the exponent bits (0: 2^-127)
#pragma unroll
    for (int q = 0; q < N; ++q) {
        const uint32_t lo = __builtin_amdgcn_perm(row.y, row.x, w[q] & 0x07070707u) | ((w[q] << 4) & 0x80808080u);
        const uint32_t hi = __builtin_amdgcn_perm(row.y, row.x, (w[q] >> 4) & 0x07070707u) | (w[q] & 0x80808080u);
        const v2b x[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true),
                          __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true)};
        v[q] = __builtin_bit_cast(v8b, x);
    }
}

// eight probabilities as the sum of two bf16 each (the first cut off, the second rounded: 16 bits)
__device__ __forceinline__ void split8(const float* x, v8b& hi, v8b& lo) {
    uint32_t h[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        h[j] = __builtin_amdgcn_perm(as_u(x[2 * j + 1]), as_u(x[2 * j]), 0x07060302u);
        lo[2 * j] = (__bf16)(x[2 * j] - as_f(as_u(x[2 * j]) & 0xffff0000u));
        lo[2 * j + 1] = (__bf16)(x[2 * j + 1] - as_f(as_u(x[2 * j + 1]) & 0xffff0000u));
    }
    hi = __builtin_bit_cast(v8b, make_uint4(h[0], h[1], h[2], h[3]));
}

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
// over the four lanes of a column (16 and 32 apart)
__device__ __forceinline__ float column_max(float v) {
    auto r = __builtin_amdgcn_permlane32_swap(as_u(v), as_u(v), false, false);
    v = fmaxf(as_f(r[0]), as_f(r[1]));
    r = __builtin_amdgcn_permlane16_swap(as_u(v), as_u(v), false, false);
    return fmaxf(as_f(r[0]), as_f(r[1]));
}
__device__ __forceinline__ float column_sum(float v) {
    auto r = __builtin_amdgcn_permlane32_swap(as_u(v), as_u(v), false, false);
    v = as_f(r[0]) + as_f(r[1]);
    r = __builtin_amdgcn_permlane16_swap(as_u(v), as_u(v), false, false);
    return as_f(r[0]) + as_f(r[1]);
}

// over the two lanes of a column of 32 x 32
__device__ __forceinline__ float pair_max(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(as_u(v), as_u(v), false, false);
    return fmaxf(as_f(r[0]), as_f(r[1]));
}
__device__ __forceinline__ float pair_sum(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(as_u(v), as_u(v), false, false);
    return as_f(r[0]) + as_f(r[1]);
}

constexpr float kNone = -__builtin_inff();
constexpr float kLog2e = 1.44269504088896340736f;

// Which keys a block of query rows sees, and how they are split between workgroups: alike in the kernel that adds the parts up.
struct Range {
    int first, end, whole;       // chunks of 32: [first, end), values quantized below `whole`
    int steps, parts;            // of four chunks (16 rows: of whole ones); workgroups that have some
};
__device__ __forceinline__ Range key_range(const AttentionArgs& a, const Sequence& s, int group, int row0) {
    Range r;
    const int rows = s.n * group, last_row = min(row0 + a.rows, rows) - 1;
    const int p_min = s.length - s.n + row0 / group, p_max = s.length - s.n + last_row / group;
    const int t_end = min(p_max + 1, s.length), t_begin = a.window > 0 ? max(0, p_min - a.window + 1) : 0;
    r.first = t_begin / 32;
    r.end = t_end > t_begin && a.paged.n_pages > 0 ? (t_end + 31) / 32 : r.first;
    r.whole = min(r.end, s.length / 32);
    r.steps = (max(a.rows == 16 ? r.whole : r.end, r.first) - r.first + 3) / 4;
    r.parts = min(a.splits, max(1, (r.steps + a.split_steps - 1) / a.split_steps));
    return r;
}

// eight elements of a query row (`flip`: with what signs)
__device__ __forceinline__ v8b query8(const uint16_t* at, bool ok, uint32_t flip) {
    uint4 v = make_uint4(0, 0, 0, 0);
    if (ok) {
        v = *reinterpret_cast<const uint4*>(at);
        v = make_uint4(v.x ^ flip, v.y ^ flip, v.z ^ flip, v.w ^ flip);
    }
    return __builtin_bit_cast(v8b, v);
}

// What turns scores into exponents to base 2.  Where there is neither cap nor bias (nor a scale of zero) a score stays as it is,
// masked or not, until the largest is taken from it (the factor is positive: its sign goes into the query).
// cap tanh(y) = cap - 2 cap / (exp(2 y) + 1), for a score z = cap y.  That is a difference of numbers of size cap, off by about 2^-22 cap.  Up to
// a cap of 128 that is 2^-15 of a probability, which a bf16 result does not show.  Above, a score below |y| = 1/8 is the series
// z (1 - y^2 / 3 + 2 y^4 / 15) instead, off by 17/315 y^6 < 2^-22 of itself, so that it is off by 2^-19 of itself at most whatever the cap is, and
// a cap that no score comes near leaves it alone.  (2048 tokens over 16384, 32 heads of 128: 765 us, with the series 910.)
template <bool EXTRA>
struct Scores {
    float factor, cap, twice, slope;
    uint32_t reach;              // a key so many positions behind the query, or less, is seen
    __device__ __forceinline__ Scores(const AttentionArgs& a)
        : factor(fabsf(a.scale) * kLog2e), cap(a.softcap * kLog2e), twice(a.softcap > 0.0f ? fminf(2.0f / a.softcap, 3e38f) : 0.0f), slope(0.0f),
          reach(a.window > 0 ? (uint32_t)a.window - 1u : 0x7fffffffu) {}
    // N scores whose keys are 0, 1, .. positions on from one `behind` behind the query
    template <int N>
    __device__ __forceinline__ void bend(float* x, int behind) const {
        if constexpr (EXTRA) {
            if (cap > 0.0f) {
                asm volatile("");                                   // one branch
                auto far = [&](float t) { return fmaf(-2.0f * cap, __builtin_amdgcn_rcpf(exp2_(t) + 1.0f), cap); };
                if (cap <= 128.0f * kLog2e) {
                    const float by = fminf(factor * twice, 3e38f);  // (finite: a score may be zero)
#pragma unroll
                    for (int i = 0; i < N; ++i) x[i] = far(x[i] * by);
                } else {
                    constexpr float k = 0.5f / kLog2e;              // y = k t
#pragma unroll
                    for (int i = 0; i < N; ++i) {
                        const float z = x[i] * factor, t = z * twice, t2 = t * t;
                        const float near = fmaf(z, t2 * fmaf(t2, 2.0f / 15.0f * k * k * k * k, -k * k / 3.0f), z);
                        x[i] = fabsf(t) < 0.125f / k ? near : far(t);
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) x[i] *= factor;
            }
            if (slope != 0.0f) {
                const float lean = -slope * (float)behind;
#pragma unroll
                for (int i = 0; i < N; ++i) x[i] += fmaf(slope, (float)i, lean);
            }
        }
    }
    // keys after the query are a large number of positions behind it
    __device__ __forceinline__ float mask(float x, int behind) const { return (uint32_t)behind <= reach ? x : kNone; }
    __device__ __forceinline__ float log2_of(float x) const { return EXTRA ? x : x * factor; }      // of the largest score
    __device__ __forceinline__ float above(float x, float base) const { return EXTRA ? x - base : fmaf(x, factor, -base); }
};
constexpr int kMaxParts = 256;       // the joining kernel has a thread for each
constexpr int kNever = -0x40000000;      // positions behind: a key that is not there

// BYTES from `from` (wave-uniform) to LDS at `to`, lane by lane 16 bytes, by loads that no register receives (loads_of(BYTES) of
// them: what waits for them counts them).  An instruction's offset counts for both addresses.
constexpr int loads_of(uint32_t bytes) { return (int)((bytes + 1023) / 1024); }
template <uint32_t BYTES>
__device__ __forceinline__ void load_to_lds(const uint8_t* from, uint32_t to, uint32_t lane) {
    each<loads_of(BYTES)>([&](auto n_c) {
        constexpr uint32_t at = decltype(n_c)::value * 1024u, whole = at / 4096u * 4096u;
        const uint32_t offset = lane * 16u + whole, lds = to + whole;
        const uint8_t* const base = from;
        if (at + 1024u <= BYTES || lane * 16u < BYTES - at)
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 offset:%3" ::"s"(lds), "v"(offset), "s"(base), "n"(at - whole) : "m0", "memory");
    });
}
// until at most N vector memory operations are under way (those begin and end in order)
template <int N>
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
// until LDS has answered: what it was read for may be overwritten
__device__ __forceinline__ void wait_reads() { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); }

// One workgroup: 16 query rows of a KV head and a contiguous part of their keys; its four waves take steps of 128 keys in turn and
// add up in LDS.  A step's cells come to LDS whole, by loads that bypass the registers: the next step's keys are asked for as soon as
// this one's are multiplied, its values as soon as these are, so that a wave has 9 KiB (head_dim 128) or more under way all the time.
// 48 sequences of about 8192 tokens, 32 heads of 128 on 8 (439 MB), one token each: 118 us = 3.7 TB/s; one token over 131072 (147 MB)
// 35 us and the join 5.  What bounds it: some 1300 vector instructions a wave and step beside 96 matrix instructions, each behind the one
// before with two waves to a SIMD: counters say that vector instructions issue 47 % of the time, matrix instructions are busy 13 %, and a
// wave waits for 30 %.  Codes loaded to registers at the top of a step took 170 us, three waves to a SIMD (168 registers, spilled) 136.
template <int D, bool EXTRA>
__global__ __launch_bounds__(kThreads, 2) void paged_attention_kernel(AttentionArgs a) {
    using C = Cell<D>;
    constexpr int KT = C::KT, NJ = C::NJ;
    constexpr uint32_t kPitch = D + 4;
    __shared__ __attribute__((aligned(16))) uint8_t s_rows[kDialects * 8];
    // a wave's step as it lies in memory: keys of four chunks, then their values; at the end the waves' sums.  Wide heads have one
    // place for both in turn, so that two workgroups fit on a compute unit: one's loads run beside the other's arithmetic.
    constexpr bool kShared = D > 128;
    constexpr uint32_t kValuesAt = kShared ? 0u : 4 * C::kKeys, kStage = 4 * (kShared ? (C::kKeys > C::kValues ? C::kKeys : C::kValues) : C::kKeys + C::kValues),
                       kSums = 16 * kPitch * 4;
    static_assert(kStage >= kSums, "");
    __shared__ __attribute__((aligned(16))) uint8_t s_stage[kWaves * kStage];
    float* const s_o = reinterpret_cast<float*>(s_stage);
    __shared__ float s_m[kWaves][16], s_l[kWaves][16];
    const uint32_t tid = threadIdx.x, lane = tid & 63u, c = lane & 15u, g = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)(tid >> 6));
    const PagedArgs& p = a.paged;
    const int b = (int)(blockIdx.x / (uint32_t)p.kv_heads), kv_head = (int)(blockIdx.x % (uint32_t)p.kv_heads), part = (int)blockIdx.y;
    const int group = a.heads / p.kv_heads;
    const Sequence s = sequence(p, b);
    if (tid < kDialects * 8 / 4) reinterpret_cast<uint32_t*>(s_rows)[tid] = reinterpret_cast<const uint32_t*>(&g_f8_rows.b[0][0])[tid];
    __syncthreads();
    const uint2* const table = reinterpret_cast<const uint2*>(s_rows);
    Scores<EXTRA> rule(a);

    for (int row0 = (int)blockIdx.z * 16; row0 < s.n * group; row0 += (int)gridDim.z * 16) {
        const Range r = key_range(a, s, group, row0);
        if (part >= r.parts) continue;
        const int step0 = part * a.split_steps, step1 = part == r.parts - 1 ? r.steps : min(r.steps, step0 + a.split_steps);
        const int row = row0 + (int)c;
        const bool row_ok = row < s.n * group;
        // positions of the first and the last row
        const int p_min = s.length - s.n + row0 / group, p_max = s.length - s.n + (min(row0 + 16, s.n * group) - 1) / group;
        const int head = kv_head * group + (row_ok ? row % group : 0);
        const int64_t token = s.first + (row_ok ? row / group : 0);
        const int pos = s.length - s.n + (row_ok ? row / group : 0);
        if (EXTRA && a.slopes) rule.slope = a.slopes[head] * kLog2e;

        // a lane's elements of the 128 of kt: as its codes lie (paged.h)
        v8b q[KT][4];
        each<KT>([&](auto kt_c) {
            constexpr int kt = decltype(kt_c)::value, nb = C::blocks(kt);
            const uint16_t* src = a.q + token * a.q_stride + (int64_t)head * a.q_head_stride + kt * 128;
#pragma unroll
            for (int n = 0; n < nb; ++n)
                q[kt][n] = query8(src + (n < 2 ? 16u * g + 8u * n : nb == 3 ? 64u + 8u * g : 64u + 16u * g + 8u * (n - 2)), row_ok, a.scale < 0.0f ? 0x80008000u : 0u);
        });

        v4f o[NJ];
#pragma unroll
        for (int j = 0; j < NJ; ++j) o[j] = v4f{0, 0, 0, 0};
        float m = kNone, l = 0.0f;

        // the running maximum takes in `top`; what was added up so far is scaled to it
        auto raise = [&](float top) {
            const float next = fmaxf(m, rule.log2_of(column_max(top))), base = next == kNone ? 0.0f : next;
            if (__any(next > m)) {
                const float by = exp2_(m - base);
                l *= by;
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[j][i] *= by;
                m = next;
            }
            return base;
        };

        // scores of a tile: the lane's token is at kc's place `token`; scales and dialects of its blocks g / 2 and 2 + g / 2 (of three: 2)
        auto scores = [&](const uint8_t* kc, uint32_t token, const uint32_t (&scale)[KT][2], const uint32_t (&id)[KT][2]) {
            v4f acc = v4f{0, 0, 0, 0};
            each<KT>([&](auto kt_c) {
                constexpr int kt = decltype(kt_c)::value, nb = C::blocks(kt);
                const uint8_t* row = kc + token * (D / 2) + kt * 64;
                uint32_t w[4];
                if constexpr (nb == 4) {
                    const uint4 x = *reinterpret_cast<const uint4*>(row + g * 16u);
                    w[0] = x.x, w[1] = x.y, w[2] = x.z, w[3] = x.w;
                } else {
                    const uint2 x = *reinterpret_cast<const uint2*>(row + g * 8u);
                    w[0] = x.x, w[1] = x.y;
                    if constexpr (nb == 3) w[2] = *reinterpret_cast<const uint32_t*>(row + 32u + g * 4u);
                }
                v8b k[4];
                expand_bf16<2>(w, table[id[kt][0]], scale[kt][0], k);
                if constexpr (nb > 2) expand_bf16<nb - 2>(w + 2, table[id[kt][1]], scale[kt][1], k + 2);
#pragma unroll
                for (int n = 0; n < nb; ++n) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[n], q[kt][n], acc, 0, 0, 0);
            });
            return acc;
        };
        // places of the scales and the dialects of a lane's blocks: `half` 0: g / 2, 1: 2 + g / 2 (of three: 2); dialects of blocks p and p + 2 share a byte
        auto scale_at = [&](int kt, uint32_t half) {
            const uint32_t block = half == 0 ? g >> 1 : C::blocks(kt) == 3 ? 2u : 2u + (g >> 1);
            return C::kKExps + ((c & 3u) * C::NB + 4u * kt + block) * 8u;
        };
        auto id_at = [&](int kt, uint32_t half) { return C::kKIds + ((c & 3u) * C::NP + kt * 2 + (half == 1 && C::blocks(kt) == 3 ? 0u : g >> 1)) * 8u; };

        constexpr int kKeyLoads = 4 * loads_of(C::kKeys), kValueLoads = 4 * loads_of(C::kValues);
        uint8_t* const stage = s_stage + wave * kStage;
        const uint32_t stage_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)stage;
        auto ask = [&](const Four& at, auto values_c) {
            constexpr bool kVal = decltype(values_c)::value;
            constexpr uint32_t kBytes = kVal ? C::kValues : C::kKeys;
            auto one = [&](int64_t cell_at, uint32_t k) {             // (absent ones: the pool's first, so that every step has as many loads)
                load_to_lds<kBytes>(p.pages + (cell_at < 0 ? (int64_t)0 : cell_at) + (kVal ? C::kKeys : 0u), stage_at + (kVal ? kValuesAt : 0u) + k * kBytes, lane);
            };
            one(at.c0, 0), one(at.c1, 1), one(at.c2, 2), one(at.c3, 3);
        };
        Four next = {-1, -1, -1, -1};
        FourPages pages = {};
        if (step0 + wave < step1) {
            const int chunk0 = r.first + 4 * (step0 + wave);
            next = four_cells<D>(p, kv_head, chunk0, r.whole, four_pages_uniform(p, b, chunk0, r.whole));
            pages = four_pages_uniform(p, b, chunk0 + 4 * kWaves, r.whole);
            ask(next, std::false_type{});
            if (!kShared) ask(next, std::true_type{});
        }
        for (int step = step0 + wave; step < step1; step += kWaves) {
            const int chunk0 = r.first + 4 * step;
            const bool more = step + kWaves < step1;
            // absent keys are masked, their values finite
            const Four at = next;
            const bool here = (at.there() >> g) & 1u;
            const uint8_t *kc = stage + (c >> 2) * C::kKeys, *vc = stage + kValuesAt + g * C::kValues - C::kVCodes;
            wait_loads<kShared ? 0 : kValueLoads>();                               // the keys are there

            // ---- scores of 128 keys
            float x[8][4];
            {
                uint2 scales[KT][2], ids[KT][2];
#pragma unroll
                for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                    for (int half = 0; half < (C::blocks(kt) > 2 ? 2 : 1); ++half) {
                        scales[kt][half] = *reinterpret_cast<const uint2*>(kc + scale_at(kt, half));
                        ids[kt][half] = half == 1 && C::blocks(kt) == 4 ? ids[kt][0] : *reinterpret_cast<const uint2*>(kc + id_at(kt, half));
                    }
                each<8>([&](auto t_c) {
                    constexpr int t = decltype(t_c)::value;
                    uint32_t scale[KT][2], id[KT][2];
#pragma unroll
                    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                        for (int half = 0; half < (C::blocks(kt) > 2 ? 2 : 1); ++half) {
                            scale[kt][half] = ((t < 4 ? scales[kt][half].x : scales[kt][half].y) >> (8 * (t & 3))) & 0xffu;
                            id[kt][half] = ((t < 4 ? ids[kt][half].x : ids[kt][half].y) >> (8 * (t & 3) + 4 * half)) & 15u;
                        }
                    const v4f acc = scores(kc, 4u * t + (c & 3u), scale, id);
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[t][i] = acc[i];
                });
            }

            wait_reads();
            if (kShared) ask(at, std::true_type{});
            if (more) {
                next = four_cells<D>(p, kv_head, chunk0 + 4 * kWaves, r.whole, pages);
                pages = four_pages_uniform(p, b, chunk0 + 8 * kWaves, r.whole);
                if (!kShared) ask(next, std::false_type{});
            }

            // ---- softmax
            const int behind = here ? pos - 32 * (chunk0 + (int)g) : kNever;
            rule.template bend<32>(&x[0][0], behind);
            if (!(at.there() == 15u && 32 * chunk0 + 127 <= p_min && p_max - 32 * chunk0 <= (int)rule.reach)) {
                asm volatile("");                                    // a branch, not 32 selections at every step
#pragma unroll
                for (int t = 0; t < 8; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[t][i] = rule.mask(x[t][i], behind - 4 * t - i);
            }
            float top = kNone;
#pragma unroll
            for (int t = 0; t < 8; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) top = fmaxf(top, x[t][i]);
            const float base = raise(top);
            v8b p_hi[4], p_lo[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x[2 * q + i / 4][i % 4] = exp2_(rule.above(x[2 * q + i / 4][i % 4], base));
                    l += x[2 * q + i / 4][i % 4];
                }
                split8(x[2 * q], p_hi[q], p_lo[q]);
            }

            // ---- values
            if (more && !kShared) wait_loads<kKeyLoads>();
            else wait_loads<0>();
            const uint32_t shift = 4u * (c & 1u);
#pragma unroll
            for (int w = 0; w < (NJ + 3) / 4; ++w) {
                uint32_t scales = *reinterpret_cast<const uint32_t*>(vc + C::kVExps + c * C::VE + 4 * w);
                const uint32_t ids = *reinterpret_cast<const uint32_t*>(vc + C::kVIds + (c >> 1) * C::VE + 4 * w) >> shift;
                if (!here) scales = 0x7f7f7f7fu;                    // finite (the probabilities are zero)
#pragma unroll
                for (int jj = 0; jj < 4 && 4 * w + jj < NJ; ++jj) {
                    const int j = 4 * w + jj;
                    v8b v[4];
                    const uint4 w4 = *reinterpret_cast<const uint4*>(vc + C::kVCodes + (16u * j + c) * 16u);
                    expand_bf16<4>(&w4.x, table[(ids >> (8 * jj)) & 15u],
                                (scales >> (8 * jj)) & 0xffu, v);
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        o[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[q], p_hi[q], o[j], 0, 0, 0);
                        o[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[q], p_lo[q], o[j], 0, 0, 0);
                    }
                }
            }
            wait_reads();
            if (more) ask(next, std::integral_constant<bool, !kShared>{});
        }

        // ---- the incomplete chunk: 32 keys, row 4 g + i of tile t (0, 1) is token 8 g + 4 t + i
        const int left = r.end > r.whole ? s.length - 32 * r.whole : 0;
        if (left > 0 && part == r.parts - 1 && wave == (step1 - step0) % kWaves && s.slot >= 0) {
            const uint8_t* kc = cell<D>(p, b, kv_head, r.whole);
            if (kc) {
                float x[8];
                each<2>([&](auto t_c) {
                    constexpr int t = decltype(t_c)::value;
                    const uint32_t token_in = 8u * (c >> 2) + 4u * t + (c & 3u);
                    uint32_t scale[KT][2], id[KT][2];
#pragma unroll
                    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
                        for (int half = 0; half < (C::blocks(kt) > 2 ? 2 : 1); ++half) {
                            scale[kt][half] = kc[scale_at(kt, half) + (token_in >> 2)];
                            id[kt][half] = (kc[id_at(kt, half) + (token_in >> 2)] >> (4 * half)) & 15u;
                        }
                    const v4f acc = scores(kc, token_in, scale, id);
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[4 * t + i] = acc[i];
                });
                float top = kNone;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int in = 8 * (int)g + i, behind = in < left ? pos - 32 * r.whole - in : kNever;
                    rule.template bend<1>(&x[i], behind);
                    x[i] = rule.mask(x[i], behind);
                    top = fmaxf(top, x[i]);
                }
                const float base = raise(top);
                v8b p_hi, p_lo;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x[i] = exp2_(rule.above(x[i], base));
                    l += x[i];
                }
                split8(x, p_hi, p_lo);
                const uint16_t* v = residual<D>(p, s.slot, kv_head, r.whole);
#pragma unroll
                for (int j = 0; j < NJ; ++j) {
                    const uint4 w = *reinterpret_cast<const uint4*>(v + (16u * j + c) * 32u + 8u * g);
                    uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {       // what the slot holds beyond the tokens there are is anything
                        if (8 * (int)g + 2 * i >= left) u[i] = 0;
                        else if (8 * (int)g + 2 * i + 1 >= left) u[i] &= 0xffffu;
                    }
                    const v8b vv = __builtin_bit_cast(v8b, make_uint4(u[0], u[1], u[2], u[3]));
                    o[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, p_hi, o[j], 0, 0, 0);
                    o[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, p_lo, o[j], 0, 0, 0);
                }
            }
        }

        // ---- the four waves together
        l = column_sum(l);
        __syncthreads();                                             // the stages are read
        if (lane < 16) {
            s_m[wave][c] = m;
            s_l[wave][c] = l;
        }
        __syncthreads();
        const float all = fmaxf(fmaxf(s_m[0][c], s_m[1][c]), fmaxf(s_m[2][c], s_m[3][c]));
        const float by = m == kNone ? 0.0f : exp2_(m - all);
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            float4 v = make_float4(o[j][0] * by, o[j][1] * by, o[j][2] * by, o[j][3] * by);
            *reinterpret_cast<float4*>(&s_o[(wave * 16 + c) * kPitch + 16 * j + 4 * g]) = v;
        }
        __syncthreads();
        for (uint32_t i = tid; i < 16u * (D / 8); i += kThreads) {
            const uint32_t rr = i / (D / 8), d = i % (D / 8) * 8u;
            const int at_row = row0 + (int)rr;
            if (at_row >= s.n * group) break;
            const float top = fmaxf(fmaxf(s_m[0][rr], s_m[1][rr]), fmaxf(s_m[2][rr], s_m[3][rr]));
            float sum = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) sum += s_m[w][rr] == kNone ? 0.0f : s_l[w][rr] * exp2_(s_m[w][rr] - top);
            float v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] = 0.0f;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) v[j] += s_o[(w * 16 + rr) * kPitch + d + j];
            }
            const int64_t t = s.first + at_row / group;
            const int h = kv_head * group + at_row % group;
            if (r.parts == 1) {
                const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
                v8b y;
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = (__bf16)(v[j] * inv);
                *reinterpret_cast<v8b*>(a.out + t * a.out_stride + (int64_t)h * a.out_head_stride + d) = y;
                if (a.lse && d == 0) a.lse[t * a.heads + h] = sum > 0.0f ? (top + log2f(sum)) / kLog2e : kNone;
            } else {
                const int64_t slot = (t * a.heads + h) * a.splits + part;
                float4* dst = reinterpret_cast<float4*>(a.partial + slot * D + d);
                dst[0] = make_float4(v[0], v[1], v[2], v[3]);
                dst[1] = make_float4(v[4], v[5], v[6], v[7]);
                if (d == 0) {
                    float* ml = a.partial + (int64_t)p.tokens * a.heads * a.splits * D + slot * 2;
                    ml[0] = top;
                    ml[1] = sum;
                }
            }
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------------------------------------------------------------
// Many query rows (head_dim up to 128): a workgroup expands every step of 128 keys once into LDS, as the operands that all its waves read,
// and each wave does both products for 32 rows, on 32 x 32 x 16: a query is a column again, now of two lanes (h, c).  They hold rows
// 8 a + 4 h + i of a 32 x 32 tile; row 8 a + 4 h + i of a tile of scores is token
// 16 h + 4 a + i of a chunk, so that a lane supplies the probabilities of the 16 tokens whose scores it has, eight to an instruction.
// A chunk is a tile: its cell, and whether it is there, are the same for all lanes.
// Codes of the next step are loaded while this one is multiplied, and expanded into the other half of LDS: one barrier a step.
// The incomplete chunk is part of the last step: its values are stored to LDS as they are.
// A probability is rounded to one bf16 number here, which leaves a result off by 1.4 times its own rounding to bf16 (1.0 with two, as above).
// Two numbers are half again as many matrix instructions, which nothing hides: 2048 tokens over 16384 702 us instead of 530, three chunks of about 310 over
// 4000 with a bias, heads of 64, 106 instead of 93.
// 2048 tokens over 16384, 32 heads of 128 on 8: 520 to 530 us = 0.98 PFLOP/s (a large bf16 library product: 1.25).  16 rows a workgroup took
// 1630.  What bounds it: about 4100 clocks of matrix and 4900 of vector instructions a step and SIMD (40 and 48 %, counters), which hardly overlap, the two
// waves of a SIMD being in the same part of a step (10200 clocks); LDS is read for 26 % of the time, without conflicts.  Operands read one,
// three, five or seven instructions ahead make no difference.  Tried, with keys in FP8: one of the two waves half a step behind
// (registers spilled: 750 us instead of 490), steps of 64 keys (543), two workgroups of half the rows on a compute unit (587), the next step's scores
// between this one's exponentials (560 to 600).
// ---------------------------------------------------------------------------------------------------------------------------------
template <int D>
struct Wide {
    static constexpr int kWaves = 8, kThreads = 64 * kWaves, kRows = 32 * kWaves;
    static constexpr int NC = 4;                                     // chunks of a step
    static constexpr int KS = (D + 63) / 64, DT = D / 32;            // pieces of 64 elements of a key, tiles of V^T
    static constexpr int KP = (NC * KS + kWaves - 1) / kWaves, VP = (NC * DT + kWaves - 1) / kWaves;      // pieces that a wave expands
    static constexpr int KI = D / 16;                                // instructions that add over a key
    static constexpr uint32_t kK = NC * KI * 1024, kV = NC * DT * 2048, kStep = kK + kV;
};

template <int D, bool EXTRA>
__global__ __launch_bounds__(Wide<D>::kThreads, 2) void paged_attention_wide_kernel(AttentionArgs a) {
    using C = Cell<D>;
    using W = Wide<D>;
    constexpr int KS = W::KS, KI = W::KI, DT = W::DT, NC = W::NC, KP = W::KP, VP = W::VP;
    __shared__ __attribute__((aligned(16))) uint8_t s_x[2 * W::kStep];
    __shared__ __attribute__((aligned(16))) uint8_t s_rows[kDialects * 8];
    const uint32_t tid = threadIdx.x, lane = tid & 63u, c = lane & 31u, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane((int)(tid >> 6));
    const PagedArgs& p = a.paged;
    const int b = (int)(blockIdx.x / (uint32_t)p.kv_heads), kv_head = (int)(blockIdx.x % (uint32_t)p.kv_heads), part = (int)blockIdx.y;
    const int group = a.heads / p.kv_heads;
    const Sequence s = sequence(p, b);
    if (tid < kDialects * 8 / 4) reinterpret_cast<uint32_t*>(s_rows)[tid] = reinterpret_cast<const uint32_t*>(&g_f8_rows.b[0][0])[tid];
    __syncthreads();
    const uint2* const table = reinterpret_cast<const uint2*>(s_rows);
    const uint32_t key = 16u * ((c >> 2) & 1u) + 4u * (c >> 3) + (c & 3u);      // token of row c of a tile of scores

    for (int row0 = (int)blockIdx.z * W::kRows; row0 < s.n * group; row0 += (int)gridDim.z * W::kRows) {
        const Range r = key_range(a, s, group, row0);
        if (part >= r.parts) continue;
        const int step0 = part * a.split_steps, step1 = part == r.parts - 1 ? r.steps : min(r.steps, step0 + a.split_steps);
        const int wave_row = row0 + wave * 32, rows = s.n * group;
        // positions of the wave's rows (rows beyond the last have those of the last)
        const int p_min = s.length - s.n + min(wave_row, rows - 1) / group, p_max = s.length - s.n + (min(wave_row + 32, rows) - 1) / group;
        const int row = wave_row + (int)c, held = min(row, rows - 1);
        const int head = kv_head * group + held % group, pos = s.length - s.n + held / group;
        Scores<EXTRA> rule(a);
        if (EXTRA && a.slopes) rule.slope = a.slopes[head] * kLog2e;

        // ---- queries: halves h of all blocks
        v8b q[KI];
        {
            const uint16_t* src = a.q + (int64_t)(s.first + held / group) * a.q_stride + (int64_t)head * a.q_head_stride;
#pragma unroll
            for (int n = 0; n < KI; ++n) q[n] = query8(src + n / 2 * 32 + h * 16u + n % 2 * 8, row < rows, a.scale < 0.0f ? 0x80008000u : 0u);
        }
        v16f o[DT];
#pragma unroll
        for (int j = 0; j < DT; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[j][i] = 0.0f;
        float m = kNone, l = 0.0f;

        // ---- what a wave expands of a step: pieces wave, wave + kWaves, .. of the keys (chunk, ks) and of the values (chunk, tile)
        uint2 k_code[KP][2], v_code[VP];
        uint32_t k_id[KP], k_scale[KP][2], v_id[VP], v_scale[VP];
        uint32_t there = 0;                                          // of the step loaded: bit k: chunk k
        int pages = step0 < step1 ? four_pages(p, b, r.first + NC * step0, r.end) : 0;
        auto load = [&](int step) {
            const int chunk0 = r.first + NC * step;
            // lanes 0 .. 3: whether the chunk is there, and its cell (the pool's first page for one that is not)
            const int chunk = chunk0 + (int)(lane & 3u);
            const bool held_page = (uint32_t)pages < (uint32_t)p.n_pages;
            there = (uint32_t)__ballot(chunk < r.end && held_page && (chunk < r.whole || s.slot >= 0)) & ((1u << NC) - 1u);
            const int number = (int)cell_number(p, kv_head, chunk, place_in_table(p, chunk), held_page ? pages : 0);
            auto place = [&](int k) { return p.pages + (uint64_t)(uint32_t)__builtin_amdgcn_readlane(number, k) * C::kBytes; };
#pragma unroll
            for (int n = 0; n < KP; ++n) {
                const int piece = min(wave + n * W::kWaves, NC * KS - 1), ks = piece % KS;
                const uint8_t* kc = place(piece / KS);
                const uint8_t* at = kc + key * (D / 2);
                // (of a last block alone: the other half is not multiplied, and what is read there is the first's)
                const int u0 = 4 * ks + (int)h, other = 2 * ks + 1 < C::NB, u1 = u0 + 2 * other;
                k_code[n][0] = *reinterpret_cast<const uint2*>(at + C::k_unit(u0) * 8);
                k_code[n][1] = *reinterpret_cast<const uint2*>(at + C::k_unit(u1) * 8);
                const uint8_t* exps = kc + C::kKExps + ((key & 3u) * C::NB + 2 * ks) * 8u + (key >> 2);
                k_scale[n][0] = exps[0];
                k_scale[n][1] = exps[8 * other];
                // dialects of blocks 2 ks and 2 ks + 1: the same half of two bytes (pairs are two blocks apart)
                const uint8_t* ids = kc + C::kKIds + ((key & 3u) * C::NP + ks / 2 * 2) * 8u + (key >> 2);
                k_id[n] = ((uint32_t)ids[0] | (uint32_t)ids[8] << 8) >> (ks & 1 ? 4 : 0);
            }
#pragma unroll
            for (int n = 0; n < VP; ++n) {
                const int piece = min(wave + n * W::kWaves, NC * DT - 1), tile = piece % DT;
                const uint8_t* vc = place(piece / DT);
                const uint32_t d = 32u * tile + c;
                v_code[n] = *reinterpret_cast<const uint2*>(vc + C::kVCodes + d * 16u + h * 8u);
                v_scale[n] = vc[C::kVExps + (d & 15u) * C::VE + (d >> 4)];
                v_id[n] = vc[C::kVIds + ((d & 15u) >> 1) * C::VE + (d >> 4)];
            }
            pages = four_pages(p, b, chunk0 + NC, r.end);
        };
        auto store = [&](uint8_t* to, int step) {
            const int chunk0 = r.first + NC * step;
#pragma unroll
            for (int n = 0; n < KP; ++n) {
                const int piece = wave + n * W::kWaves;
                if (NC * KS % W::kWaves != 0 && piece >= NC * KS) break;
                const int ks = piece % KS;
                v8b k[4];
                expand_bf16<2>(&k_code[n][0].x, table[k_id[n] & 15u], k_scale[n][0], k);
                expand_bf16<2>(&k_code[n][1].x, table[(k_id[n] >> 8) & 15u], k_scale[n][1], k + 2);
                uint8_t* at = to + (piece / KS * KI + ks * 4) * 1024 + lane * 16u;
#pragma unroll
                for (int m = 0; m < 4; ++m)
                    if (4 * ks + m < KI) *reinterpret_cast<v8b*>(at + m * 1024) = k[m];
            }
#pragma unroll
            for (int n = 0; n < VP; ++n) {
                const int piece = wave + n * W::kWaves, chunk = chunk0 + piece / DT;
                if (NC * DT % W::kWaves != 0 && piece >= NC * DT) break;
                const uint32_t d = 32u * (piece % DT) + c;
                v8b v[2];
                // an absent chunk: anything finite (its probabilities are zero)
                const bool here = (there >> (piece / DT)) & 1u;
                expand_bf16<2>(&v_code[n].x, table[(v_id[n] >> (4u * (d & 1u))) & 15u], here ? v_scale[n] : 127u, v);
                if (here && chunk >= r.whole) {
                    const uint16_t* from = residual<D>(p, s.slot, kv_head, chunk) + d * 32u + h * 16u;
                    const int left = s.length - 32 * chunk - 16 * (int)h;
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        const uint4 w = *reinterpret_cast<const uint4*>(from + 8 * q);
                        uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                        for (int k = 0; k < 4; ++k) {                // what the slot holds beyond the tokens there are is anything
                            if (8 * q + 2 * k >= left) u[k] = 0;
                            else if (8 * q + 2 * k + 1 >= left) u[k] &= 0xffffu;
                        }
                        v[q] = __builtin_bit_cast(v8b, make_uint4(u[0], u[1], u[2], u[3]));
                    }
                }
                uint8_t* at = to + W::kK + piece * 2048 + lane * 16u;
                *reinterpret_cast<v8b*>(at) = v[0];
                *reinterpret_cast<v8b*>(at + 1024) = v[1];
            }
        };
        auto work = [&](const uint8_t* from, int step, uint32_t present) {
            const int chunk0 = r.first + NC * step;
            if (wave_row >= rows || 32 * chunk0 > p_max) return;     // no rows, or all of them earlier
            const bool inside = present == (1u << NC) - 1u && 32 * (chunk0 + NC) - 1 <= p_min && chunk0 + NC <= r.whole &&
                                (a.window <= 0 || 32 * chunk0 > p_max - a.window);
            // operands are read three instructions ahead
            auto key_tile = [&](int n) { return *reinterpret_cast<const v8b*>(from + n * 1024 + lane * 16u); };
            auto value_tile = [&](int n) { return *reinterpret_cast<const v8b*>(from + W::kK + n * 1024 + lane * 16u); };
            v16f x[NC];
            v8b k8[4] = {key_tile(0), key_tile(1), key_tile(2)};
            each<NC>([&](auto t_c) {
                constexpr int t = decltype(t_c)::value;
#pragma unroll
                for (int i = 0; i < 16; ++i) x[t][i] = 0.0f;
                each<KI>([&](auto i_c) {
                    constexpr int i = decltype(i_c)::value, n = t * KI + i;
                    if constexpr (n + 3 < NC * KI) k8[(n + 3) & 3] = key_tile(n + 3);
                    x[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k8[n & 3], q[i], x[t], 0, 0, 0);
                });
            });
            v8b v[2][DT];
#pragma unroll
            for (int j = 0; j < DT; ++j) v[0][j] = value_tile(2 * j);
            const int behind = pos - 32 * chunk0 - 16 * (int)h;      // positions that token 16 h of the first chunk is behind the query
            if constexpr (EXTRA) {
#pragma unroll
                for (int t = 0; t < NC; ++t) {
                    float y[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) y[i] = x[t][i];
                    rule.template bend<16>(y, behind - 32 * t);
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[t][i] = y[i];
                }
            }
            if (!inside) {
                asm volatile("");                                    // a branch, not 64 selections at every step
#pragma unroll
                for (int t = 0; t < NC; ++t) {
                    const int from_t = (present >> t) & 1u ? behind - 32 * t : kNever;
#pragma unroll
                    for (int i = 0; i < 16; ++i) x[t][i] = rule.mask(x[t][i], from_t - i);
                }
            }
            float top = kNone;
#pragma unroll
            for (int t = 0; t < NC; ++t)
#pragma unroll
                for (int i = 0; i < 16; ++i) top = fmaxf(top, x[t][i]);
            const float next = fmaxf(m, rule.log2_of(pair_max(top))), base = next == kNone ? 0.0f : next;
            if (__any(next > m)) {
                const float by = exp2_(m - base);
                l *= by;
#pragma unroll
                for (int j = 0; j < DT; ++j)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[j][i] *= by;
                m = next;
            }
            each<NC>([&](auto t_c) {
                constexpr int t = decltype(t_c)::value;
                v8b pr[2];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float e = exp2_(rule.above(x[t][i], base));
                    l += e;
                    pr[i / 8][i % 8] = (__bf16)e;
                }
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    if (2 * t + q + 1 < 2 * NC) {
#pragma unroll
                        for (int j = 0; j < DT; ++j) v[1 - q][j] = value_tile(((t + q) * DT + j) * 2 + 1 - q);
                    }
#pragma unroll
                    for (int j = 0; j < DT; ++j) o[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[q][j], pr[q], o[j], 0, 0, 0);
                }
            });
        };

        __syncthreads();                                             // of the row block before
        if (step0 < step1) {
            load(step0);
            store(s_x, step0);
            uint32_t present = there;
            for (int step = step0; step < step1; ++step) {
                const uint8_t* from = s_x + ((step - step0) & 1) * W::kStep;
                __syncthreads();
                load(step + 1);                                      // (beyond the last: anything)
                work(from, step, present);
                present = there;
                store(s_x + ((step + 1 - step0) & 1) * W::kStep, step + 1);
            }
        }

        const float sum = pair_sum(l);
        if (row < rows) {
            const int64_t t = s.first + row / group;
            // rows 8 a + 4 h + i of a tile: elements of head_dim
            if (r.parts == 1) {
                const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
                uint16_t* dst = a.out + t * a.out_stride + (int64_t)head * a.out_head_stride + 4u * h;
#pragma unroll
                for (int j = 0; j < DT; ++j)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        typedef __bf16 v4b __attribute__((ext_vector_type(4)));
                        v4b y;
#pragma unroll
                        for (int i = 0; i < 4; ++i) y[i] = (__bf16)(o[j][4 * k + i] * inv);
                        *reinterpret_cast<v4b*>(dst + 32 * j + 8 * k) = y;
                    }
                if (a.lse && h == 0) a.lse[t * a.heads + head] = sum > 0.0f ? (m + log2f(sum)) / kLog2e : kNone;
            } else {
                const int64_t slot = (t * a.heads + head) * a.splits + part;
                float* dst = a.partial + slot * D + 4u * h;
#pragma unroll
                for (int j = 0; j < DT; ++j)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        *reinterpret_cast<v4f*>(dst + 32 * j + 8 * k) = v4f{o[j][4 * k], o[j][4 * k + 1], o[j][4 * k + 2], o[j][4 * k + 3]};
                if (h == 0) {
                    float* ml = a.partial + (int64_t)p.tokens * a.heads * a.splits * D + slot * 2;
                    ml[0] = m;
                    ml[1] = sum;
                }
            }
        }
    }
}

// Adds up the parts of a query row.  Parts in their order: the same sum every time.  Few parts: D / 4 threads a row, all of whose
// parts are loaded at once (28000 rows of 64: a wave a row, part after part, 15 us, so 8).
constexpr int kFewParts = 8;
template <int D>
__global__ __launch_bounds__(kThreads) void paged_attention_join_few_kernel(AttentionArgs a) {
    constexpr uint32_t kLanes = D / 4, kRows = kThreads / kLanes;
    const PagedArgs& p = a.paged;
    const uint32_t sub = threadIdx.x % kLanes;
    const int b = (int)blockIdx.x, group = a.heads / p.kv_heads;
    const Sequence s = sequence(p, b);
    if (threadIdx.x >= kLanes * kRows) return;
    for (int row = (int)(blockIdx.y * kRows + threadIdx.x / kLanes); row < s.n * a.heads; row += (int)(gridDim.y * kRows)) {
        const int64_t t = s.first + row / a.heads;
        const int h = row % a.heads, in_group = row / a.heads * group + h % group;
        const int parts = key_range(a, s, group, in_group / a.rows * a.rows).parts;
        if (parts == 1) continue;                       // written by the only part
        const int64_t slot = (t * a.heads + h) * a.splits;
        const float* ml = a.partial + (int64_t)p.tokens * a.heads * a.splits * D + slot * 2;
        float2 w[kFewParts];
        float4 v[kFewParts];
#pragma unroll
        for (int k = 0; k < kFewParts; ++k) {
            const int at = k < parts ? k : 0;
            w[k] = *reinterpret_cast<const float2*>(ml + 2 * at);
            v[k] = *reinterpret_cast<const float4*>(a.partial + (slot + at) * D + 4u * sub);
        }
        float top = kNone, sum = 0.0f;
#pragma unroll
        for (int k = 0; k < kFewParts; ++k) top = fmaxf(top, w[k].x);
        float4 o = make_float4(0, 0, 0, 0);
#pragma unroll
        for (int k = 0; k < kFewParts; ++k) {
            const float by = k < parts && w[k].x != kNone ? exp2_(w[k].x - top) : 0.0f;
            sum += by * w[k].y;
            o.x += by * v[k].x; o.y += by * v[k].y; o.z += by * v[k].z; o.w += by * v[k].w;
        }
        const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
        typedef __bf16 v4b __attribute__((ext_vector_type(4)));
        const v4b y = {(__bf16)(o.x * inv), (__bf16)(o.y * inv), (__bf16)(o.z * inv), (__bf16)(o.w * inv)};
        *reinterpret_cast<v4b*>(a.out + t * a.out_stride + (int64_t)h * a.out_head_stride + 4u * sub) = y;
        if (a.lse && sub == 0) a.lse[t * a.heads + h] = sum > 0.0f ? (top + log2f(sum)) / kLog2e : kNone;
    }
}
// Many parts: one workgroup a row.  D / 4 threads take all of its elements of every (256 * 4 / D)-th part, so that
// 256 parts are read in a few round trips (one wave, part after part: 60 us of 97 for one token over 131072).  The order in which
// parts are added depends on their number alone: the same sum every time.
template <int D>
__global__ __launch_bounds__(kThreads) void paged_attention_join_kernel(AttentionArgs a) {
    constexpr uint32_t kLanes = D / 4, kGroups = kThreads / kLanes;
    __shared__ float s_w[kMaxParts], s_red[kWaves], s_l[kWaves];
    __shared__ __attribute__((aligned(16))) float s_o[kGroups * D];
    const PagedArgs& p = a.paged;
    const uint32_t tid = threadIdx.x;
    const int b = (int)blockIdx.x, group = a.heads / p.kv_heads;
    const Sequence s = sequence(p, b);
    for (int64_t row = blockIdx.y; row < (int64_t)s.n * a.heads; row += gridDim.y) {
        const int64_t t = s.first + row / a.heads;
        const int h = (int)(row % a.heads), in_group = (int)(row / a.heads) * group + h % group;
        const int parts = key_range(a, s, group, in_group / a.rows * a.rows).parts;
        if (parts == 1) continue;                       // written by the only part
        const int64_t slot = (t * a.heads + h) * a.splits;
        const float* ml = a.partial + (int64_t)p.tokens * a.heads * a.splits * D + slot * 2;
        // weights of the parts (at most one a thread)
        float mine = kNone, size = 0.0f;
        if ((int)tid < parts) {
            mine = ml[2 * tid];
            size = ml[2 * tid + 1];
        }
        float top = mine;
#pragma unroll
        for (int k = 1; k < 64; k *= 2) top = fmaxf(top, __shfl_xor(top, k));
        if ((tid & 63u) == 0) s_red[tid >> 6] = top;
        __syncthreads();
        top = fmaxf(fmaxf(s_red[0], s_red[1]), fmaxf(s_red[2], s_red[3]));
        const float by = mine == kNone ? 0.0f : exp2_(mine - top);
        s_w[tid] = by;
        float sum = by * size;
#pragma unroll
        for (int k = 1; k < 64; k *= 2) sum += __shfl_xor(sum, k);
        if ((tid & 63u) == 0) s_l[tid >> 6] = sum;
        __syncthreads();
        sum = s_l[0] + s_l[1] + s_l[2] + s_l[3];
        const uint32_t d = tid % kLanes, first = tid / kLanes;
        float4 o = make_float4(0, 0, 0, 0);
        if (first < kGroups) {
#pragma unroll 4
            for (int k = (int)first; k < parts; k += (int)kGroups) {
                const float4 v = *reinterpret_cast<const float4*>(a.partial + (slot + k) * D + 4u * d);
                const float w = s_w[k];
                o.x += w * v.x; o.y += w * v.y; o.z += w * v.z; o.w += w * v.w;
            }
            *reinterpret_cast<float4*>(&s_o[first * D + 4u * d]) = o;
        }
        __syncthreads();
        const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
        if (tid < (uint32_t)D) {
            float v = 0.0f;
#pragma unroll
            for (uint32_t k = 0; k < kGroups; ++k) v += s_o[k * D + tid];
            reinterpret_cast<__bf16*>(a.out)[t * a.out_stride + (int64_t)h * a.out_head_stride + tid] = (__bf16)(v * inv);
        }
        if (a.lse && tid == 0) a.lse[t * a.heads + h] = sum > 0.0f ? (top + log2f(sum)) / kLog2e : kNone;
        __syncthreads();
    }
}

struct Split {
    int rows, blocks;            // query rows of a workgroup, workgroups along them
    int splits, steps;           // workgroups along the keys, steps of 128 keys of each
};
// How many parts the keys are split in, from what the host knows.  A workgroup costs what a round of 512 keys costs, or two, before its
// first; `at_once` of them run at a time.  Of the numbers of parts that fill the chip once, twice, three or four times the one whose
// (times) x (rounds + that) is least.
Split choose_split(const dfp4_cache& cache, const dfp4_batch& batch, int64_t heads, int64_t window) {
    const int64_t new_tokens = likely_new(batch);
    int64_t most = batch.table_width * cache.page_tokens;
    if (batch.max_length > 0 && batch.max_length < most) most = batch.max_length;
    const int64_t new_rows = new_tokens * (heads / cache.kv_heads);
    // In rounds of 512 keys of 16 rows.  The wide kernel expands keys once for 256 rows but wants a compute unit for itself: 8 KV heads,
    // us wide / 16 rows a workgroup, heads of 64, 96 and 128: 64 rows of 16 sequences of 4000 tokens 43 / 39, 51 / 47, 55 / 56, 96 rows 45 / 57, 55 / 76,
    // 58 / 93; 96 rows of 4 sequences (1536 rounds) 20 / 24, 25 / 29, 27 / 34; 512 rows of one sequence of 2000 (1024 rounds) 22 / 18, 28 / 22, 31 / 26,
    // 1024 rows (2048) 25 / 21, 31 / 27, 36 / 32, 2048 rows (4096) 30 / 33, 38 / 45, 41 / 54.  One KV head of 128: 96 x 8 rows of 4 sequences (1536) 33 / 34,
    // 192 rows of 16 (1536) 29 / 34, 160 rows of 48 of 1000 (960) 29 / 20.  Heads above 128 leave
    // it no registers (a version with half the waves took 729 us for 2048 rows of 4 sequences, heads of 256; 609 so).
    const int64_t keys = window > 0 && window + new_tokens < most ? window + new_tokens : most;
    // (its workgroups of 512 threads: fewer than 2^32 threads a launch.)
    const bool wide = cache.head_dim <= 128 && new_rows > 64 && batch.batch * cache.kv_heads < (int64_t)1 << 23 &&
                      batch.batch * cache.kv_heads * ((new_rows + 15) / 16) * ((keys + 511) / 512) > 5 * (int64_t)device_cu_count();
    const int64_t rows = wide ? 256 : 16;
    int64_t blocks = (new_rows + rows - 1) / rows;
    if (batch.max_new == 0) {
        // one sequence may have most of the rows: workgroups for as many as it could have, of which those without rows cost 0.6 ns each
        const int64_t could = (batch.tokens * (heads / cache.kv_heads) + rows - 1) / rows, cheap = (wide ? 16384 : 4096) / (batch.batch * cache.kv_heads);
        const int64_t more = could < cheap ? could : cheap;
        if (more > blocks) blocks = more;
    }
    if (blocks > 65535) blocks = 65535;
    const int64_t seen = (rows + heads / cache.kv_heads - 1) / (heads / cache.kv_heads) + window + 31;      // by a block of rows, with a window
    if (window > 0 && seen < most) most = seen;
    const int64_t rounds = most > 0 ? (most + 511) / 512 : 1;
    // (sequences have fewer new tokens than the one with most: the rows of all of them, and a block begun for each, bound the blocks too)
    const int64_t all = (batch.tokens * (heads / cache.kv_heads) + rows - 1) / rows + batch.batch;
    const int64_t groups = cache.kv_heads * (all < batch.batch * blocks ? all : batch.batch * blocks);
    const int64_t at_once = (int64_t)device_cu_count() * (wide ? 1 : 2), before = wide ? 1 : 2;
    int64_t best = 1, cost = ((groups + at_once - 1) / at_once) * (before + rounds);
    for (int64_t times = 1; times <= 4; ++times) {
        int64_t want = times * at_once / groups;
        if (want > rounds) want = rounds;
        if (want > kMaxParts) want = kMaxParts;
        if (want < 2) continue;
        const int64_t c = ((groups * want + at_once - 1) / at_once) * (before + (rounds + want - 1) / want);
        if (c < cost) best = want, cost = c;
    }
    const int64_t per = (rounds + best - 1) / best;
    return Split{(int)rows, (int)blocks, (int)((rounds + per - 1) / per), (int)(per * 4)};
}

}  // namespace

int paged_attention_rows(const dfp4_cache& cache, const dfp4_batch& batch, int64_t heads, int64_t window) {
    return choose_split(cache, batch, heads, window).rows;
}

size_t paged_attention_workspace_bytes(const dfp4_cache& cache, const dfp4_batch& batch, int64_t heads, int64_t window) {
    const Split sp = choose_split(cache, batch, heads, window);
    return sp.splits > 1 ? (size_t)(batch.tokens * heads * sp.splits) * (size_t)(cache.head_dim + 2) * 4u : 0;
}

int launch_paged_attention(AttentionArgs a, const dfp4_cache& cache, const dfp4_batch& batch, hipStream_t stream) {
    const Split sp = choose_split(cache, batch, a.heads, a.window);
    a.splits = sp.splits;
    a.split_steps = sp.steps;
    a.rows = sp.rows;
    const dim3 grid((uint32_t)(batch.batch * cache.kv_heads), (uint32_t)sp.splits, (uint32_t)sp.blocks);
    const bool extra = a.softcap > 0.0f || a.slopes || a.scale == 0.0f;
    with_head_dim(cache.head_dim, [&](auto d) {
        constexpr int kD = decltype(d)::value;
        if constexpr (kD <= 128) {
            if (sp.rows > 16) {
                if (extra) hipLaunchKernelGGL((paged_attention_wide_kernel<kD, true>), grid, dim3(Wide<kD>::kThreads), 0, stream, a);
                else hipLaunchKernelGGL((paged_attention_wide_kernel<kD, false>), grid, dim3(Wide<kD>::kThreads), 0, stream, a);
            }
        }
        if (sp.rows == 16) {
            if (extra) hipLaunchKernelGGL((paged_attention_kernel<kD, true>), grid, dim3(kThreads), 0, stream, a);
            else hipLaunchKernelGGL((paged_attention_kernel<kD, false>), grid, dim3(kThreads), 0, stream, a);
        }
        if (sp.splits > 1) {
            const int64_t rows = likely_new(batch) * a.heads;
            const int64_t blocks = sp.splits <= kFewParts ? (rows + 1024 / kD - 1) / (1024 / kD) : rows;
            const dim3 join((uint32_t)batch.batch, (uint32_t)(blocks < 65535 ? blocks : 65535));
            if (sp.splits <= kFewParts) hipLaunchKernelGGL((paged_attention_join_few_kernel<kD>), join, dim3(kThreads), 0, stream, a);
            else hipLaunchKernelGGL((paged_attention_join_kernel<kD>), join, dim3(kThreads), 0, stream, a);
        }
    });
    return check_launch();
}

}  // namespace dfp4
